"""Calls on a given stream while another is current: their memory is the given stream's own, whatever the current one still has queued."""
import pytest
import torch

from test_gpu_policy_step import all_calls

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_memory_that_the_current_stream_has_dropped_but_not_read_yet(dtype):
    """Tensors of the sizes of all outputs are dropped while their copies are still queued behind long products; the given stream is idle
    and runs ahead of them."""
    _, step = all_calls(dtype)
    want = [t.clone() for t in step() if t is not None]
    a = torch.randn(4096, 4096, device="cuda")
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    dropped = [torch.full_like(t, 3) for t in want]
    at = {t.data_ptr() for t in dropped if t.numel()}
    torch.cuda.synchronize()
    for _ in range(16):
        a = a @ a * 1e-2
    kept = [t.clone() for t in dropped]
    del dropped
    got = [t for t in step(stream=other) if t is not None]
    assert not at & {t.data_ptr() for t in got}
    torch.cuda.synchronize()
    for i, (t, g, w) in enumerate(zip(kept, got, want)):
        assert (t == 3).all() and torch.equal(g, w), i


def test_outputs_of_a_given_stream_stay_while_the_current_one_reads_them():
    """An output of the given stream, dropped while the current stream still has to read it, is not that stream's to fill yet."""
    _, step = all_calls(torch.float32)
    want = [t.clone() for t in step() if t is not None]
    a = torch.randn(4096, 4096, device="cuda")
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = [t for t in step(stream=other) if t is not None]
    torch.cuda.current_stream().wait_stream(other)
    for _ in range(16):
        a = a @ a * 1e-2
    kept = [t.clone() for t in got]
    sizes = [t.shape for t in got]
    del got
    with torch.cuda.stream(other):
        filled = [torch.full(s, float("nan"), device="cuda") for s in sizes]
    torch.cuda.synchronize()
    assert len(filled) == len(kept)
    for i, (t, w) in enumerate(zip(kept, want)):
        assert torch.equal(t, w), i
