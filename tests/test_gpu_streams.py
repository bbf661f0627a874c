"""Calls on a given stream while another is current: their memory is the given stream's own, whatever the current one still has queued."""
import pytest
import torch

import paper_2511_00413_amd as T
import workloads as W
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


def tree_calls():
    """Rotation, attention (whole and partitioned), loss, convolution and gated delta rule of one small tree; returns a step."""
    tree = W.random_tree(31, n_nodes=9, lo=20, hi=90)
    meta = T.tree_build_meta(tree.parent, tree.seg_len, tree.trained)
    n = meta.n_tokens
    dev = lambda a: torch.from_numpy(a).cuda()                                  # noqa: E731
    g = torch.Generator().manual_seed(2)
    r = lambda *s, t=torch.bfloat16: torch.randn(s, generator=g).to(t).cuda()   # noqa: E731
    q, k, v, do = r(n, 4, 64), r(n, 2, 64), r(n, 2, 64), r(n, 4, 64)
    mask, pos, pred, w = [dev(a) for a in (meta.kend, meta.ktile_kend_min, meta.ktile_kend_max)], dev(meta.tok_pos), dev(meta.tok_pred), dev(meta.tok_weight)
    parts = T.tree_partition_plan(tree.parent, tree.seg_len, 200).to_device()
    logits, target = r(n, 1000), torch.randint(0, 1000, (n,), generator=g, dtype=torch.int32).cuda()
    x, cw, cb, dy = r(n, 128), r(128, 4, t=torch.float32), r(128, t=torch.float32), r(n, 128)
    cplan, gplan = T.tree_conv_plan(meta.tok_pred, 4).to_device(), T.tree_gdn_plan(tree.parent, tree.seg_len).to_device()
    sq, sk, sv, sdo = (torch.nn.functional.normalize(r(n, h, 128).float(), dim=-1).bfloat16() for h in (1, 1, 2, 2))
    decay, beta = -torch.rand(n, 2, generator=g).cuda(), torch.rand(n, 2, generator=g).cuda()
    dx, dw, db = torch.empty_like(x), torch.empty_like(cw), torch.empty_like(cb)      # (given by the caller)

    def step(stream=None):
        s = {"stream": stream}
        out = [T.tree_rope(q, pos, **s)]
        o, lse = T.tree_attn_fwd(q, k, v, *mask, **s)
        out += [o, lse, *T.tree_attn_bwd(q, k, v, *mask, o, do, lse, **s)]
        o, lse = T.tree_attn_partitioned_fwd(q, k, v, parts, **s)
        out += [o, lse, *T.tree_attn_partitioned_bwd(q, k, v, parts, o, do, lse, **s)]
        lp = T.tree_weighted_logprob(logits, target, w, **s)
        out += [*lp, T.tree_weighted_logprob_bwd(logits, target, w, lp[1], **s), *T.tree_weighted_logprob_fwd_bwd(logits, target, w, **s)]
        out += [T.tree_conv_fwd(x, cw, cb, pred, **s), *T.tree_conv_bwd(x, cw, cb, pred, dy, cplan, **s)]
        assert T.tree_conv_bwd_static(x, cw, cb, pred, dy, cplan, dx, dw, db, **s) is None
        out += [dx, dw, db, T.tree_gdn_fwd(sq, sk, sv, decay, beta, gplan, **s), *T.tree_gdn_bwd(sq, sk, sv, decay, beta, sdo, gplan, **s)]
        return out
    return step


def test_the_other_calls_on_a_given_stream():
    """As the first test, for the calls on trees that allocate their outputs and workspaces."""
    step = tree_calls()
    want = [t.clone() for t in step()]
    a = torch.randn(4096, 4096, device="cuda")
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    dropped = [torch.full_like(t, 3) for t in want]
    torch.cuda.synchronize()
    for _ in range(16):
        a = a @ a * 1e-2
    kept = [t.clone() for t in dropped]
    del dropped
    got = step(stream=other)
    torch.cuda.synchronize()
    for i, (t, g, w) in enumerate(zip(kept, got, want)):
        assert (t == 3).all() and torch.equal(g, w), i
