"""Rows and states further than 2^31 elements from the first: the same bits as from a compact copy."""
import numpy as np
import pytest
import torch

import paper_2511_00413_amd as T

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def far(rows, width, step):
    """[rows, width] bf16 rows `step` elements apart, and the same numbers close together."""
    assert (rows - 1) * step > 1 << 31
    g = torch.Generator(device="cuda").manual_seed(rows)
    close = torch.randn(rows, width, generator=g, device="cuda").to(BF16)
    buf = torch.empty((rows - 1) * step + width, dtype=BF16, device="cuda").as_strided((rows, width), (step, 1))
    buf.copy_(close)
    return buf, close


def test_logprob_entropy():
    z, close = far(4, 5003, 800_000_008)
    y = torch.tensor([0, 5002, 77, -1], dtype=torch.int32, device="cuda")
    got, want = T.tree_logprob_entropy(z, y, top_k=7), T.tree_logprob_entropy(close, y, top_k=7)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    d = torch.ones(4, device="cuda")
    want = T.tree_logprob_entropy_bwd(close, y, got[2], got[1], d, d)
    assert torch.equal(T.tree_logprob_entropy_bwd(z, y, got[2], got[1], d, d, out=z), want) and torch.equal(z, want)


def test_rope_axes():
    x, close = far(5, 3 * 64, 600_000_000)
    pos = torch.arange(15, dtype=torch.int32, device="cuda").view(3, 5)
    want = T.tree_rope_axes(close.view(5, 3, 64), pos, (12, 10, 10))
    out = x.unflatten(1, (3, 64))
    assert torch.equal(T.tree_rope_axes(out, pos, (12, 10, 10)), want)
    T.tree_rope_axes(out, pos, (12, 10, 10), out=out)
    assert torch.equal(out, want)


def test_scan():
    n, ch, m = 4800, 192, 8
    rows, close = far(n, 4 * ch + 2 * m, 500_000)
    plan = T.tree_gdn_plan(np.array([-1, 0, 0, 2], np.int32), np.array([900, 1100, 700, n - 2700], np.int32))
    g = torch.Generator(device="cuda").manual_seed(1)
    A, D = -torch.rand(ch, m, generator=g, device="cuda") - 0.1, torch.ones(ch, device="cuda")

    def calls(t):
        x, dt, z, dy, B, C = t.split([ch, ch, ch, ch, m, m], 1)
        B, C = B.unflatten(1, (1, m)), C.unflatten(1, (1, m))
        k = {"D": D, "z": z, "dt_bias": D}
        return (T.tree_scan_fwd(x, dt, A, B, C, plan, **k), *(t for t in T.tree_scan_bwd(x, dt, A, B, C, dy, plan, **k) if t is not None))

    for i, (a, b) in enumerate(zip(calls(rows), calls(close))):
        assert torch.equal(a, b), i
    x, dt, z, _, B, C = close.split([ch, ch, ch, ch, m, m], 1)
    out = rows[:, 3 * ch:4 * ch]
    T.tree_scan_fwd(x, dt, A, B.unflatten(1, (1, m)), C.unflatten(1, (1, m)), plan, D=D, z=z, dt_bias=D, out=out)
    assert torch.equal(out, calls(close)[0])


def test_states_of_a_long_list():
    slots, ch, m, n = 17_000, 8192, 16, 33
    state = torch.empty(slots, ch, m, device="cuda")
    assert state.numel() > 1 << 31
    g = torch.Generator(device="cuda").manual_seed(2)
    index = torch.randperm(slots - 1, generator=g, device="cuda", dtype=torch.int32)[:n].contiguous()
    index[0], index[1] = slots - 1, slots
    used = torch.randn(n, ch, m, generator=g, device="cuda")
    state[index[index < slots].long()] = used[index < slots]
    used[1] = 0
    r = lambda *s: torch.randn(s, generator=g, device="cuda").to(BF16)          # noqa: E731
    x, dt, B, C, A = r(n, ch), r(n, ch), r(n, 1, m), r(n, 1, m), -torch.rand(ch, m, generator=g, device="cuda")
    for a, b in zip(T.tree_scan_step(x, dt, A, B, C, state, index=index), T.tree_scan_step(x, dt, A, B, C, used)):
        assert torch.equal(a, b)
    del state
    slots, taps = 90_000, 4
    state = torch.empty(slots, taps - 1, ch, dtype=BF16, device="cuda")
    assert state.numel() > 1 << 31
    index[0], index[1] = slots - 1, -1
    index[2:] = torch.randperm(slots - 1, generator=g, device="cuda", dtype=torch.int32)[:n - 2]
    used = r(n, taps - 1, ch)
    state[index[index >= 0].long()] = used[index >= 0]
    used[1] = 0
    w = torch.randn(ch, taps, generator=g, device="cuda")
    for a, b in zip(T.tree_conv_step(x, state, w, index=index), T.tree_conv_step(x, used, w)):
        assert torch.equal(a, b)
