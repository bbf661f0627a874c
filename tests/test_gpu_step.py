"""Single-token scan and convolution from saved states, against the recurrence in float64, and against the whole-tree calls."""
import numpy as np
import pytest
import torch

import paper_2511_00413_amd as T
import scan_ref as R
from test_gpu_scan import HALF, cuda, f64, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,slots,ch,m,groups,fused,gated", [
    (1, 1, 64, 16, 1, False, True), (5, 3, 70, 16, 1, True, False), (33, 9, 256, 8, 4, False, True), (7, 40, 129, 4, 1, False, True),
    (40000, 2, 4, 4, 1, False, False)])
def test_scan_step(rows, slots, ch, m, groups, fused, gated, dtype):
    print(f"[case] scan_step rows={rows} slots={slots} channels={ch} states={m} groups={groups} {dtype}", flush=True)
    k = make(rows, ch, m, groups, dtype, rows + ch, gated=gated, fused=fused)
    g = torch.Generator().manual_seed(1)
    state = torch.randn((slots, ch, m), generator=g)
    index = torch.randint(0, slots, (rows,), generator=g, dtype=torch.int32)
    if rows > 4:
        index[0], index[1], index[2] = -1, slots, 2 ** 31 - 1        # starts of sequences
    d = cuda(k)
    y, out = T.tree_scan_step(d["x"], d["dt"], d["A"], d["B"], d["C"], state.cuda(), index=index.cuda(), D=d["D"], z=d["z"],
                              dt_bias=d["dt_bias"])
    torch.cuda.synchronize()
    ins = f64(k)
    per = ch // groups
    delta = R.softplus(ins["dt"] + ins["dt_bias"])
    ok = (index >= 0) & (index < slots)
    before = torch.where(ok[:, None, None], state.double()[index.clamp(0, slots - 1).long()], torch.zeros(1, dtype=torch.float64))
    u = (delta * ins["x"])[..., None] * ins["B"].repeat_interleave(per, 1)
    kept = torch.exp(delta[..., None] * ins["A"]) * before
    h = kept + u
    Cc = ins["C"].repeat_interleave(per, 1)
    yy = (Cc * h).sum(-1) + ins["D"] * ins["x"]
    size = (Cc.abs() * (kept.abs() + u.abs())).sum(-1) + (ins["D"] * ins["x"]).abs()
    if gated:
        yy, size = yy * ins["z"] * torch.sigmoid(ins["z"]), size * ins["z"].abs()
    R.assert_close(out, h, (kept.abs() + u.abs()).numpy(), 1, 1, 0, "state")
    R.assert_close(y, yy, size.numpy(), 1, m, HALF[dtype], "y")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,slots,ch,taps,silu", [(1, 1, 4, 4, True), (9, 4, 100, 3, False), (40, 3, 1028, 2, True), (33000, 2, 8, 4, True)])
def test_conv_step(rows, slots, ch, taps, silu, dtype):
    """Four products, their sum, a sigmoid (two units) and a product: 16 units of 2^-24 of the terms' absolute values (|silu'| <=
    1.1), and the rounding of the result."""
    print(f"[case] conv_step rows={rows} slots={slots} channels={ch} taps={taps} {dtype}", flush=True)
    g = torch.Generator().manual_seed(rows)
    buf = torch.randn((rows, ch + 8), generator=g).to(dtype)
    x = buf[:, 4:4 + ch]
    state = torch.randn((slots, taps - 1, ch), generator=g).to(dtype)
    w, b = torch.randn((ch, taps), generator=g), torch.randn(ch, generator=g)
    index = torch.randint(0, slots, (rows,), generator=g, dtype=torch.int32)
    if rows > 4:
        index[0], index[1] = -5, slots
    y, out = T.tree_conv_step(buf.cuda()[:, 4:4 + ch], state.cuda(), w.cuda(), b.cuda(), index=index.cuda(), silu=silu)
    torch.cuda.synchronize()
    ok = (index >= 0) & (index < slots)
    hist = torch.where(ok[:, None, None], state[index.clamp(0, slots - 1).long()], torch.zeros(1, dtype=dtype))
    window = torch.cat([hist, x[:, None]], 1)
    assert torch.equal(out.cpu(), window[:, 1:])
    terms = window.double() * w.T.double()
    pre = terms.sum(1) + b.double()
    yy = pre * torch.sigmoid(pre) if silu else pre
    err = 1.1 * 16 * 2.0 ** -24 * (terms.abs().sum(1) + b.abs()) + HALF[dtype] * yy.abs()
    assert ((y.cpu().double() - yy).abs() <= err + 1e-37).all()


def test_in_place():
    k = make(6, 64, 16, 1, torch.bfloat16, 2)
    d = cuda(k)
    args, layer = [d[i] for i in ("x", "dt", "A", "B", "C")], {i: d[i] for i in ("D", "z", "dt_bias")}
    state = torch.randn(8, 64, 16, device="cuda")
    want = T.tree_scan_step(*args, state, **layer)
    keep = state.clone()
    y, s = T.tree_scan_step(*args, state, state_out=state, **layer)
    assert s is state and torch.equal(y, want[0]) and torch.equal(state[:6], want[1]) and torch.equal(state[6:], keep[6:])
    cs, w = torch.randn(8, 3, 64, device="cuda", dtype=torch.bfloat16), torch.randn(64, 4, device="cuda")
    want = T.tree_conv_step(d["x"], cs, w)
    keep = cs.clone()
    y, s = T.tree_conv_step(d["x"], cs, w, state_out=cs)
    assert torch.equal(y, want[0]) and torch.equal(cs[:6], want[1]) and torch.equal(cs[6:], keep[6:])
    idx = torch.zeros(6, dtype=torch.int32, device="cuda")
    with pytest.raises(T.TreeTrainError):
        T.tree_scan_step(*args, state[:6], index=idx, state_out=state[:6], **layer)
    with pytest.raises(T.TreeTrainError):
        T.tree_conv_step(d["x"], cs[:6], w, index=idx, state_out=cs[:6])
    e = T.tree_scan_step(*(t if i == 2 else t[:0] for i, t in enumerate(args)), state, index=idx[:0])
    assert e[0].shape == (0, 64) and e[1].shape == (0, 64, 16)
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_steps_go_on_from_a_tree(dtype):
    """Three rollouts of four tokens go on from two nodes of a tree: token by token, and as longer branches of the tree."""
    ch, m, taps, more = 128, 16, 4, 4
    parent, seg = [-1, 0, 0], [30, 70, 2]
    starts = [1, 2, 1]                                        # node that each rollout goes on from
    n = sum(seg)
    g = torch.Generator().manual_seed(8)
    k = make(n + 3 * more, ch, m, 1, dtype, 5)
    d = cuda(k)
    w, b = torch.randn((ch, taps), generator=g).cuda(), torch.randn(ch, generator=g).cuda()
    layer = {i: d[i] for i in ("D", "dt_bias")}
    # whole: the tree with the rollouts as branches; tokens n + 4 r + i are rollout r's
    big_parent, big_seg = parent + starts, seg + [more] * 3
    meta = T.tree_build_meta(big_parent, big_seg)
    first = {int(node): int(meta.node_start[i]) for i, node in enumerate(meta.dfs_order)}
    src = np.concatenate([first[i] + np.arange(big_seg[i]) for i in range(6)])       # place of every token in DFS order
    order = torch.from_numpy(np.argsort(src)).cuda()
    place = torch.from_numpy(src).cuda()
    full = {i: d[i][order].contiguous() for i in ("x", "dt", "z", "B", "C")}
    conv = T.tree_conv_fwd(full["x"], w, b, torch.from_numpy(meta.tok_pred).cuda())
    y = T.tree_scan_fwd(conv, full["dt"], d["A"], full["B"], full["C"], T.tree_gdn_plan(big_parent, big_seg), z=full["z"], **layer)[place]
    conv = conv[place]
    # the tree alone, then token by token
    small = T.tree_build_meta(parent, seg)
    pred = torch.from_numpy(small.tok_pred).cuda()
    c0 = T.tree_conv_fwd(d["x"][:n].contiguous(), w, b, pred)
    _, states = T.tree_scan_fwd(c0, d["dt"][:n], d["A"], d["B"][:n], d["C"][:n], T.tree_gdn_plan(parent, seg, [1, 2]), z=d["z"][:n],
                                return_states=True, **layer)
    ends = [99, 101]                                          # last tokens of the two nodes
    hist = []
    for e in ends:
        rows = [e]
        while len(rows) < taps - 1:
            rows.append(int(small.tok_pred[rows[-1]]))
        hist.append(d["x"][torch.tensor(rows[::-1], device="cuda")])
    conv_state, index = torch.stack(hist), torch.tensor([s - 1 for s in starts], dtype=torch.int32, device="cuda")
    for i in range(more):
        rows = torch.tensor([n + more * r + i for r in range(3)], device="cuda")
        u, conv_state = T.tree_conv_step(d["x"][rows], conv_state, w, b, index=index)
        out, states = T.tree_scan_step(u, d["dt"][rows], d["A"], d["B"][rows], d["C"][rows], states, index=index, z=d["z"][rows], **layer)
        index = None
        half = HALF[dtype]
        assert ((u.double() - conv[rows].double()).abs() <= 2 * half * conv[rows].double().abs() + 1e-4).all()
        # both rest on the same convolution up to its rounding; the states differ by 100 decays' roundings
        tol = 4 * half + 500 * 2.0 ** -24
        assert (out.double() - y[rows].double()).norm() <= tol * y[rows].double().norm()
    torch.cuda.synchronize()
