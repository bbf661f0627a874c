"""Selective scan with tree state routing, forward and backward, against the token recurrence in float64 and its automatic
derivative.  The bounds are derived in scan_ref."""
import numpy as np
import pytest
import torch

import paper_2511_00413_amd as T
import scan_ref as R
import workloads as W

pytestmark = pytest.mark.gpu
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def make(n, ch, m, groups, dtype, seed, gated=True, skip=True, bias=True, fused=False):
    """Inputs on the CPU, rounded to their type; as the slices of one projection when fused."""
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=g)                                # noqa: E731
    k = {"A": -(torch.arange(1, m + 1).float() * torch.exp(0.2 * rnd(ch, m))), "D": 1 + 0.1 * rnd(ch) if skip else None,
         "dt_bias": -4 + 2 * torch.rand(ch, generator=g) if bias else None}
    widths = [ch, ch, ch, groups * m, groups * m]
    if fused:
        pad = -sum(widths) % 4 + 4
        parts = rnd(n, sum(widths) + pad).to(dtype)[:, :sum(widths)].split([widths[i] for i in (3, 4, 0, 1, 2)], 1)
        parts = [parts[2], parts[3], parts[4], parts[0], parts[1]]
    else:
        parts = [rnd(n, w).to(dtype) for w in widths]
    x, dt, z, B, C = parts
    k.update(x=x, dt=dt, z=z if gated else None, B=B.unflatten(1, (groups, m)), C=C.unflatten(1, (groups, m)))
    return k


def cuda(k):
    """On the GPU, slices of a buffer staying slices of a copy of it."""
    seen, out = {}, {}
    for name, t in k.items():
        if t is None:
            out[name] = None
            continue
        base = t._base if t._base is not None else t
        root = seen.setdefault(base.data_ptr(), base.cuda())
        out[name] = root.as_strided(t.shape, t.stride(), t.storage_offset())
    return out


def f64(k):
    return {name: None if t is None else t.double() for name, t in k.items()}


TREES = {
    "one": ([-1], [1]), "two_roots": ([-1, -1], [1, 3]), "chunk": ([-1], [64]), "chunk_and_one": ([-1], [65]),
    "long": ([-1], [331]), "fork": ([-1, 0, 0], [64, 65, 1]), "empty_nodes": ([-1, 0, 1, 1, 0, -1], [5, 0, 70, 9, 0, 2]),
    "empty_root": ([-1, 0, 0], [0, 7, 130]), "worked": ([-1, 0, 1, 1, 0], [64, 48, 32, 40, 56]),
}


def tree_of(name):
    if name in TREES:
        return TREES[name]
    t = W.random_tree(int(name[6:]), n_nodes=14, lo=1, hi=60, n_roots=2, p_zero=0.15)
    return t.parent, t.seg_len


def run_case(tree, ch, m, groups, dtype, gated=True, skip=True, bias=True, fused=False, softplus=True, gateway=False, seed=0):
    parent, seg = tree_of(tree)
    meta = T.tree_build_meta(parent, seg)
    n, pred = meta.n_tokens, meta.tok_pred.tolist()
    k = make(n, ch, m, groups, dtype, seed + n + ch, gated, skip, bias, fused)
    if not softplus:                  # (positive steps, no bias: one of -4 makes a state of rate -16 grow by e^64, past fp32, in a token)
        k["dt"] = k["dt"].abs() * 0.05
    g = torch.Generator().manual_seed(seed)
    dy = torch.randn((n, ch), generator=g).to(dtype)
    caps, cap_tok, init, d_end = [], [], None, None
    if gateway:
        nodes = [int(i) for i in range(len(seg)) if seg[i] > 0]
        caps = [nodes[-1]] + ([nodes[0]] if len(nodes) > 1 else [])
        order = meta.dfs_order.tolist()
        cap_tok = [int(meta.node_end[order.index(i)]) - 1 for i in caps]
        init = torch.randn((ch, m), generator=g)
        d_end = torch.randn((len(caps), ch, m), generator=g)
    plan = T.tree_gdn_plan(parent, seg, caps)
    d = cuda(k)
    A, x, dt, B, C = (d[i] for i in ("A", "x", "dt", "B", "C"))
    layer = {"D": d["D"], "z": d["z"], "dt_bias": d["dt_bias"], "softplus": softplus, "initial_state": None if init is None else init.cuda()}
    buf = torch.full((n, ch + 5), 7.0, dtype=dtype, device="cuda")
    got = T.tree_scan_fwd(x, dt, A, B, C, plan, return_states=gateway, out=buf[:, 2:2 + ch], **layer)
    y, states = got if gateway else (got, None)
    grads = T.tree_scan_bwd(x, dt, A, B, C, dy.cuda(), plan, d_state_out=None if d_end is None else d_end.cuda(),
                            want_d_initial_state=gateway, **layer)
    again = T.tree_scan_bwd(x, dt, A, B, C, dy.cuda(), plan, d_state_out=None if d_end is None else d_end.cuda(),
                            want_d_initial_state=gateway, **layer)
    torch.cuda.synchronize()
    assert (buf[:, :2] == 7).all() and (buf[:, 2 + ch:] == 7).all()
    for a, b in zip(grads, again):
        assert a is None or torch.equal(a, b)

    ins = f64(k)
    if init is not None:
        ins["initial_state"] = init.double()
    for t in ins.values():
        if t is not None:
            t.requires_grad_(True)
    yy, h = R.forward(pred, **ins, use_softplus=softplus)
    total = (yy * dy.double()).sum()
    if gateway:
        total = total + (h[cap_tok] * d_end.double()).sum()
    total.backward()
    size = R.magnitudes(pred, dy.double(), d_end, cap_tok, **{a: (None if b is None else b.detach()) for a, b in ins.items()},
                        use_softplus=softplus)
    depth, half = max(R.depth_of(pred)), HALF[dtype]
    R.assert_close(y, yy, size["y"], depth, m, half, "y")
    if gateway:
        R.assert_close(states, h[cap_tok], size["h"][cap_tok], depth, 1, 0, "states")
    for name, adds in (("dx", m), ("ddt", m), ("dA", n), ("dB", ch), ("dC", ch), ("dD", n), ("dz", m), ("ddt_bias", n + m),
                       ("d_initial_state", n)):
        t, src = getattr(grads, name), ins.get(name[2:] if name != "dA" else "A", None) if name.startswith("d_") else ins.get(name[1:])
        assert (t is None) == (src is None), name
        if t is not None:
            R.assert_close(t, src.grad, size[name], 2 * depth, adds, half if t.dtype == dtype else 0, name)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tree", list(TREES) + ["random3", "random8"])
def test_trees(tree, dtype):
    print(f"[case] scan tree={tree} {dtype}", flush=True)
    run_case(tree, 70, 16, 1, dtype, gateway=True)


@pytest.mark.parametrize("ch,m,groups", [(1, 4, 1), (3, 16, 1), (64, 8, 1), (65, 4, 1), (128, 8, 2), (256, 16, 4), (260, 16, 1), (192, 4, 3)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_channels_states_and_groups(ch, m, groups, dtype):
    print(f"[case] scan channels={ch} states={m} groups={groups} {dtype}", flush=True)
    run_case("random5", ch, m, groups, dtype)


@pytest.mark.parametrize("option", ["plain", "no_gate", "no_skip", "no_bias", "steps_as_given", "fused", "fused_fp32"])
def test_options(option):
    print(f"[case] scan {option}", flush=True)
    dtype = torch.float32 if option == "fused_fp32" else torch.bfloat16
    run_case("random6", 128, 16, 2, dtype, gated=option not in ("plain", "no_gate"), skip=option not in ("plain", "no_skip"),
             bias=option not in ("plain", "no_bias", "steps_as_given"), softplus=option != "steps_as_given", fused=option.startswith("fused"),
             gateway=option == "fused")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_long_chunks_give_the_same(dtype):
    """One chunk for a whole sequence against chunks of 64."""
    n, ch, m = 531, 96, 16
    d = cuda(make(n, ch, m, 1, dtype, 4))
    plan = T.tree_gdn_plan([-1], [n], [0])
    i32 = lambda *v: np.array(v, np.int32)                                      # noqa: E731
    one = T.GdnPlan(1, 0, i32(0), i32(n), i32(-1), i32(-1), i32(0), n_capture=1)
    args, layer = [d[i] for i in ("x", "dt", "A", "B", "C")], {i: d[i] for i in ("D", "z", "dt_bias")}
    (a, sa), (b, sb) = (T.tree_scan_fwd(*args, p, return_states=True, **layer) for p in (plan, one))
    torch.cuda.synchronize()
    assert (a.float() - b.float()).norm() <= (2.0 ** -8 if dtype == torch.bfloat16 else n * 2.0 ** -23) * b.float().norm()
    assert (sa - sb).norm() <= n * 2.0 ** -23 * sb.norm()


def test_many_channels_join_chunks():
    """Enough channels that the forward's program is joined: the same as the program itself through the backward's recomputation
    is covered elsewhere; here the joined forward meets the float64 recurrence on some channels."""
    parent, seg = [-1, 0, 0], [900, 700, 300]
    n, ch, m, dtype = 1900, 64 * 1024, 4, torch.bfloat16
    plan = T.tree_gdn_plan(parent, seg)
    k = make(n, ch, m, 1, dtype, 9, gated=False)
    d = cuda(k)
    y = T.tree_scan_fwd(d["x"], d["dt"], d["A"], d["B"], d["C"], plan, D=d["D"], dt_bias=d["dt_bias"])
    torch.cuda.synchronize()
    assert max(plan._scan_program(ch, False)[1]) > 64
    pick = [0, 1, 4097, ch - 1]
    ins = f64({i: (t if t is None or i in ("B", "C") else (t[pick] if i in ("A", "D", "dt_bias") else t[:, pick])) for i, t in k.items()})
    pred = T.tree_build_meta(parent, seg).tok_pred.tolist()
    yy, _ = R.forward(pred, **ins)
    size = R.magnitudes(pred, None, None, [], **ins)
    R.assert_close(y[:, pick], yy, size["y"], max(R.depth_of(pred)), m, HALF[dtype], "y")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_partitions_through_the_gateway(dtype):
    """A parent's partition and its two children, states down and gradients up, against the whole tree in one call."""
    parent, seg = [-1, 0, 0, 1], [80, 70, 33, 64]
    n, ch, m = sum(seg), 128, 16
    d = cuda(make(n, ch, m, 1, dtype, 12))
    order = T.tree_build_meta(parent, seg).dfs_order.tolist()
    assert order == [0, 1, 3, 2]
    dy = torch.randn((n, ch), generator=torch.Generator().manual_seed(2)).to(dtype).cuda()
    names = ("x", "dt", "A", "B", "C")
    layer = {i: d[i] for i in ("D", "z", "dt_bias")}
    y = T.tree_scan_fwd(*(d[i] for i in names), T.tree_gdn_plan(parent, seg), **layer)
    g = T.tree_scan_bwd(*(d[i] for i in names), dy, T.tree_gdn_plan(parent, seg), **layer)

    def cut(a, b):
        part = {i: (t if i in ("A", "D", "dt_bias") else t[a:b]) for i, t in d.items()}
        return [part[i] for i in names], {i: part[i] for i in ("D", "z", "dt_bias")}
    a1, l1 = cut(0, 80)
    a2, l2 = cut(80, 214)
    a3, l3 = cut(214, n)
    p1, p2, p3 = T.tree_gdn_plan([-1], [80], [0]), T.tree_gdn_plan([-1, 0], [70, 64]), T.tree_gdn_plan([-1], [33])
    y1, s = T.tree_scan_fwd(*a1, p1, return_states=True, **l1)
    y2, y3 = T.tree_scan_fwd(*a2, p2, initial_state=s[0], **l2), T.tree_scan_fwd(*a3, p3, initial_state=s[0], **l3)
    g2 = T.tree_scan_bwd(*a2, dy[80:214], p2, initial_state=s[0], want_d_initial_state=True, **l2)
    g3 = T.tree_scan_bwd(*a3, dy[214:], p3, initial_state=s[0], want_d_initial_state=True, **l3)
    g1 = T.tree_scan_bwd(*a1, dy[:80], p1, d_state_out=(g2.d_initial_state + g3.d_initial_state)[None].contiguous(), **l1)
    torch.cuda.synchronize()
    half = 2 * HALF[dtype] + 500 * 2.0 ** -24
    close = lambda a, b, tol: (a.double() - b.double()).norm() <= tol * b.double().norm()      # noqa: E731
    assert close(torch.cat([y1, y2, y3]), y, half)
    for i, name in enumerate(("dx", "ddt", "dB", "dC", "dz")):
        assert close(torch.cat([getattr(q, name) for q in (g1, g2, g3)]), getattr(g, name), half), name
    for name in ("dA", "dD", "ddt_bias"):
        assert close(sum(getattr(q, name) for q in (g1, g2, g3)), getattr(g, name), 2000 * 2.0 ** -24), name


def test_no_tokens():
    d = cuda(make(0, 64, 8, 1, torch.bfloat16, 1))
    plan = T.tree_gdn_plan([-1], [0])
    args = [d[i] for i in ("x", "dt", "A", "B", "C")]
    assert T.tree_scan_fwd(*args, plan, D=d["D"], z=d["z"]).shape == (0, 64)
    g = T.tree_scan_bwd(*args, d["x"], plan, D=d["D"], z=d["z"], dt_bias=d["dt_bias"], want_d_initial_state=True)
    torch.cuda.synchronize()
    assert g.dx.shape == (0, 64) and (g.dA == 0).all() and (g.dD == 0).all() and (g.ddt_bias == 0).all() and (g.d_initial_state == 0).all()


def test_extreme_steps():
    """Steps that leave nothing of a state, or everything; rates of zero."""
    n, ch, m = 130, 64, 4
    k = make(n, ch, m, 1, torch.float32, 3, gated=False, bias=False)
    k["dt"][::3] = 80.0
    k["dt"][1::3] = -60.0
    k["A"][:, 0] = 0.0
    d = cuda(k)
    args = [d[i] for i in ("x", "dt", "A", "B", "C")]
    y = T.tree_scan_fwd(*args, T.tree_gdn_plan([-1], [n]), D=d["D"])
    g = T.tree_scan_bwd(*args, d["x"], T.tree_gdn_plan([-1], [n]), D=d["D"])
    torch.cuda.synchronize()
    ins = {i: None if t is None else t.requires_grad_(True) for i, t in f64(k).items()}
    pred = list(range(-1, n - 1))
    yy, _ = R.forward(pred, **ins)
    (yy * k["x"].double()).sum().backward()
    size = R.magnitudes(pred, k["x"].double(), None, [], **{i: None if t is None else t.detach() for i, t in ins.items()})
    R.assert_close(y, yy, size["y"], n, m, 2.0 ** -24, "y")
    for name, adds in (("dx", m), ("ddt", m), ("dA", n), ("dB", ch), ("dC", ch), ("dD", n)):
        R.assert_close(getattr(g, name), ins[name[1:]].grad, size[name], 2 * n, adds, 2.0 ** -24, name)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("ch", [6, 70])
def test_more_branch_points_than_fit_on_chip(ch, dtype):
    """A binary tree of 511 nodes has 255 branch points, whose states are kept in the workspace; 6 x 16 and 70 x 16 states leave lanes
    and whole waves of a workgroup without an entry."""
    parent = [-1] + [(i - 1) // 2 for i in range(1, 511)]
    TREES["binary"] = (parent, [1 + i % 2 for i in range(511)])
    run_case("binary", ch, 16, 1, dtype, gateway=True)
    assert T.tree_gdn_plan(*TREES["binary"]).n_slots == 255


def test_given_workspaces_are_not_overrun():
    parent, seg = TREES["worked"]
    n, ch = sum(seg), 200
    d = cuda(make(n, ch, 8, 1, torch.bfloat16, 6))
    args, layer = [d[i] for i in ("x", "dt", "A", "B", "C")], {i: d[i] for i in ("D", "z", "dt_bias")}
    plan = T.tree_gdn_plan(parent, seg)
    for back in (False, True):
        need = T.tree_scan_workspace(d["x"], d["A"], d["B"], plan, backward=back)
        ws = torch.full((need + 4096,), 77, dtype=torch.uint8, device="cuda")
        call = (lambda w: T.tree_scan_bwd(*args, d["x"], plan, workspace=w, **layer)) if back else (lambda w: T.tree_scan_fwd(*args, plan, workspace=w, **layer))
        a, b = call(ws), call(None)
        for p, q in zip(a, b) if back else [(a, b)]:
            assert p is q or torch.equal(p, q)
        assert (ws[need:] == 77).all()
        with pytest.raises(T.TreeTrainError):
            call(ws[:need - 1])
    torch.cuda.synchronize()


def test_order_of_the_pieces():
    """Pieces are independent: started in another order they give the same bits."""
    tree = W.random_tree(21, n_nodes=14, lo=30, hi=400)
    plan = T.tree_gdn_plan(tree.parent, tree.seg_len)
    k = cuda(make(int(tree.seg_len.sum()), 320, 16, 1, torch.bfloat16, 3))
    run = lambda: T.tree_scan_fwd(k["x"], k["dt"], k["A"], k["B"], k["C"], plan, D=k["D"], z=k["z"], dt_bias=k["dt_bias"])    # noqa: E731
    want = run()
    held = next(v for key, v in plan.scan_programs.items() if len(key) == 3)
    for order in (None, torch.arange(held[1].n_chunks - 1, -1, -1, dtype=torch.int32, device="cuda")):
        held[1].chunk_order = None if order is None else order.data_ptr()
        assert torch.equal(run(), want)
