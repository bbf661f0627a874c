"""The operators of a policy-gradient step together, as a model uses them on a rollout tree: convolution, selective scan and gate of an
SSM layer, multi-axis rotation and tree attention, log-prob and entropy of the sampled tokens with their gradient back to every
parameter; against the same step in float64 with automatic differentiation.  And the new calls in a HIP graph and on other streams."""
import numpy as np
import pytest
import torch

import paper_2511_00413_amd as T
import scan_ref as R
import workloads as W

pytestmark = pytest.mark.gpu

PARENT, SEG = [-1, 0, 0, 1, 1], [37, 30, 21, 16, 70]
GRID = [[0, 0, 0], [1, 5, 6], [0, 0, 0], [2, 2, 4], [0, 0, 0]]
CH, M, HQ, HKV, D, V, TAPS = 128, 16, 4, 2, 64, 517, 4
SECTIONS = (8, 12, 12)


def function(fwd, bwd):
    """An autograd function of a pair of library calls: fwd(*tensors) -> (outputs, saved), bwd(saved, *grads) -> grads."""
    class F(torch.autograd.Function):
        @staticmethod
        def forward(ctx, *ts):
            out, ctx.kept = fwd(*ts)
            return out

        @staticmethod
        def backward(ctx, *gs):
            return bwd(ctx.kept, *(g.contiguous() for g in gs))
    return F.apply


def parameters(n):
    g = torch.Generator().manual_seed(5)
    r = lambda *s, std=1.0: torch.randn(s, generator=g) * std                   # noqa: E731
    E = HQ * D
    return {"x": r(n, CH), "cw": r(CH, TAPS, std=0.5), "cb": r(CH, std=0.1), "Wdt": r(CH, CH, std=0.05), "Wbc": r(CH, 2 * M, std=0.1), "z": r(n, CH),
            "A": -(torch.arange(1, M + 1).float() * torch.exp(0.1 * r(CH, M))), "Dk": 1 + 0.1 * r(CH), "bias": r(CH, std=0.5) - 3,
            "Wq": r(CH, E, std=0.1), "Wk": r(CH, HKV * D, std=0.1), "Wv": r(CH, HKV * D, std=0.1), "Wo": r(E, V, std=0.1)}


def library_step(p, meta, target, d_logp, d_ent):
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()          # noqa: E731
    pred, axes = dev(meta.tok_pred), dev(T.tree_axis_positions(PARENT, SEG, GRID))
    plan, cplan = T.tree_gdn_plan(PARENT, SEG), T.tree_conv_plan(meta.tok_pred, TAPS)
    mask = [dev(a) for a in (meta.kend, meta.ktile_kend_min, meta.ktile_kend_max)]
    conv = function(lambda x, w, b: (T.tree_conv_fwd(x, w, b, pred), (x, w, b)), lambda s, dy: T.tree_conv_bwd(*s, pred, dy, cplan))
    scan = function(lambda x, dt, A, B, C, Dk, z, bias: (T.tree_scan_fwd(x, dt, A, B, C, plan, D=Dk, z=z, dt_bias=bias), (x, dt, A, B, C, Dk, z, bias)),
                    lambda s, dy: tuple(T.tree_scan_bwd(*s[:5], dy, plan, D=s[5], z=s[6], dt_bias=s[7]))[:8])
    rope = function(lambda x: (T.tree_rope_axes(x, axes, SECTIONS, interleaved=True), None),
                    lambda _, dy: T.tree_rope_axes(dy, axes, SECTIONS, interleaved=True, inverse=True))

    def attn_fwd(q, k, v):
        o, lse = T.tree_attn_fwd(q, k, v, *mask)
        return o, (q, k, v, o, lse)
    attn = function(attn_fwd, lambda s, do: T.tree_attn_bwd(*s[:3], *mask, s[3], do, s[4]))

    def loss_fwd(z):
        logp, ent, lse, _, _ = T.tree_logprob_entropy(z, target)
        return (logp, ent), (z, lse, ent)
    loss = function(loss_fwd, lambda s, g1, g2: T.tree_logprob_entropy_bwd(s[0], target, s[1], s[2], g1, g2))

    u = conv(p["x"], p["cw"], p["cb"])
    bc = (u @ p["Wbc"]).unflatten(1, (2, 1, M))
    y = scan(u, u @ p["Wdt"], p["A"], bc[:, 0].contiguous(), bc[:, 1].contiguous(), p["Dk"], p["z"], p["bias"])
    q, k = rope((y @ p["Wq"]).unflatten(1, (HQ, D))), rope((y @ p["Wk"]).unflatten(1, (HKV, D)))
    o = attn(q, k, (y @ p["Wv"]).unflatten(1, (HKV, D)))
    logp, ent = loss(o.flatten(1) @ p["Wo"])
    return (logp * d_logp).sum() + (ent * d_ent).sum(), logp, ent


def plain_step(p, meta, target, d_logp, d_ent):
    n, pred = meta.n_tokens, meta.tok_pred.tolist()
    chain = [list(range(n))]
    for _ in range(TAPS - 1):
        chain.append([pred[t] if t >= 0 else -1 for t in chain[-1]])
    pre = p["cb"].expand(n, CH)
    for m in range(TAPS):
        idx = torch.tensor(chain[m])
        pre = pre + torch.where(idx[:, None] >= 0, p["x"][idx.clamp(min=0)], torch.zeros(1, dtype=torch.float64)) * p["cw"][:, TAPS - 1 - m]
    u = pre * torch.sigmoid(pre)
    bc = (u @ p["Wbc"]).unflatten(1, (2, 1, M))
    y, _ = R.forward(pred, u, u @ p["Wdt"], p["A"], bc[:, 0], bc[:, 1], p["Dk"], p["z"], p["bias"])
    pos = torch.from_numpy(T.tree_axis_positions(PARENT, SEG, GRID)).double()
    half = D // 2
    axis = [i % 3 if i < 3 * SECTIONS[i % 3] else 0 for i in range(half)]
    ang = (pos[axis].T * 1.0e6 ** (-torch.arange(half, dtype=torch.float64) / half))[:, None]

    def rope(x):
        lo, hi = x[..., :half], x[..., half:]
        return torch.cat([lo * ang.cos() - hi * ang.sin(), hi * ang.cos() + lo * ang.sin()], -1)
    q, k = rope((y @ p["Wq"]).unflatten(1, (HQ, D))), rope((y @ p["Wk"]).unflatten(1, (HKV, D)))
    v = (y @ p["Wv"]).unflatten(1, (HKV, D))
    i = torch.arange(n)
    seen = (i[None, :] <= i[:, None]) & (i[:, None] < torch.from_numpy(meta.kend).long()[None, :])
    o = []
    for h in range(HQ):
        s = (q[:, h] @ k[:, h * HKV // HQ].T) * D ** -0.5
        o.append(torch.softmax(s.masked_fill(~seen, -float("inf")), -1) @ v[:, h * HKV // HQ])
    lp = torch.log_softmax(torch.cat(o, 1) @ p["Wo"], -1)
    ok = (target >= 0) & (target < V)
    logp = torch.where(ok, lp.gather(1, target.clamp(0, V - 1).long()[:, None])[:, 0], torch.zeros(1, dtype=torch.float64))
    ent = torch.where(ok, -(lp.exp() * lp).sum(1), torch.zeros(1, dtype=torch.float64))
    return (logp * d_logp).sum() + (ent * d_ent).sum(), logp, ent


def test_policy_gradient_step():
    """fp32 throughout.  The attention's fp32 kernels are bounded by 1e-5 (relative, L2), the other calls by less; a gradient passes
    some ten of them twice, so 2e-4."""
    meta = T.tree_build_meta(PARENT, SEG)
    n = meta.n_tokens
    g = torch.Generator().manual_seed(1)
    target = torch.randint(0, V, (n,), generator=g, dtype=torch.int32)
    target[::9] = -1                                                    # tokens that are not trained
    d_logp, d_ent = torch.randn(n, generator=g) / n, 0.01 * torch.rand(n, generator=g)
    p32 = {k: v.cuda().requires_grad_(True) for k, v in parameters(n).items()}
    p64 = {k: v.double().requires_grad_(True) for k, v in parameters(n).items()}
    got = library_step(p32, meta, target.cuda(), d_logp.cuda(), d_ent.cuda())
    got[0].backward()
    torch.cuda.synchronize()
    want = plain_step(p64, meta, target, d_logp.double(), d_ent.double())
    want[0].backward()
    close = lambda a, b: float((a.detach().double().cpu() - b.detach()).norm() / b.detach().norm())      # noqa: E731
    for i, name in ((1, "logp"), (2, "entropy")):
        assert close(got[i], want[i]) <= 2e-4, name
    for name in p64:
        assert close(p32[name].grad, p64[name].grad) <= 2e-4, (name, close(p32[name].grad, p64[name].grad))


def all_calls(dtype):
    """Every new call on one set of inputs; returns (inputs, step)."""
    g = torch.Generator().manual_seed(3)
    meta = T.tree_build_meta(PARENT, SEG)
    n = meta.n_tokens
    r = lambda *s, std=1.0, t=dtype: (torch.randn(s, generator=g) * std).to(t).cuda()      # noqa: E731
    x, dt, z, dy = (r(n, CH) for _ in range(4))
    Bv, Cv, q = r(n, 1, M), r(n, 1, M), r(n, HQ, D)
    A, Dk, bias = -torch.rand(CH, M, generator=g).cuda() - 0.5, r(CH, t=torch.float32), r(CH, t=torch.float32) - 4
    logits, target = r(n, 4111, std=2.0), torch.randint(0, 4111, (n,), generator=g, dtype=torch.int32).cuda()
    few, few_t = r(2, 60000, std=2.0), torch.tensor([5, 59999], dtype=torch.int32).cuda()
    d1, d2 = r(n, t=torch.float32), r(n, t=torch.float32)
    axes = torch.from_numpy(T.tree_axis_positions(PARENT, SEG, GRID)).cuda()
    plan = T.tree_gdn_plan(PARENT, SEG, [2, 4])
    init, d_end = r(CH, M, t=torch.float32), r(2, CH, M, t=torch.float32)
    w, cs, idx = r(CH, TAPS, t=torch.float32), r(2, TAPS - 1, CH), torch.tensor([1, 0, 1, -1], dtype=torch.int32).cuda()

    def step(stream=None):
        s = {"stream": stream}
        layer = {"D": Dk, "z": z, "dt_bias": bias, **s}
        y, ends = T.tree_scan_fwd(x, dt, A, Bv, Cv, plan, initial_state=init, return_states=True, **layer)
        grads = T.tree_scan_bwd(x, dt, A, Bv, Cv, dy, plan, initial_state=init, d_state_out=d_end, want_d_initial_state=True, **layer)
        layer["z"] = z[:4]
        one = T.tree_scan_step(x[:4], dt[:4], A, Bv[:4], Cv[:4], ends, index=idx, **layer)
        conv = T.tree_conv_step(x[:4], cs, w, bias, index=idx, **s)
        lp = T.tree_logprob_entropy(logits, target, top_k=7, **s)
        lf = T.tree_logprob_entropy(few, few_t, top_k=64, **s)
        dz = T.tree_logprob_entropy_bwd(logits, target, lp[2], lp[1], d1, d2, **s)
        rot = T.tree_rope_axes(q, axes, SECTIONS, **s)
        return (y, ends) + tuple(grads) + one + conv + lp + lf + (dz, rot)
    return (x, dt, logits, few, q), step


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_in_a_graph(dtype):
    """Captured once, replayed with other work in between and with new inputs: every replay is the eager result, bit for bit."""
    inputs, step = all_calls(dtype)
    want = [t.clone() for t in step()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):                                                # two graphs of the same calls, replayed in turn
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            outs = step()
        graphs.append((g, outs))
    for replay in range(2):
        for g, outs in graphs:
            for t in outs:
                t.zero_()
            (inputs[0].float() * 2).sum().item()
            step()                                                    # eager calls with workspaces of their own
            g.replay()
            torch.cuda.synchronize()
            for i, (a, b) in enumerate(zip(outs, want)):
                assert torch.equal(a, b), (replay, i)
    for t in inputs:
        t.mul_(0.5)
    want = [t.clone() for t in step()]
    for g, outs in graphs:
        g.replay()
    torch.cuda.synchronize()
    for g, outs in graphs:
        for i, (a, b) in enumerate(zip(outs, want)):
            assert torch.equal(a, b), i


def test_on_other_streams():
    """The current stream and a stream given by the caller, two at a time, against the default stream."""
    _, step = all_calls(torch.bfloat16)
    want = [t.clone() for t in step()]
    torch.cuda.synchronize()
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    for s in (one, two):
        s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(one):
        a = step()
    with torch.cuda.stream(two):                                      # (outputs and workspaces come from this stream's pool)
        b = step(stream=two)
    torch.cuda.synchronize()
    for i, (x, y, z) in enumerate(zip(a, b, want)):
        assert torch.equal(x, z) and torch.equal(y, z), i


def test_tensors_off_the_gpu_are_refused():
    x = torch.zeros(6, 64, device="cuda")
    A, Bc, plan = torch.zeros(64, 16, device="cuda"), torch.zeros(6, 1, 16), T.tree_gdn_plan([-1], [6])
    with pytest.raises(ValueError):
        T.tree_scan_fwd(x, x, A, Bc, Bc, plan)
    with pytest.raises(ValueError):
        T.tree_logprob_entropy(x, torch.zeros(6, dtype=torch.int32))


def test_a_given_stream_while_another_is_current():
    """Temporaries of a call on a given stream are not handed out again while that stream still works on them."""
    _, step = all_calls(torch.float32)
    want = [t.clone() for t in step()]
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    for _ in range(3):
        other.wait_stream(torch.cuda.current_stream())                # (the memory may have been the current stream's until now)
        got = step(stream=other)
        for size in (1 << 20, 1 << 22, 1 << 24):                      # the current stream takes and fills memory of all sizes
            torch.full((size,), float("nan"), device="cuda")
    torch.cuda.synchronize()
    for i, (a, b) in enumerate(zip(got, want)):
        assert torch.equal(a, b), i


def scan_inputs(n=300, channels=256):
    g = torch.Generator(device="cuda").manual_seed(8)
    f = lambda *s: torch.randn(s, generator=g, device="cuda")          # noqa: E731
    return f(n, channels), f(n, channels), -f(channels, 8).abs(), f(n, 1, 8), f(n, 1, 8)


def test_a_plan_dropped_behind_its_call():
    """The plan's device copy stays until the stream that a call was given is through with it."""
    ins, tree = scan_inputs(), ([-1, 0, 0, 1, 1], [60] * 5)
    want = T.tree_scan_fwd(*ins, T.tree_gdn_plan(*tree))
    busy = torch.randn(4096, 4096, device="cuda")
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        for _ in range(8):
            busy = busy @ busy * 1e-2
    T.tree_scan_fwd(*ins, plan := T.tree_gdn_plan(*tree))               # the copy is made on the current stream
    pieces = plan._scan_program(256, False).size
    got = T.tree_scan_fwd(*ins, plan, stream=other)
    del plan
    for _ in range(20):                                                 # the current stream takes and clears memory of that size
        torch.zeros(pieces, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_a_first_scan_call_is_not_captured():
    ins, tree = scan_inputs(), ([-1, 0], [200, 100])
    plan, want = T.tree_gdn_plan(*tree), T.tree_scan_fwd(*ins, T.tree_gdn_plan(*tree))
    torch.cuda.synchronize()
    with pytest.raises(RuntimeError, match="before the capture"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            T.tree_scan_fwd(*ins, plan)
    assert torch.equal(T.tree_scan_fwd(*ins, plan), want)
