"""The selective scan in float64, token by token (torch on the CPU, differentiable), and bounds of what fp32 may be off by.

Bound.  Every term of an output is a product of one input term and at most `depth` decays.  A decay exp(delta A) rounds by 2^-23
(exponential) and 2^-24 (product), its exponent moves by |delta A| times what delta is off by (softplus: 4 units of 2^-24) and the
product's own rounding; where a chunk's decay is one exponential of a sum of steps, that sum's roundings stand in the place of the
single exponents'.  |delta A| of a chain adds up to what the term has decayed by, exp(-s), and s exp(-s) <= 1, so per term the
exponents cost no more than 8 units once and the rest 4 units of 2^-24 per decay.  Adding the terms up costs at most one unit per
addition.  So an output is off by at most (4 depth + additions + 64) 2^-24 times M, the same formula with every factor's absolute
value (the gradient's chains run up and down: twice the depth)."""
import numpy as np
import torch


def softplus(r):
    return torch.clamp(r, min=0) + torch.log1p(torch.exp(-r.abs()))


def forward(pred, x, dt, A, B, C, D=None, z=None, dt_bias=None, use_softplus=True, initial_state=None):
    """All arguments float64 CPU tensors; returns (y, states [n, channels, states])."""
    n, ch = x.shape
    per = ch // B.shape[1]
    raw = dt + (dt_bias if dt_bias is not None else 0.0)
    delta = softplus(raw) if use_softplus else raw
    start = initial_state if initial_state is not None else torch.zeros(ch, A.shape[1], dtype=torch.float64)
    Bc, Cc = B.repeat_interleave(per, 1), C.repeat_interleave(per, 1)
    hs = []
    for t in range(n):
        before = hs[pred[t]] if pred[t] >= 0 else start
        hs.append(torch.exp(delta[t][:, None] * A) * before + (delta[t] * x[t])[:, None] * Bc[t])
    h = torch.stack(hs) if n else torch.zeros(0, ch, A.shape[1], dtype=torch.float64)
    y = (Cc * h).sum(-1)
    if D is not None:
        y = y + D * x
    if z is not None:
        y = y * z * torch.sigmoid(z)
    return y, h


def depth_of(pred):
    d = [0] * len(pred)
    for t, p in enumerate(pred):
        d[t] = d[p] + 1 if p >= 0 else 1
    return d


def magnitudes(pred, dy, d_end, caps, x, dt, A, B, C, D=None, z=None, dt_bias=None, use_softplus=True, initial_state=None):
    """M of every output and gradient (numpy); d_end: upstream gradients of the states after the tokens `caps`."""
    f = lambda t: None if t is None else np.abs(t.detach().numpy())           # noqa: E731
    n, ch = x.shape
    groups, m = B.shape[1], B.shape[2]
    per = ch // groups
    raw = dt + (dt_bias if dt_bias is not None else 0.0)
    delta = (softplus(raw) if use_softplus else raw).detach().numpy()
    decay = np.exp(delta[:, :, None] * A.detach().numpy()) if n else np.zeros((0, ch, m))
    u = np.abs(delta) * f(x)
    Bc, Cc = np.repeat(f(B), per, 1), np.repeat(f(C), per, 1)
    start = f(initial_state) if initial_state is not None else np.zeros((ch, m))
    h, hp = np.zeros((n, ch, m)), np.zeros((n, ch, m))
    for t in range(n):
        hp[t] = h[pred[t]] if pred[t] >= 0 else start
        h[t] = decay[t] * hp[t] + u[t][:, None] * Bc[t]
    y = (Cc * h).sum(-1) + (f(D) * f(x) if D is not None else 0.0)
    gate = f(z) if z is not None else None                                      # |silu(z)| <= |z|, |silu'(z)| <= 1.1
    out = {"y": y * gate if z is not None else y, "h": h}
    if dy is None:
        return out
    g = f(dy) * (gate if z is not None else 1.0)
    G = Cc * g[:, :, None]
    for i, t in enumerate(caps):
        if t >= 0:
            G[t] += f(d_end)[i]
    d0 = np.zeros((ch, m))
    for t in reversed(range(n)):
        if pred[t] >= 0:
            G[pred[t]] += decay[t] * G[t]
        else:
            d0 += decay[t] * G[t]
    q = G * decay * hp
    du = (G * Bc).sum(-1)
    dd = f(x) * du + (f(A) * q).sum(-1)
    fold = lambda v: v.reshape(n, groups, per, m).sum(2)                        # noqa: E731
    out.update(dx=np.abs(delta) * du + (f(D) * g if D is not None else 0.0), ddt=dd, dA=(np.abs(delta)[:, :, None] * q).sum(0),
               dB=fold(G * u[:, :, None]), dC=fold(h * g[:, :, None]), dD=(g * f(x)).sum(0), ddt_bias=dd.sum(0), d_initial_state=d0)
    if z is not None:
        out["dz"] = 1.1 * f(dy) * y
    return out


def assert_close(got, want, size, depth, adds, half, name):
    got, want = got.detach().double().cpu().numpy(), want.detach().numpy()
    bound = (4 * depth + adds + 64) * 2.0 ** -24 * size + half * np.abs(want) + 1e-37
    bad = np.abs(got - want) > bound
    assert got.shape == want.shape and not bad.any(), (name, int(bad.sum()), float(np.max(np.abs(got - want) / bound)))
