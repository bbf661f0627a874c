"""Log-prob of given tokens, entropy and most probable alternatives, and the gradient of the first two, against the definition in
64 bits.

Tolerances.  A thread adds V / 256 terms one after the other and the joins add some ten more, each addition rounding by 2^-24 at
most, and a term exp(d) carries |d| 2^-23 from its rounded argument (|d| is at most the range of the logits, D) besides a unit of
the exponential: `acc` = (V / 256 + 16 + 2 D) 2^-24 relative on the sums s and u, all of one sign.  lse and logp move by acc plus
the rounding of the largest of the numbers they are made of; the entropy ln s - u / s by acc (1 + 2 |u / s|), |u / s| <= ln V + H.
Gradient: half a step of its type (bf16 2^-8, fp32 2^-24) on top of the errors of p, lse and entropy."""
import math

import numpy as np
import pytest
import torch

import paper_2511_00413_amd as T

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def want(z, y, k):
    """float64 numpy: logp, entropy, lse, top index, top logp."""
    z = z.double().cpu().numpy()
    y = y.cpu().numpy()
    n, vocab = z.shape
    m = z.max(1, keepdims=True)
    with np.errstate(all="ignore"):
        e = np.exp(z - m)
        s = e.sum(1, keepdims=True)
        lse = (m + np.log(s))[:, 0]
        d = np.where(np.isneginf(z), -1e300, z - m)
        ent = (np.log(s) - (e * np.where(e > 0, d, 0.0)).sum(1, keepdims=True) / s)[:, 0]
        used = (y >= 0) & (y < vocab)
        logp = np.where(used, z[np.arange(n), np.clip(y, 0, vocab - 1)] - lse, 0.0)
    ent = np.where(used, ent, 0.0)
    order = np.argsort(-z, axis=1, kind="stable")[:, :k]
    return logp, ent, lse, order, np.take_along_axis(z, order, 1) - lse[:, None]


def tolerances(z, ent):
    zf = z.double().cpu().numpy()
    vocab = zf.shape[1]
    fin = np.where(np.isfinite(zf), zf, 0.0)
    rng = min(float(np.ptp(fin)), 100.0)
    acc = (vocab / 256 + 16 + 2 * rng) * 2.0 ** -24
    big = np.abs(fin).max(1)
    point = acc + 4 * (big + math.log(vocab) + 1) * 2.0 ** -24
    return point, acc * (1 + 2 * (math.log(vocab) + np.abs(ent))) + 2.0 ** -22


def check(z, y, k, got):
    n = z.shape[0]
    logp, ent, lse, idx, top = want(z, y, k)
    tol, tol_e = tolerances(z, ent)
    f = lambda t: t.double().cpu().numpy()                                    # noqa: E731
    assert (np.abs(f(got[0]) - logp) <= tol + 2.0 ** -23 * np.abs(logp)).all()
    assert (np.abs(f(got[1]) - ent) <= tol_e).all()
    assert (np.abs(f(got[2]) - lse) <= tol).all()
    if k:
        assert np.array_equal(got[3].cpu().numpy(), idx)
        with np.errstate(invalid="ignore"):
            d = np.abs(f(got[4]) - top)
        assert ((d <= tol[:, None] + 2.0 ** -23 * np.abs(top)) | (np.isneginf(f(got[4])) & np.isneginf(top))).all()
    else:
        assert got[3] is None and got[4] is None
    assert got[0].shape == (n,)


def make(n, vocab, dtype, seed, std=2.0, pad=0, offset=0):
    """Logits with a free row stride and a start off the 16-byte grid."""
    g = torch.Generator().manual_seed(seed)
    buf = (torch.randn((n, vocab + pad + offset), generator=g) * std).to(DT[dtype]).cuda()
    z = buf[:, offset:offset + vocab]
    y = torch.randint(0, vocab, (n,), generator=g, dtype=torch.int32).cuda()
    return z, y


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,vocab,k,pad,offset", [
    (1, 1, 1, 0, 0), (3, 2, 2, 0, 0), (2, 7, 7, 3, 1), (5, 63, 5, 0, 0), (4, 64, 64, 1, 3), (3, 65, 64, 0, 0), (7, 500, 64, 5, 2),
    (6, 1001, 20, 0, 0), (2, 2048, 64, 0, 0), (600, 2049, 8, 7, 1), (513, 4099, 1, 0, 0), (1, 32003, 20, 0, 0), (3, 151936, 64, 0, 0),
    (9, 40000, 0, 0, 0), (520, 8200, 0, 1, 1), (700, 30011, 33, 0, 0), (1, 300000, 5, 0, 0), (2, 600001, 17, 3, 1)])
def test_forward(n, vocab, k, pad, offset, dtype):
    print(f"[case] logprob_entropy n={n} vocab={vocab} k={k} pad={pad} offset={offset} {dtype}", flush=True)
    z, y = make(n, vocab, dtype, n * 7 + vocab, pad=pad, offset=offset)
    got = T.tree_logprob_entropy(z, y, top_k=k)
    again = T.tree_logprob_entropy(z, y, top_k=k)
    torch.cuda.synchronize()
    check(z, y, k, got)
    for a, b in zip(got, again):
        assert a is None or torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n", [2, 600])
@pytest.mark.parametrize("kind", ["equal", "two_values", "rising", "falling", "few_left", "mostly_masked", "lowest", "huge", "zeros"])
def test_rows_where_the_alternatives_tie_or_hide(kind, n, dtype):
    vocab, k = 5003, 20
    print(f"[case] logprob_entropy {kind} n={n} {dtype}", flush=True)
    z, y = make(n, vocab, dtype, 5)
    i = torch.arange(vocab, device="cuda").float()
    if kind == "equal":
        z = torch.full_like(z, 1.5)
    elif kind == "two_values":
        z = (z > 3.0).to(z.dtype)
    elif kind == "rising":
        z = (i / 256).expand(n, -1).to(z.dtype).contiguous()
    elif kind == "falling":
        z = (-i / 256).expand(n, -1).to(z.dtype).contiguous()
    elif kind == "few_left":                                # fewer finite entries than alternatives
        z = torch.where(i % 2000 == 7, z, torch.full_like(z, -float("inf")))
    elif kind == "mostly_masked":
        z = torch.where(i > vocab - 40, z, torch.full_like(z, -float("inf")))
    elif kind == "lowest":                                  # masks of the type's lowest value, whole rows of them too
        low = torch.finfo(z.dtype).min
        z = torch.where(i > vocab - 40, z, torch.full_like(z, low))
        z[0] = low
    elif kind == "huge":
        z = z * 1e4
    elif kind == "zeros":                                   # both signs of zero are one value
        z = torch.where(i % 2 == 0, torch.zeros_like(z), -torch.zeros_like(z))
    if kind in ("few_left", "mostly_masked"):
        y = torch.full_like(y, 2007 if kind == "few_left" else vocab - 1)
    z = z.contiguous()
    got = T.tree_logprob_entropy(z, y, top_k=k)
    torch.cuda.synchronize()
    if kind == "lowest":
        first = want(z[:1].double().cpu() * 0, y[:1], k)    # uniform, whatever its level
        assert abs(got[1][0].item() - first[1][0]) < 1e-4 and abs(got[0][0].item() - first[0][0]) < 1e-4
        assert got[3][0].tolist() == list(range(k))
        check(z[1:], y[1:], k, [t[1:] for t in got])
    else:
        check(z, y, k, got)


@pytest.mark.parametrize("n", [3, 520])
def test_rows_without_a_distribution_and_ignored_rows(n):
    z, y = make(n, 4100, "fp32", 11)
    z[0, 17] = float("nan")
    z[1, :] = -float("inf")
    z[2, 5] = float("inf")
    y2 = y.clone()
    got = T.tree_logprob_entropy(z, y, top_k=4)
    assert torch.isnan(got[0][:3]).all() and torch.isnan(got[1][:3]).all()
    assert got[3][1].tolist() == [0, 1, 2, 3] and got[3][2, 0].item() == 5
    clean = torch.nan_to_num(z[0], nan=-float("inf"))
    assert got[3][0].tolist() == torch.sort(clean, descending=True, stable=True).indices[:4].tolist()
    if n > 3:
        check(z[3:], y[3:], 4, [t[3:] for t in got])
    y2[0], y2[1], y2[2] = -1, 4100, -7
    got = T.tree_logprob_entropy(z, y2)
    assert (got[0][:3] == 0).all() and (got[1][:3] == 0).all()
    g = T.tree_logprob_entropy_bwd(z, y2, got[2], got[1], torch.ones(n, device="cuda"), torch.ones(n, device="cuda"))
    assert (g[:3] == 0).all()
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n", [2, 530])
def test_logits_near_the_ends_of_the_type(n, dtype):
    """Rows that overflow when scaled to powers of two: equal largest logits share the probability, everything below them (a step of
    the type is more than 10^29 there) has none."""
    vocab = 2500
    for top, rest in ((3.2e38, 3.0e38), (-3.0e38, -3.2e38), (2.4e38, -2.4e38), (-3.2e38, -float("inf")), (1e30, 0.0), (-1e30, -2e30)):
        z = torch.full((n, vocab), rest).to(DT[dtype]).cuda()
        z[:, 700:704] = top
        y = torch.full((n,), 702, dtype=torch.int32, device="cuda")
        y[1] = 5
        logp, ent, lse, idx, tl = T.tree_logprob_entropy(z, y, top_k=6)
        assert torch.allclose(logp[0], torch.tensor(-math.log(4.0)).cuda(), atol=1e-6) and torch.allclose(ent, torch.tensor(math.log(4.0)).cuda(), atol=1e-6)
        assert (lse - z[:, 700].float()).abs().max() <= 2.0 ** -22 * abs(top)
        assert idx[0].tolist() == [700, 701, 702, 703, 0, 1]
        assert torch.allclose(tl[:, :4], torch.tensor(-math.log(4.0)).cuda(), atol=1e-6) and (tl[:, 4:] < -1e28).all() and logp[1] < -1e28
        g = T.tree_logprob_entropy_bwd(z, y, lse, ent, torch.ones(n, device="cuda"))
        assert torch.isfinite(g).all()
    torch.cuda.synchronize()


@pytest.mark.parametrize("shift", [-5000.0, 3000.0])
def test_a_common_shift_changes_nothing_but_lse(shift):
    """In fp32, logits on a grid of 2^-8 so that the shifted ones are exact."""
    z = (torch.randn(40, 6001, generator=torch.Generator().manual_seed(4)) * 512).round().cuda() / 256
    y = torch.arange(40, dtype=torch.int32, device="cuda")
    a, b = T.tree_logprob_entropy(z, y, top_k=9), T.tree_logprob_entropy(z + shift, y, top_k=9)
    check(z + shift, y, 9, b)
    assert (a[0] - b[0]).abs().max() <= 4e-6 and (a[1] - b[1]).abs().max() <= 4e-6 and torch.equal(a[3], b[3])


def want_grad(z, y, a, b):
    zf = z.double().cpu().numpy()
    logp, ent, lse, _, _ = want(z, y, 0)
    a, b = a[:, None], b[:, None]
    n, vocab = zf.shape
    lp = zf - lse[:, None]
    p = np.exp(lp)
    lp = np.where(p > 0, lp, 0.0)
    hot = np.zeros_like(zf)
    hot[np.arange(n), y.cpu().numpy()] = 1.0
    grad = a * (hot - p) - b * p * (lp + ent[:, None])
    tol, tol_e = tolerances(z, ent)
    size = p * (np.abs(a) + np.abs(b) * (np.abs(lp) + ent[:, None]))
    err = size * (tol[:, None] * 2 + 2.0 ** -20) + p * np.abs(b) * (tol + tol_e)[:, None] + hot * np.abs(a) * 2.0 ** -22
    return grad, err


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,vocab,pad,offset,out_off", [
    (1, 1, 0, 0, 0), (3, 9, 0, 0, 0), (5, 1000, 8, 0, 0), (4, 2051, 5, 3, 3), (3, 4099, 0, 0, 1), (2, 33000, 0, 0, 0), (65, 8193, 7, 0, 0)])
@pytest.mark.parametrize("which", ["both", "logp", "entropy"])
def test_gradient(n, vocab, pad, offset, out_off, dtype, which):
    print(f"[case] logprob_entropy_bwd n={n} vocab={vocab} pad={pad} offset={offset} {dtype} {which}", flush=True)
    z, y = make(n, vocab, dtype, n + vocab, pad=pad, offset=offset)
    g = torch.Generator().manual_seed(3)
    a, b = torch.randn(n, generator=g), torch.randn(n, generator=g)
    if which == "logp":
        b = None
    if which == "entropy":
        a = None
    logp, ent, lse, _, _ = T.tree_logprob_entropy(z, y)
    buf = torch.full((n, vocab + out_off + pad), 9.0, dtype=z.dtype, device="cuda")
    out = buf[:, out_off:out_off + vocab]
    dev = lambda t: None if t is None else t.cuda()                           # noqa: E731
    got = T.tree_logprob_entropy_bwd(z, y, lse, ent, dev(a), dev(b), out=out)
    torch.cuda.synchronize()
    zero = np.zeros(n)
    grad, err = want_grad(z, y, zero if a is None else a.double().numpy(), zero if b is None else b.double().numpy())
    half = 2.0 ** (-8 if dtype == "bf16" else -24)
    assert (np.abs(got.double().cpu().numpy() - grad) <= err + half * np.abs(grad) + 1e-38).all()
    rest = torch.cat([buf[:, :out_off], buf[:, out_off + vocab:]], 1)
    assert (rest == 9.0).all()                                                # what lies beside the rows stays
    z2 = z.clone()
    assert torch.equal(T.tree_logprob_entropy_bwd(z2, y, lse, ent, dev(a), dev(b), out=z2), got) or out_off != 0
    torch.cuda.synchronize()


def test_gradient_against_differences():
    z, y = make(4, 50, "fp32", 21)
    a, b = torch.randn(4).double(), torch.randn(4).double()
    _, ent, lse, _, _ = T.tree_logprob_entropy(z, y)
    got = T.tree_logprob_entropy_bwd(z, y, lse, ent, a.float().cuda(), b.float().cuda()).double().cpu()

    def value(zz):
        logp, e, _, _, _ = want(zz, y, 0)
        return float((a.numpy() * logp + b.numpy() * e).sum())
    zc, h = z.double().cpu(), 1e-5
    for r, v in [(0, 0), (0, int(y[0])), (1, 17), (2, 49), (3, int(y[3]))]:
        up, dn = zc.clone(), zc.clone()
        up[r, v] += h
        dn[r, v] -= h
        assert abs((value(up) - value(dn)) / (2 * h) - got[r, v].item()) < 1e-5


def test_many_short_rows_and_none():
    z, y = make(70001, 11, "bf16", 2)
    got = T.tree_logprob_entropy(z, y, top_k=3)
    check(z, y, 3, got)
    e = T.tree_logprob_entropy(z[:0], y[:0], top_k=3)
    assert e[0].shape == (0,) and e[3].shape == (0, 3)
    assert T.tree_logprob_entropy_bwd(z[:0], y[:0], e[2], e[1]).shape == (0, 11)
    torch.cuda.synchronize()


def test_interleaved_slices_of_one_buffer():
    """Logits and gradient as slices of one buffer whose rows interleave."""
    buf = torch.randn(6, 2 * 512, device="cuda")
    z, out = buf[:, :512], buf[:, 512:]
    y = torch.arange(6, dtype=torch.int32, device="cuda")
    _, ent, lse, _, _ = T.tree_logprob_entropy(z, y)
    one = torch.ones(6, device="cuda")
    want_g = T.tree_logprob_entropy_bwd(z.clone(), y, lse, ent, one, one)
    assert torch.equal(T.tree_logprob_entropy_bwd(z, y, lse, ent, one, one, out=out), want_g)
    with pytest.raises(T.TreeTrainError):
        T.tree_logprob_entropy_bwd(z, y, lse, ent, one, one, out=buf[:, 256:768])


def test_given_outputs_and_workspace():
    z, y = make(3, 70001, "bf16", 8)
    need = T.tree_logprob_entropy_workspace(z, 11)
    ws = torch.full((need + 1024,), 77, dtype=torch.uint8, device="cuda")
    out = [torch.full((3,), 5.0, device="cuda") for _ in range(3)]
    idx, top = torch.zeros(3, 11, dtype=torch.int32, device="cuda"), torch.zeros(3, 11, device="cuda")
    got = T.tree_logprob_entropy(z, y, top_k=11, logp=out[0], entropy=out[1], lse=out[2], top_index=idx, top_logp=top, workspace=ws)
    torch.cuda.synchronize()
    assert got[0] is out[0] and got[3] is idx and (ws[need:] == 77).all()
    check(z, y, 11, got)
    with pytest.raises(T.TreeTrainError):
        T.tree_logprob_entropy(z, y, top_k=11, workspace=ws[:need - 1])
