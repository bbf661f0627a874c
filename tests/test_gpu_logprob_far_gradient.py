"""Gradient of log-prob and entropy for rows far from zero, where a log-sum-exp in fp32 no longer holds the logarithm of the sum,
against the formula in 64 bits.

Tolerances.  A row that is summed again: ln p = (z - m) - ln s, two roundings of at most D 2^-24 (D = 100: what lies further down has
p < 2^-126) and those of ln s, `acc` = (V / 256 + 16 + 2 D) 2^-24; p another D 2^-24 for the exponential's argument and a unit of it:
e_p = acc + (3 D + 4) 2^-24.  The gradient -p (a + b (ln p + H)) moves by e_p and four roundings of the size of its terms and by p |b| times
the errors of ln p (acc + 2 D 2^-24) and H (acc (1 + 2 (ln V + H)) + 2^-22); then half a step of its type.  A row that is not summed again
adds 3 |lse| 2^-24 to the error of ln p and p (lse: sum, product by ln 2, and its constant; the difference z - lse is one more)."""
import math

import pytest
import torch

import paper_2511_00413_amd as T
from test_gpu_logprob_masks import DT, LEVELS, exact

pytestmark = pytest.mark.gpu
HALF = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}


def run(z, y, dtype, in_place, lse_error=0.0):
    """Forward and gradient of the rows on the GPU, compared with the formula."""
    n, vocab = z.shape
    g = torch.Generator().manual_seed(n)
    a, b = torch.randn(n, generator=g), torch.randn(n, generator=g)
    zc = z.cuda()
    _, ent, lse, _, _ = T.tree_logprob_entropy(zc, y.cuda())
    got = T.tree_logprob_entropy_bwd(zc, y.cuda(), lse, ent, a.cuda(), b.cuda(), out=zc if in_place else None).double().cpu()
    _, H, _, lp = exact(z, y)
    a, b, H = a.double()[:, None], b.double()[:, None], H[:, None]
    p = lp.exp()
    inner = torch.where(p > 0, lp, torch.zeros_like(lp)) + H
    hot = torch.zeros_like(p).scatter_(1, y.long()[:, None], 1.0)
    want = a * (hot - p) - b * p * inner
    D, eps = 100, 2.0 ** -24
    acc = (vocab / 256 + 16 + 2 * D) * eps
    e_ln, e_h = acc + 2 * D * eps + lse_error, acc * (1 + 2 * (math.log(vocab) + H)) + 2.0 ** -22
    err = p * (a.abs() + b.abs() * inner.abs()) * (acc + (3 * D + 8) * eps + lse_error) + p * b.abs() * (e_ln + e_h) + 4 * eps * hot * a.abs()
    assert ((got - want).abs() <= err + HALF[dtype] * want.abs() + 1e-37).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,vocab", [(2, 20011), (600, 2500)])
@pytest.mark.parametrize("sign", [-1.0, 1.0])
def test_rows_on_a_level(sign, n, vocab, dtype):
    """Rows wholly on one level, and four equal entries above the others; in place too."""
    for i, level in enumerate(LEVELS + [3.2e38]):
        print(f"[case] logprob_entropy_bwd rows at {sign * level:g} n={n} vocab={vocab} {dtype}", flush=True)
        z = torch.full((n, vocab), sign * level).to(DT[dtype])
        z[1:] = torch.tensor(sign * level * (1.05 if sign < 0 else 0.5)).to(DT[dtype])
        z[1:, 700:704] = torch.tensor(sign * level).to(DT[dtype])
        run(z, torch.full((n,), 702, dtype=torch.int32), dtype, in_place=i % 2 == 1)


@pytest.mark.parametrize("shift,again", [(-5000.0, True), (1100.0, True), (900.0, False), (30000.0, True)])
@pytest.mark.parametrize("n,offset", [(3, 0), (600, 1)])
def test_a_common_shift(shift, again, n, offset):
    """In fp32, logits on a grid of 2^-8 so that the shifted ones are exact; on both sides of the bound."""
    vocab = 6001
    base = (torch.randn(n, vocab + offset, generator=torch.Generator().manual_seed(4)) * 512).round() / 256
    run((base + shift)[:, offset:], torch.arange(n, dtype=torch.int32), "fp32", False, 0.0 if again else 4 * 920 * 2.0 ** -24)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_far_rows_among_others(dtype):
    """Rows of all kinds in one call: ordinary ones, far ones, an ignored one on a far level, one without a distribution."""
    n, vocab = 40, 9001
    z = (torch.randn(n, vocab, generator=torch.Generator().manual_seed(6)) * 2)
    z[3:6] *= 3e4
    z[7] = -1e12
    z[9] = 4e9
    z = z.to(DT[dtype])
    y = torch.arange(n, dtype=torch.int32) * 11
    rows = [r for r in range(n) if r not in (9, 12)]
    z[12] = -float("inf")
    y[9] = -1
    one = torch.ones(n)
    zc, yc = z.cuda(), y.cuda()
    _, ent, lse, _, _ = T.tree_logprob_entropy(zc, yc)
    got = T.tree_logprob_entropy_bwd(zc, yc, lse, ent, one.cuda(), one.cuda()).cpu()
    assert (got[9] == 0).all() and torch.isnan(got[12]).all()
    run(z[rows], y[rows], dtype, False, 4 * 1024 * 2.0 ** -24)
    alone = T.tree_logprob_entropy_bwd(zc[3:6].contiguous(), yc[3:6], lse[3:6], ent[3:6].contiguous(), one[:3].cuda(), one[:3].cuda()).cpu()
    assert torch.equal(got[3:6], alone)
