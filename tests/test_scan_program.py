"""tt_tree_scan_program (host): the program cut anew walks the same tree."""
import ctypes

import numpy as np
import pytest

import paper_2511_00413_amd as T
import workloads as W
from paper_2511_00413_amd import binding as B


def ends(tok0, length, src, dst, cap, n_slots):
    """Token before every token, last token of every saved state and capture, by walking a chunk program."""
    slot, caps, pred, last = [None] * n_slots, {}, {}, None
    for a, n, s, d, c in zip(tok0, length, src, dst, cap):
        before = last if s == -2 else (-1 if s == -1 else slot[s])
        for t in range(a, a + n):
            pred[t], before = before, t
        last = a + n - 1
        if d >= 0:
            slot[d] = last
        if c >= 0:
            caps[c] = last
    return pred, slot, caps


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("channels", [8, 256, 4096, 65536])
@pytest.mark.parametrize("seed,lo,hi", [(1, 0, 40), (2, 50, 900), (3, 1, 3000)])
def test_program(seed, lo, hi, channels, backward):
    tree = W.random_tree(seed, n_nodes=25, lo=lo, hi=hi, n_roots=2)
    cuts = [i for i in range(25) if tree.seg_len[i] > 0][3::7]
    plan = T.tree_gdn_plan(tree.parent, tree.seg_len, cuts)
    out = plan._scan_program(channels, backward).tolist()
    arrays = [plan.chunk_tok0, plan.chunk_len, plan.chunk_src, plan.chunk_dst, plan.chunk_cap]
    assert ends(*out, plan.n_slots) == ends(*(a.tolist() for a in arrays), plan.n_slots)
    assert min(out[1]) >= 1
    share = sum(out[1]) * -(-channels // 64) // 1024
    if backward:
        most = tail = 64 if share >= 400 else 32 if share >= 80 else 16
    else:
        tail = max(t for t in (16, 32, 64, 128, 256, 512, 1024) if t == 16 or 5 * t <= 2 * share)
        most = min(tail, max(tail // 4, 64))
    for i, n in enumerate(out[1]):
        goes_on = out[3][i] >= 0 or out[4][i] >= 0 or (i + 1 < len(out[1]) and out[2][i + 1] == -2)
        assert n <= (most if goes_on else tail), i


def test_empty_and_refusals():
    n, a = ctypes.c_int32(0), [np.array(v, np.int32) for v in ([0, 64], [64, 64], [-1, -2], [-1, -1], [-1, -1])]
    out = [np.zeros(8, np.int32) for _ in range(5)]
    f = B._lib().tt_tree_scan_program
    p = lambda v: [B._hp(x) for x in v]                                       # noqa: E731
    assert f(2, *p(a), 64, 0, ctypes.byref(n), *p(out)) == 0 and n.value == 8 and out[1].tolist() == [16] * 8
    assert f(2, *p(a), 64, 0, ctypes.byref(n), *[None] * 5) == 0 and n.value == 8
    assert f(2, *p(a), 64, 0, ctypes.byref(n), *p(out[:4]), None) == 0
    assert f(2, *p(a), 0, 0, ctypes.byref(n), *p(out)) == -2
    assert f(-1, *p(a), 64, 0, ctypes.byref(n), *p(out)) == -2
    assert f(2, *p(a[:3]), None, None, 64, 0, ctypes.byref(n), *p(out)) == -1
    assert f(2, *p(a), 64, 0, ctypes.byref(n), None, *p(out[1:])) == -1
    assert f(2, *p(a), 64, 0, None, *p(out)) == -1
    bad = [x.copy() for x in a]
    bad[0][1] = 63
    assert f(2, *p(bad), 64, 0, ctypes.byref(n), *p(out)) == -3
    bad = [x.copy() for x in a]
    bad[1][0] = 0
    assert f(2, *p(bad), 64, 0, ctypes.byref(n), *p(out)) == -3
    assert f(0, None, None, None, None, None, 64, 1, ctypes.byref(n), None, None, None, None, None) == 0 and n.value == 0
