"""What the multi-axis rotation, the log-prob / entropy calls, the selective scan and the single-token calls refuse, before anything is
launched: C ABI by status code (the pointers are never dereferenced), binding by ValueError.  No GPU needed."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2511_00413_amd as T
from paper_2511_00413_amd import binding as B

L = B._lib()
P, NULL = ctypes.c_void_p, ctypes.c_void_p(0)
FAKE = [ctypes.c_void_p(1 << 44 | i << 36) for i in range(1, 24)]        # far apart, 16-byte aligned
BIG = 1 << 34


def test_rope_axes():
    f, m = L.tt_tree_rope_axes, bytes([0] * 16 + [1] * 48)
    ok = dict(n=0, h=4, d=128, dt=0, x=FAKE[0], xs=0, na=3, pos=FAKE[1], map=m, base=1e6, inv=0, y=FAKE[2], ys=0)
    call = lambda **k: f(*{**ok, **k}.values(), None)                       # noqa: E731
    assert call() == 0
    for bad, code in ((dict(dt=7), -4), (dict(n=-1), -2), (dict(h=0), -2), (dict(d=120), -2), (dict(d=2048), -2), (dict(h=1024), -2),
                      (dict(base=1.0), -2), (dict(base=float("inf")), -2), (dict(na=0), -8), (dict(na=5), -8), (dict(map=None), -1),
                      (dict(na=1), -2), (dict(xs=511), -2), (dict(ys=516), -2), (dict(n=4, x=NULL), -1), (dict(n=4, pos=NULL), -1),
                      (dict(n=4, x=P(FAKE[0].value + 8)), -5), (dict(n=4, y=FAKE[0], ys=1024), -2),
                      (dict(n=4, y=P(FAKE[0].value + 1024)), -2), (dict(n=4, xs=2048, ys=2048, y=P(FAKE[0].value + 512)), -2)):
        assert call(**bad) == code and T.last_error(), bad


def test_logprob_entropy():
    f, w = L.tt_tree_logprob_entropy, L.tt_tree_logprob_entropy_workspace
    ok = dict(n=4, v=128, dt=0, z=FAKE[0], zs=0, y=FAKE[1], k=5, logp=FAKE[2], ent=FAKE[3], lse=FAKE[4], ti=FAKE[5], tl=FAKE[6], ws=FAKE[7],
              wb=BIG)
    call = lambda **k: f(*{**ok, **k}.values(), None)                       # noqa: E731
    for bad, code in ((dict(dt=3), -4), (dict(n=-1), -2), (dict(n=1 << 31), -2), (dict(v=0), -2), (dict(k=-1), -2), (dict(k=65), -2),
                      (dict(v=4), -2), (dict(zs=127), -2), (dict(z=NULL), -1), (dict(y=NULL), -1), (dict(logp=NULL), -1), (dict(ent=NULL), -1),
                      (dict(ti=NULL), -1), (dict(tl=NULL), -1), (dict(k=0), -1), (dict(z=P(FAKE[0].value + 1)), -5), (dict(ws=NULL), -6),
                      (dict(wb=8), -6), (dict(ws=P(FAKE[7].value + 8)), -6)):
        assert call(**bad) == code and T.last_error(), bad
    assert w(4, 128, 0, 65) == 0 and w(-1, 128, 0, 0) == 0 and w(4, 128, 9, 0) == 0 and w(4, 128, 0, 64) > 0
    g = L.tt_tree_logprob_entropy_bwd
    ok = dict(n=4, v=128, dt=1, z=FAKE[0], zs=0, y=FAKE[1], lse=FAKE[2], ent=FAKE[3], a=NULL, b=NULL, out=FAKE[4], os=0)
    call = lambda **k: g(*{**ok, **k}.values(), None)                       # noqa: E731
    for bad, code in ((dict(dt=3), -4), (dict(v=-1), -2), (dict(zs=1), -2), (dict(os=1), -2), (dict(lse=NULL), -1), (dict(ent=NULL), -1),
                      (dict(out=NULL), -1), (dict(out=P(FAKE[4].value + 2)), -5), (dict(out=FAKE[0], os=256), -2),
                      (dict(out=P(FAKE[0].value + 64)), -2), (dict(zs=256, os=256, out=P(FAKE[0].value + 256)), -2)):
        assert call(**bad) == code and T.last_error(), bad


def scan_desc(**k):
    v = {**dict(n=100, ch=128, m=16, groups=2, dt=0, sp=1, x=0, d=0, z=0, b=0, c=0, y=0), **k}
    return B._ScanDesc(*v.values())


def chunks(**k):
    v = {**dict(n=2, slots=1, t=FAKE[0], l=FAKE[0], s=FAKE[0], d=FAKE[0], cap=None), **k}
    return B._ScanChunks(*v.values())


DESCS = [(dict(dt=2), -4), (dict(n=-1), -2), (dict(n=2 ** 31 - 1), -2), (dict(ch=0), -2), (dict(ch=1 << 19), -2), (dict(m=12), -8), (dict(m=32), -8),
         (dict(groups=0), -2), (dict(groups=3), -2), (dict(groups=4), -8), (dict(sp=2), -8), (dict(x=127), -2), (dict(d=1), -2),
         (dict(z=1), -2), (dict(y=1), -2), (dict(x=1 << 19), -2), (dict(b=31), -2), (dict(c=34), -5), (dict(c=1 << 19), -2)]


def test_scan_forward():
    f, w = L.tt_tree_scan_fwd, L.tt_tree_scan_fwd_workspace
    ok = dict(x=FAKE[0], dt=FAKE[1], A=FAKE[2], b=FAKE[3], c=FAKE[4], D=FAKE[5], z=FAKE[6], bias=FAKE[7], init=FAKE[8], so=None, y=FAKE[9],
              ws=FAKE[10], wb=BIG)
    call = lambda d=None, k=None, **a: f(ctypes.byref(scan_desc(**(d or {}))), ctypes.byref(chunks(**(k or {}))), *{**ok, **a}.values(), None)  # noqa: E731
    for d, code in DESCS:
        assert call(d) == code and T.last_error(), d
        assert w(ctypes.byref(scan_desc(**d)), 2, 1) == 0 and L.tt_tree_scan_bwd_workspace(ctypes.byref(scan_desc(**d)), 2, 1) == 0, d
    assert w(None, 2, 1) == 0 and w(ctypes.byref(scan_desc()), -1, 0) == 0 and w(ctypes.byref(scan_desc()), 2, 1) > 0
    for k, code in ((dict(n=0), -2), (dict(n=101), -2), (dict(n=-1), -2), (dict(slots=3), -2), (dict(slots=-1), -2), (dict(t=NULL), -1),
                    (dict(d=NULL), -1), (dict(cap=FAKE[0]), -1)):
        assert call(k=k) == code and T.last_error(), k
    assert call(d=dict(n=1 << 30, ch=256, m=4, groups=1), k=dict(n=1 << 24)) == -2          # more than a launch holds
    for a, code in ((dict(A=None), -1), (dict(x=None), -1), (dict(c=None), -1), (dict(y=None), -1), (dict(so=FAKE[11]), -1),
                    (dict(x=P(FAKE[0].value + 1)), -5), (dict(b=P(FAKE[3].value + 4)), -5), (dict(A=P(FAKE[2].value + 4)), -5),
                    (dict(init=P(FAKE[8].value + 4)), -5), (dict(y=P(FAKE[9].value + 1)), -5), (dict(y=FAKE[0]), -2), (dict(y=FAKE[6]), -2),
                    (dict(y=P(FAKE[1].value + 64)), -2), (dict(y=FAKE[3]), -2), (dict(ws=None), -6), (dict(wb=100), -6)):
        assert call(**a) == code and T.last_error(), a
    assert call(k=dict(cap=FAKE[0]), so=FAKE[8]) == -2                                      # state_out on initial_state
    assert f(None, ctypes.byref(chunks()), *ok.values(), None) == -1
    assert f(ctypes.byref(scan_desc()), None, *ok.values(), None) == -1


def test_scan_backward():
    f = L.tt_tree_scan_bwd
    ok = dict(x=FAKE[0], dt=FAKE[1], A=FAKE[2], b=FAKE[3], c=FAKE[4], D=FAKE[5], z=FAKE[6], bias=FAKE[7], init=FAKE[8], dy=FAKE[9], ds=None,
              dx=FAKE[10], ddt=FAKE[11], dA=FAKE[12], db=FAKE[13], dc=FAKE[14], dD=FAKE[15], dz=FAKE[16], dbias=FAKE[17], dinit=FAKE[18],
              ws=FAKE[19], wb=BIG)
    call = lambda d=None, k=None, **a: f(ctypes.byref(scan_desc(**(d or {}))), ctypes.byref(chunks(**(k or {}))), *{**ok, **a}.values(), None)  # noqa: E731
    for d, code in DESCS:
        assert call(d) == code, d
    for a, code in ((dict(dy=None), -1), (dict(dx=None), -1), (dict(dA=None), -1), (dict(dc=None), -1), (dict(dz=None), -1), (dict(z=None), -1),
                    (dict(ds=FAKE[20]), -1), (dict(dx=P(FAKE[10].value + 1)), -5), (dict(dA=P(FAKE[12].value + 4)), -5),
                    (dict(dinit=P(FAKE[18].value + 4)), -5), (dict(dx=FAKE[9]), -2), (dict(dz=FAKE[6]), -2), (dict(dA=FAKE[2]), -2),
                    (dict(ddt=FAKE[10]), -2), (dict(dinit=FAKE[8]), -2), (dict(wb=100), -6), (dict(ws=None), -6)):
        assert call(**a) == code and T.last_error(), a


def test_steps():
    f = L.tt_tree_scan_step
    ok = dict(x=FAKE[0], dt=FAKE[1], A=FAKE[2], b=FAKE[3], c=FAKE[4], D=FAKE[5], z=FAKE[6], bias=FAKE[7], slots=100, s=FAKE[8], i=FAKE[9],
              so=FAKE[10], y=FAKE[11])
    call = lambda d=None, **a: f(ctypes.byref(scan_desc(**(d or {}))), *{**ok, **a}.values(), None)      # noqa: E731
    for d, code in DESCS:
        assert call(d) == code, d
    for a, code in ((dict(slots=-1), -2), (dict(slots=99, i=None), -2), (dict(s=None), -1), (dict(so=None), -1), (dict(y=None), -1), (dict(so=FAKE[8]), -2),
                    (dict(so=P(FAKE[8].value + 16), i=None), -2), (dict(s=P(FAKE[8].value + 8)), -5), (dict(y=FAKE[0]), -2)):
        assert call(**a) == code and T.last_error(), a
    g = L.tt_tree_conv_step
    ok = dict(n=8, c=64, k=4, dt=0, act=1, x=FAKE[0], xs=0, w=FAKE[1], b=FAKE[2], slots=8, s=FAKE[3], i=FAKE[4], so=FAKE[5], y=FAKE[6], ys=0)
    call = lambda **a: g(*{**ok, **a}.values(), None)                       # noqa: E731
    for a, code in ((dict(dt=5), -4), (dict(n=-1), -2), (dict(k=1), -8), (dict(k=5), -8), (dict(act=2), -8), (dict(c=66), -2), (dict(c=0), -2),
                    (dict(xs=60), -5), (dict(ys=66), -5), (dict(w=None), -1), (dict(slots=7, i=None), -2), (dict(x=None), -1), (dict(s=None), -1),
                    (dict(x=P(FAKE[0].value + 4)), -5), (dict(so=FAKE[3]), -2), (dict(y=FAKE[0]), -2), (dict(y=FAKE[3]), -2)):
        assert call(**a) == code and T.last_error(), a


def test_scan_outputs_on_other_tensors():
    f = L.tt_tree_scan_fwd
    ok = dict(x=FAKE[0], dt=FAKE[1], A=FAKE[2], b=FAKE[3], c=FAKE[4], D=FAKE[5], z=FAKE[6], bias=FAKE[7], init=FAKE[8], so=FAKE[11], y=FAKE[9],
              ws=FAKE[10], wb=BIG)
    call = lambda **a: f(ctypes.byref(scan_desc()), ctypes.byref(chunks(cap=FAKE[0])), *{**ok, **a}.values(), None)      # noqa: E731
    for i in (2, 5, 7, 8, 11):
        assert call(y=FAKE[i]) == -2 and T.last_error(), i
    for i in range(10):
        assert call(so=FAKE[i]) == -2 and T.last_error(), i
    f = L.tt_tree_scan_step
    ok = dict(x=FAKE[0], dt=FAKE[1], A=FAKE[2], b=FAKE[3], c=FAKE[4], D=FAKE[5], z=FAKE[6], bias=FAKE[7], slots=100, s=FAKE[8], i=FAKE[9],
              so=FAKE[10], y=FAKE[11])
    call = lambda **a: f(ctypes.byref(scan_desc()), *{**ok, **a}.values(), None)                                          # noqa: E731
    for i in range(11):
        assert call(y=FAKE[i]) == -2 and T.last_error(), i
        if i < 10:
            assert call(so=FAKE[i]) == -2 and T.last_error(), i


def test_binding():
    z, y = torch.zeros(4, 50), torch.zeros(4, dtype=torch.int32)
    f32 = lambda *s: torch.zeros(s)                                           # noqa: E731
    plan = T.tree_gdn_plan([-1], [6])
    x, A, Bc = f32(6, 64), f32(64, 16), f32(6, 1, 16)
    pos = torch.zeros(3, 6, dtype=torch.int32)
    q = f32(6, 2, 32)
    bad = [
        lambda: T.tree_logprob_entropy(z, y),                                                          # on the CPU
        lambda: T.tree_logprob_entropy(z.half(), y), lambda: T.tree_logprob_entropy(z.T, y), lambda: T.tree_logprob_entropy(z, y.long()),
        lambda: T.tree_logprob_entropy(z, y[:3]), lambda: T.tree_logprob_entropy(z, y, top_k=51), lambda: T.tree_logprob_entropy(z, y, top_k=-1),
        lambda: T.tree_logprob_entropy(z[0], y), lambda: T.tree_logprob_entropy(z, y, logp=f32(5)),
        lambda: T.tree_logprob_entropy(z, y, top_index=torch.zeros(4, 2, dtype=torch.int32)),
        lambda: T.tree_logprob_entropy(z.as_strided((4, 50), (10, 1)), y),                             # rows that overlap
        lambda: T.tree_logprob_entropy_bwd(z, y, f32(4), None), lambda: T.tree_logprob_entropy_bwd(z, y, f32(4), f32(3)),
        lambda: T.tree_logprob_entropy_bwd(z, y, f32(4), f32(4), f32(4), out=z.bfloat16()),
        lambda: T.tree_rope_axes(q, pos, (4, 6, 6)), lambda: T.tree_rope_axes(q, pos, (4, 6, 5)), lambda: T.tree_rope_axes(q, pos, (8, 8)),
        lambda: T.tree_rope_axes(q, pos, (20, -2, -2)), lambda: T.tree_rope_axes(q, pos.long(), (4, 6, 6)),
        lambda: T.tree_rope_axes(q, pos[:, :5].contiguous(), (4, 6, 6)), lambda: T.tree_rope_axes(q.transpose(0, 1), pos, (4, 6, 6)),
        lambda: T.tree_rope_axes(q, torch.zeros(5, 6, dtype=torch.int32), (4, 3, 3, 3, 3)), lambda: T.tree_rope_axes(q, pos, (4, 6, 6), out=q[:5]),
        lambda: T.tree_scan_fwd(x, x, A, Bc, Bc, plan), lambda: T.tree_scan_fwd(x, x, A, Bc, Bc, T.tree_gdn_plan([-1], [5])),
        lambda: T.tree_scan_fwd(x, x[:, :32], A, Bc, Bc, plan), lambda: T.tree_scan_fwd(x, x.bfloat16(), A, Bc, Bc, plan),
        lambda: T.tree_scan_fwd(x, x, A[:, :8], Bc, Bc, plan), lambda: T.tree_scan_fwd(x, x, A, Bc[:, 0], Bc, plan),
        lambda: T.tree_scan_fwd(x, x, A, Bc, Bc, plan, D=f32(63)), lambda: T.tree_scan_fwd(x, x, A, Bc, Bc, plan, z=f32(5, 64)),
        lambda: T.tree_scan_fwd(x, x, A, Bc, Bc, plan, initial_state=f32(64, 8)), lambda: T.tree_scan_fwd(x, x, A.double(), Bc, Bc, plan),
        lambda: T.tree_scan_bwd(x, x, A, Bc, Bc, f32(6, 63), plan), lambda: T.tree_scan_bwd(x, x, A, Bc, Bc, x, plan, d_state_out=f32(1, 64, 16)),
        lambda: T.tree_scan_step(x, x, A, Bc, Bc, f32(6, 64, 16)), lambda: T.tree_scan_step(x, x, A, Bc, Bc, f32(6, 64, 8)),
        lambda: T.tree_scan_step(x, x, A, Bc, Bc, f32(6, 64, 16), index=torch.zeros(6)),
        lambda: T.tree_scan_step(x, x, A, Bc, Bc, f32(6, 64, 16), state_out=f32(7, 64, 16)),
        lambda: T.tree_conv_step(x, f32(6, 3, 64), f32(64, 4)), lambda: T.tree_conv_step(x, f32(6, 2, 64), f32(64, 4)),
        lambda: T.tree_conv_step(x, f32(6, 3, 64).bfloat16(), f32(64, 4)), lambda: T.tree_conv_step(x, f32(6, 3, 64), f32(64, 4), f32(63)),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i} was accepted")


def test_every_kernel_has_a_name():
    import os
    import re
    from tt_testutil import ROOT
    text = open(os.path.join(ROOT, "include", "treetrain.h")).read()
    assert int(re.search(r"#define TT_N_KERNELS\s+(\d+)", text).group(1)) == len(B.KERNEL_NAMES)
    assert int(re.search(r"#define TT_LOGPROB_TOP_MAX (\d+)", text).group(1)) == T.LOGPROB_TOP_MAX


def test_a_stream_of_another_device():
    """Tensors (here: on the CPU) that are not on the device of the stream that the call is given."""
    from types import SimpleNamespace
    other = SimpleNamespace(device_index=1, cuda_stream=64)
    z, y, f32 = torch.zeros(4, 50), torch.zeros(4, dtype=torch.int32), lambda *s: torch.zeros(s)
    plan = T.tree_gdn_plan([-1], [6])
    x, A, Bc = f32(6, 64), f32(64, 16), f32(6, 1, 16)
    for call in (lambda: T.tree_logprob_entropy(z, y, stream=other), lambda: T.tree_logprob_entropy_bwd(z, y, f32(4), f32(4), stream=other),
                 lambda: T.tree_rope_axes(f32(6, 2, 32), torch.zeros(3, 6, dtype=torch.int32), (4, 6, 6), stream=other),
                 lambda: T.tree_scan_fwd(x, x, A, Bc, Bc, plan, stream=other), lambda: T.tree_scan_bwd(x, x, A, Bc, Bc, x, plan, stream=other),
                 lambda: T.tree_scan_step(x, x, A, Bc, Bc, f32(6, 64, 16), stream=other),
                 lambda: T.tree_conv_step(x, f32(6, 3, 64), f32(64, 4), stream=other)):
        with pytest.raises(ValueError, match="stream of cuda:1"):
            call()
