"""Outputs that lie on inputs or on other outputs are refused before anything is launched (the pointers are never dereferenced)."""
import ctypes

from test_operator_refusals import BIG, FAKE, L, P, T, chunks, scan_desc

WIDTH = 128 * 16 * 4                                                    # bytes of a state of scan_desc()


def behind(p, n):
    return P(p.value + n)


def test_the_second_captured_state():
    """state_out and d_state_out hold n_capture states; an overlap with any of them counts."""
    f = L.tt_tree_scan_fwd
    ok = dict(x=FAKE[0], dt=FAKE[1], A=FAKE[2], b=FAKE[3], c=FAKE[4], D=FAKE[5], z=FAKE[6], bias=FAKE[7], init=FAKE[8], so=FAKE[11], y=FAKE[9],
              ws=FAKE[10], wb=BIG)

    def forward(n_capture=2, **a):
        k = chunks(cap=FAKE[0], slots=2, n=4)
        k.n_capture = n_capture
        return f(ctypes.byref(scan_desc()), ctypes.byref(k), *{**ok, **a}.values(), None)
    for i in range(1, 10):
        assert forward(so=behind(FAKE[i], -WIDTH)) == -2 and "shares memory" in T.last_error(), i
        assert forward(n_capture=4, so=behind(FAKE[i], -3 * WIDTH)) == -2 and "shares memory" in T.last_error(), i
    assert forward(y=behind(FAKE[11], WIDTH)) == -2 and "shares memory" in T.last_error()
    assert forward(n_capture=-1) == -2 and forward(n_capture=5) == -2 and "captured" in T.last_error()
    g = L.tt_tree_scan_bwd
    okb = dict(x=FAKE[0], dt=FAKE[1], A=FAKE[2], b=FAKE[3], c=FAKE[4], D=FAKE[5], z=FAKE[6], bias=FAKE[7], init=FAKE[8], dy=FAKE[9], ds=FAKE[20],
               dx=FAKE[10], ddt=FAKE[11], dA=FAKE[12], db=FAKE[13], dc=FAKE[14], dD=FAKE[15], dz=FAKE[16], dbias=FAKE[17], dinit=FAKE[18],
               ws=FAKE[19], wb=BIG)

    def backward(**a):
        k = chunks(cap=FAKE[0], slots=2, n=4)
        k.n_capture = 3
        return g(ctypes.byref(scan_desc()), ctypes.byref(k), *{**okb, **a}.values(), None)
    for name in ("dx", "ddt", "dA", "db", "dc", "dD", "dz", "dbias", "dinit"):
        assert backward(**{name: behind(FAKE[20], 2 * WIDTH)}) == -2 and "shares memory" in T.last_error(), name


def test_scan_outputs_on_the_chunk_program():
    f = L.tt_tree_scan_fwd
    ok = dict(x=FAKE[0], dt=FAKE[1], A=FAKE[2], b=FAKE[3], c=FAKE[4], D=FAKE[5], z=FAKE[6], bias=FAKE[7], init=FAKE[8], so=FAKE[11], y=FAKE[9],
              ws=FAKE[10], wb=BIG)
    for i, name in enumerate(("chunk_tok0", "chunk_len", "chunk_src", "chunk_dst", "chunk_cap", "chunk_order")):
        for out in ("y", "so"):
            k = chunks(t=FAKE[12], l=FAKE[13], s=FAKE[14], d=FAKE[15], cap=FAKE[16])
            setattr(k, name, FAKE[17].value)
            assert f(ctypes.byref(scan_desc()), ctypes.byref(k), *{**ok, out: FAKE[17]}.values(), None) == -2, (name, out)
            assert "shares memory" in T.last_error()
    g = L.tt_tree_scan_bwd
    okb = dict(x=FAKE[0], dt=FAKE[1], A=FAKE[2], b=FAKE[3], c=FAKE[4], D=FAKE[5], z=FAKE[6], bias=FAKE[7], init=FAKE[8], dy=FAKE[9], ds=None,
               dx=FAKE[10], ddt=FAKE[11], dA=FAKE[12], db=FAKE[13], dc=FAKE[14], dD=FAKE[15], dz=FAKE[16], dbias=FAKE[17], dinit=FAKE[18],
               ws=FAKE[19], wb=BIG)
    assert g(ctypes.byref(scan_desc()), ctypes.byref(chunks(s=FAKE[12])), *okb.values(), None) == -2 and "shares memory" in T.last_error()


def test_convolution_step():
    f = L.tt_tree_conv_step
    ok = dict(n=8, c=64, k=4, dt=0, act=1, x=FAKE[0], xs=0, w=FAKE[1], b=FAKE[2], slots=8, s=FAKE[3], i=FAKE[4], so=FAKE[5], y=FAKE[6], ys=0)
    call = lambda **a: f(*{**ok, **a}.values(), None)                       # noqa: E731
    for i, size in ((1, 64 * 4 * 4), (2, 64 * 4), (4, 8 * 4)):              # weight, bias, index: on them, on their last bytes
        for at in (FAKE[i], behind(FAKE[i], size - 8), behind(FAKE[i], -8)):
            assert call(y=at) == -2 and "shares memory" in T.last_error(), i
            assert call(so=at) == -2 and "shares memory" in T.last_error(), i


def test_logprob_entropy():
    """Outputs on the logits, the targets, or each other; the gradient on the per-row inputs."""
    f = L.tt_tree_logprob_entropy
    n, v, k = 4, 128, 5
    ok = dict(n=n, v=v, dt=0, z=FAKE[0], zs=0, y=FAKE[1], k=k, logp=FAKE[2], ent=FAKE[3], lse=FAKE[4], ti=FAKE[5], tl=FAKE[6], ws=FAKE[7], wb=BIG)
    call = lambda **a: f(*{**ok, **a}.values(), None)                       # noqa: E731
    outs = {"logp": n * 4, "ent": n * 4, "lse": n * 4, "ti": n * k * 4, "tl": n * k * 4}
    for name, size in outs.items():
        for at in (behind(FAKE[0], n * v * 2 - 4), FAKE[1], behind(FAKE[1], 4 - size), behind(FAKE[0], 4 - size)):
            assert call(**{name: at}) == -2 and "shares memory" in T.last_error(), name
        for other in outs:
            if other != name:
                assert call(**{name: behind(ok[other], 4 - size)}) == -2 and "shares memory" in T.last_error(), (name, other)
    g = L.tt_tree_logprob_entropy_bwd
    ok = dict(n=n, v=v, dt=1, z=FAKE[0], zs=0, y=FAKE[1], lse=FAKE[2], ent=FAKE[3], a=FAKE[5], b=FAKE[6], out=FAKE[4], os=0)
    for name in ("y", "lse", "ent", "a", "b"):
        for at in (FAKE[4], behind(FAKE[4], n * v * 4 - 4), behind(FAKE[4], 4 - n * 4)):
            assert g(*{**ok, name: at}.values(), None) == -2 and "shares memory" in T.last_error(), name


def test_rotation_on_its_positions():
    ok = dict(n=4, h=4, d=128, dt=0, x=FAKE[0], xs=0, na=3, pos=FAKE[1], map=bytes(64), base=1e6, inv=0, y=FAKE[2], ys=0)
    for at in (FAKE[2], behind(FAKE[2], 4 * 512 * 2 - 4), behind(FAKE[2], 4 - 3 * 4 * 4)):
        assert L.tt_tree_rope_axes(*{**ok, "pos": at}.values(), None) == -2 and "shares memory" in T.last_error()
