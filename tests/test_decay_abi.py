"""Host-side checks of linear attention with a decay for each head, rotary positions and layer norm: what is refused before a launch."""
import ctypes

import pytest

OK = 0x1000          # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def L():
    from paper_2405_18428_b200 import build, dig
    build.build()
    return dig.lib()


def floats(*v):
    return (ctypes.c_float * len(v))(*v)


def test_decay_workspace(L):
    from paper_2405_18428_b200 import dig
    ask = lambda B=1, H=6, Hk=6, gh=16, gw=16, dk=64, dv=64, dtype=dig.DIG_BF16, bwd=0: L.dig_decay_workspace_bytes(B, H, Hk, gh, gw, dk, dv, dtype, bwd)
    assert ask() > 0 and ask(bwd=1) > 0 and ask(dtype=dig.DIG_F32) > 0
    # shared heads: their gradients before they are summed
    assert ask(H=6, Hk=2, bwd=1) >= ask(bwd=1) + 256 * 6 * (64 + 64) * 4
    # never more than twice a machine full of segments' states beyond the partial gradients
    assert ask(B=1, H=16, Hk=16, gh=128, gw=128, dk=128, dv=128, bwd=1) < 1 << 30
    for bad in (dict(B=0), dict(H=5, Hk=2), dict(Hk=0), dict(H=257, Hk=1), dict(dk=60), dict(dv=136), dict(dk=0), dict(gh=0), dict(gh=5000, gw=5000),
                dict(dtype=dig.DIG_BF16_F32OUT), dict(dtype=3), dict(B=40000, H=2, Hk=2)):
        assert ask(**bad) == 0


def test_decay_refusals(L):
    from paper_2405_18428_b200 import dig
    lam = floats(-0.1, -0.2)
    st = (ctypes.c_longlong * 6)(128 * 16, 128, 128 * 16, 128, 128 * 16, 128)

    def fwd(q=OK, k=OK, v=OK, strides=None, decay=lam, lengths=None, s_in=None, out=OK, s_out=None, B=1, H=2, Hk=2, gh=4, gw=4, dk=64, dv=64, dir=0, dtype=1, ws=OK,
            n=1 << 30):
        return L.dig_decay_fwd(q, k, v, strides, decay, lengths, s_in, out, s_out, B, H, Hk, gh, gw, dk, dv, dir, dtype, ws, n, None)

    for bad in (dict(q=None), dict(k=OK + 8), dict(v=None), dict(decay=None), dict(out=None), dict(s_in=OK + 4), dict(s_out=OK + 4), dict(s_in=OK, s_out=OK), dict(lengths=OK + 2), dict(H=3), dict(dir=4),
                dict(dir=-1), dict(dtype=2), dict(dk=4), dict(gw=0), dict(strides=(ctypes.c_longlong * 6)(4, 128, 128, 128, 128, 128)),
                dict(strides=(ctypes.c_longlong * 6)(128, -128, 128, 128, 128, 128)), dict(decay=floats(-0.1, 0.2)), dict(decay=floats(float("nan"), -0.2)),
                dict(decay=floats(-0.1, float("-inf")))):
        assert fwd(**bad) == dig.DIG_ERR_INVALID_ARG, bad
    assert fwd(ws=None) == fwd(n=0) == fwd(ws=OK + 8) == dig.DIG_ERR_WORKSPACE
    assert fwd(lengths=OK, dir=2) == dig.DIG_ERR_UNSUPPORTED
    assert list(st)            # a valid array is not refused for its strides: the next argument is
    assert fwd(strides=st, ws=None) == dig.DIG_ERR_WORKSPACE

    def bwd(q=OK, d_out=OK, ds_out=None, dq=OK, dk=OK, dv=OK, ds_in=None, decay=lam, lengths=None, dir=0, n=1 << 30, dtype=1):
        return L.dig_decay_bwd(q, OK, OK, None, decay, lengths, d_out, None, ds_out, dq, dk, dv, ds_in, 1, 2, 2, 4, 4, 64, 64, dir, dtype, OK, n, None)

    for bad in (dict(q=None), dict(d_out=None), dict(dq=None), dict(dk=None), dict(dv=OK + 8), dict(ds_out=OK + 8), dict(ds_in=OK + 8), dict(ds_in=OK, ds_out=OK), dict(decay=floats(1.0, -1.0)), dict(dtype=2)):
        assert bwd(**bad) == dig.DIG_ERR_INVALID_ARG, bad
    assert bwd(n=0) == dig.DIG_ERR_WORKSPACE and bwd(lengths=OK, dir=3) == dig.DIG_ERR_UNSUPPORTED

    def step(q=OK, s_in=OK, out=OK, s_out=OK, decay=lam, B=1, H=2, Hk=2, dk=64, dv=64, dtype=1):
        return L.dig_decay_step(q, OK, OK, decay, s_in, out, s_out, B, H, Hk, dk, dv, dtype, None)

    for bad in (dict(q=None), dict(s_in=None), dict(s_out=OK + 8), dict(out=None), dict(decay=None), dict(decay=floats(0.1, 0.0)), dict(B=0), dict(Hk=3), dict(dk=132), dict(dtype=2),
                dict(B=65536)):
        assert step(**bad) == dig.DIG_ERR_INVALID_ARG, bad


def test_rope_refusals(L):
    from paper_2405_18428_b200 import dig

    def rope(q=OK, k=OK + 64, strides=None, pos=OK, pb=1, axes_n=2, freqs=(ctypes.c_double * 4)(1, 1, 1, 1), axes=(ctypes.c_int * 4)(0, 0, 1, 1), n=4, qo=OK, ko=OK + 64, B=2, Lq=4, H=2, Hk=2,
             d=8, dtype=1):
        return L.dig_rope(q, k, strides, pos, pb, axes_n, freqs, axes, n, qo, ko, B, Lq, H, Hk, d, 0, 0, dtype, None)

    nan = (ctypes.c_double * 4)(1, float("nan"), 1, 1)
    for bad in (dict(q=None), dict(pos=None), dict(pos=OK + 2), dict(freqs=None), dict(axes=None), dict(qo=None), dict(ko=None), dict(k=None), dict(q=OK + 8), dict(B=0), dict(Lq=0),
                dict(H=0), dict(Hk=0), dict(d=12), dict(d=136), dict(dtype=2), dict(pb=3), dict(axes_n=0), dict(axes_n=1), dict(n=0), dict(n=5), dict(n=3), dict(freqs=nan),
                dict(axes=(ctypes.c_int * 4)(0, -1, 1, 1)), dict(ko=OK), dict(qo=OK + 64, ko=OK + 128), dict(qo=OK + 128, ko=OK), dict(strides=(ctypes.c_longlong * 4)(8, 4, 8, 8))):
        assert rope(**bad) == dig.DIG_ERR_INVALID_ARG, bad
    assert rope(B=1 << 20, pb=1, Lq=1 << 20) == rope(H=4097) == rope(H=70000) == dig.DIG_ERR_UNSUPPORTED


def test_rope_freqs():
    from paper_2405_18428_b200 import dig
    freqs, axes = dig.dig_rope_freqs((2, 3), theta=100.0)
    assert axes == [0, 0, 1, 1, 1]
    assert freqs == pytest.approx([1, 0.1, 1, 100 ** (-1 / 3), 100 ** (-2 / 3)])


def test_layernorm_refusals(L):
    from paper_2405_18428_b200 import dig

    def fwd(x=OK, w=None, b=None, y=OK, rows=4, groups=1, D=8, eps=1e-5, dtype=1):
        return L.dig_layernorm_fwd(x, w, b, y, rows, groups, D, eps, dtype, None)

    def bwd(x=OK, dy=OK, w=None, dx=OK, dw=OK, db=OK, rows=4, groups=1, D=8, eps=1e-5, dtype=1, ws=OK, n=1 << 30):
        return L.dig_layernorm_bwd(x, dy, w, dx, dw, db, rows, groups, D, eps, dtype, ws, n, None)

    sizes = (dict(rows=0), dict(groups=0), dict(groups=3), dict(D=0), dict(D=8193), dict(eps=-1.0), dict(eps=float("nan")), dict(dtype=2), dict(rows=70000, groups=70000))
    for bad in (dict(x=None), dict(y=None), dict(x=OK + 2), dict(w=OK + 4), dict(b=OK + 4), *sizes):
        assert fwd(**bad) == dig.DIG_ERR_INVALID_ARG, bad
    for bad in (dict(x=None), dict(dy=None), dict(dx=None), dict(dy=OK + 2), dict(dw=OK + 4), *sizes):
        assert bwd(**bad) == dig.DIG_ERR_INVALID_ARG, bad
    assert bwd(ws=None) == bwd(n=8) == dig.DIG_ERR_WORKSPACE
    assert L.dig_layernorm_bwd_workspace_bytes(4, 3, 8) == L.dig_layernorm_bwd_workspace_bytes(4, 1, 9000) == 0
    assert L.dig_layernorm_bwd_workspace_bytes(4, 1, 8) > 0


def test_binding_refuses_what_it_is_not_given():
    import torch
    from paper_2405_18428_b200 import dig
    z = lambda *s, dtype=torch.bfloat16: torch.zeros(*s, dtype=dtype)
    with pytest.raises(ValueError, match="CUDA tensor"):
        dig.dig_decay_fwd(z(1, 4, 2, 8), z(1, 4, 2, 8), z(1, 4, 2, 8), [0.0, 0.0], 2, 2)
    with pytest.raises(TypeError):
        dig.dig_decay_fwd(z(1, 4, 2, 8, dtype=torch.float16), z(1, 4, 2, 8), z(1, 4, 2, 8), [0.0, 0.0], 2, 2)
    with pytest.raises(ValueError):
        dig.dig_decay_step(z(1, 2, 8), z(1, 2, 8), z(1, 2, 8), [0.0, 0.0], z(1, 2, 8, 8, dtype=torch.float32))
    with pytest.raises(ValueError):
        dig.dig_rope(z(1, 4, 2, 8), None, z(4, 1, dtype=torch.int32), [1.0], [0])
    with pytest.raises(ValueError):
        dig.dig_layernorm_fwd(z(4, 8))
    with pytest.raises(TypeError):
        dig.dig_layernorm_fwd([1.0])
