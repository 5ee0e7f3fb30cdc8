"""Refusals of the decoding step's entry points, before any launch (these calls
never reach the HIP runtime, so they run without a GPU), and of the binding."""

import ctypes
import os

import pytest
import torch

nacl = pytest.importorskip("paper_2408_03675_amd.nacl")
INVALID, UNSUPPORTED, WORKSPACE = nacl.NACL_ERR_INVALID_ARG, nacl.NACL_ERR_UNSUPPORTED, nacl.NACL_ERR_WORKSPACE
B, H, G, T, L, D = 4, 2, 2, 3, 100, 128
AT = 1 << 30
SIZE = 1 << 24


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(nacl.LIB_PATH):
        pytest.skip("libnacl.so not built")
    return nacl.load_library()


def at(i, off=0):
    """Addresses far apart, never dereferenced."""
    return ctypes.c_void_p(AT + i * SIZE + off)


def _prob(**kw):
    return nacl.Problem(kw.get("B", B), H, kw.get("L", L), kw.get("D", D), kw.get("dtype", "bf16"), [0], q_group=G,
                        k_stride=kw.get("k_stride"), v_stride=kw.get("v_stride"))


def _step(p, t=T, **kw):
    s = nacl._Step.from_buffer_copy(nacl.Step(p, t).c)
    for key, value in kw.items():
        if key.endswith("stride"):
            getattr(s, key)[:] = value
        else:
            setattr(s, key, value)
    return s


def _rotation(**kw):
    r = nacl._Rotation()
    r.rot, r.eps, r.inv_freq, r.pos_stride = D, 1e-6, AT + 10 * SIZE, T
    for key, value in kw.items():
        setattr(r, key, value)
    return r


def _rotate(lib, p=None, s=None, r=None, pos=at(11), q=at(0), kn=at(1), vn=at(2), qo=at(3), k=at(4), v=at(5)):
    p = p or _prob()
    s = s or _step(p)
    r = r or _rotation()
    return lib.nacl_rotate_append(p.ref(), ctypes.byref(s), ctypes.byref(r), pos, q, kn, vn, qo, k, v, None)


@pytest.mark.parametrize("kw,code", [
    (dict(t=0), INVALID), (dict(t=-1), INVALID), (dict(t=(1 << 19) + 1), UNSUPPORTED), (dict(row0=-1), INVALID),
    (dict(lens=AT + 2), INVALID), (dict(n_new=AT + 1), INVALID), (dict(q_stride=(-8, 128, 128)), INVALID),
    (dict(q_stride=(1024, 128, 129)), INVALID), (dict(k_stride=(1024, 128, 4)), INVALID),
    (dict(v_stride=(1 << 41, 128, 128)), UNSUPPORTED), (dict(q_out_stride=(1536, 0, 128)), INVALID),
    (dict(q_out_stride=(1536, 384, 64)), INVALID),
])
def test_step_refusals(lib, kw, code):
    p = _prob()
    assert _rotate(lib, p, _step(p, **kw)) == code and lib.nacl_last_error_detail()


@pytest.mark.parametrize("kw,code", [
    (dict(rot=-16), INVALID), (dict(rot=D + 16), INVALID), (dict(rot=24), UNSUPPORTED), (dict(eps=-1.0), INVALID),
    (dict(eps=float("nan")), INVALID), (dict(pos_stride=-1), INVALID), (dict(pos_stride=T - 1), INVALID),
    (dict(inv_freq=None), INVALID), (dict(inv_freq=AT + 2), INVALID), (dict(q_weight=AT + 8), INVALID),
])
def test_rotation_refusals(lib, kw, code):
    assert _rotate(lib, r=_rotation(**kw)) == code and lib.nacl_last_error_detail()


@pytest.mark.parametrize("kw", [
    dict(pos=None), dict(q=None), dict(kn=None), dict(vn=None), dict(qo=None), dict(k=None), dict(v=None),
    dict(q=at(0, 8)), dict(k=at(4, 2)), dict(v=at(4, 4096)), dict(kn=at(4, 4096)), dict(vn=at(5, 256)),
    dict(qo=at(5, 1024)), dict(qo=at(0, 256)), dict(qo=at(1)), dict(qo=at(2, 16)), dict(q=at(5)),
])
def test_rotate_pointer_refusals(lib, kw):
    assert _rotate(lib, **kw) == INVALID and lib.nacl_last_error_detail()


def test_rotate_in_place_needs_the_same_strides(lib):
    p = _prob()
    assert _rotate(lib, p, _step(p, q_out_stride=(4096, 1024, 128)), qo=at(0)) == INVALID
    assert lib.nacl_rotate_append(p.ref(), None, ctypes.byref(_rotation()), at(11), *[at(i) for i in range(6)], None) == INVALID
    s = _step(p)
    assert lib.nacl_rotate_append(p.ref(), ctypes.byref(s), None, at(11), *[at(i) for i in range(6)], None) == INVALID
    assert _rotate(lib, _prob(D=96)) == UNSUPPORTED


def _prefix(**kw):
    x = nacl._Prefix()
    x.G, x.L, x.k, x.v = 2, 1000, AT + 6 * SIZE, AT + 7 * SIZE
    x.k_stride[:] = x.v_stride[:] = (H * 1000 * D, 1000 * D, D)
    for key, value in kw.items():
        if key.endswith("stride"):
            getattr(x, key)[:] = value
        else:
            setattr(x, key, value)
    return x


def _attend(lib, p=None, s=None, x=None, q=at(0), k=at(4), v=at(5), out=at(1), lse=at(2), ws=at(8), n=None):
    p = p or _prob()
    s = s or _step(p)
    x = x or _prefix()
    if n is None:
        n = lib.nacl_prefix_workspace_bytes(p.ref(), ctypes.byref(s), ctypes.byref(x)) or 1 << 30
    return lib.nacl_prefix_attention(p.ref(), ctypes.byref(s), ctypes.byref(x), q, k, v, out, lse, ws, n, None)


@pytest.mark.parametrize("kw,code", [
    (dict(G=0), INVALID), (dict(G=3), INVALID), (dict(L=0), INVALID), (dict(L=(1 << 19) + 1), UNSUPPORTED),
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(k=AT + 8), INVALID), (dict(lens=AT + 1), INVALID),
    (dict(k_stride=(128, 128, 64)), INVALID), (dict(v_stride=(128, 128, 0)), INVALID),
    (dict(k_stride=(-8, 128, 128)), INVALID), (dict(v_stride=(128, 100, 128)), INVALID),
    (dict(k_stride=(128, 128, 1 << 21)), UNSUPPORTED), (dict(L=10, v_stride=(128, 128, 1 << 23)), UNSUPPORTED),
])
def test_prefix_refusals(lib, kw, code):
    assert _attend(lib, x=_prefix(**kw)) == code and lib.nacl_last_error_detail()


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(out=None), INVALID),
    (dict(q=at(0, 2)), INVALID), (dict(out=at(1, 8)), INVALID), (dict(lse=at(2, 2)), INVALID),
    (dict(out=at(4, 512)), INVALID), (dict(lse=at(5, 512)), INVALID), (dict(ws=at(6, 1024)), INVALID),
    (dict(out=at(7)), INVALID), (dict(lse=at(1, 256)), INVALID), (dict(ws=at(1)), INVALID), (dict(ws=at(0)), INVALID),
    (dict(ws=None), WORKSPACE), (dict(ws=at(8, 16)), WORKSPACE), (dict(n=256), WORKSPACE),
])
def test_attend_pointer_refusals(lib, kw, code):
    assert _attend(lib, **kw) == code and lib.nacl_last_error_detail()


def test_attend_row_strides_and_sizes(lib):
    assert _attend(lib, _prob(k_stride=(H * L * D, L * D, 0))) == INVALID
    assert _attend(lib, _prob(v_stride=(H * L * D, L * D, 1 << 23))) == UNSUPPORTED
    p = _prob(B=4)
    s = _step(p, 1 << 19)
    assert lib.nacl_prefix_workspace_bytes(p.ref(), ctypes.byref(s), None) > 0
    big = nacl.Problem(32, 32, L, D, "bf16", [0], q_group=8)
    s = _step(big, 1 << 13)
    assert lib.nacl_prefix_workspace_bytes(big.ref(), ctypes.byref(s), None) == 0
    assert b"2^26" in lib.nacl_last_error_detail()
    assert lib.nacl_prefix_workspace_bytes(p.ref(), None, None) == 0


def _draw(**kw):
    d = nacl._draw(5, 1000)
    for key, value in kw.items():
        setattr(d, key, value)
    return d


def _sample(lib, d=None, x=at(0), u=at(1), tok=at(2), lp=at(3), ws=at(4), n=1 << 24):
    return lib.nacl_sample(ctypes.byref(d or _draw()), x, u, tok, lp, ws, n, None)


@pytest.mark.parametrize("kw,code", [
    (dict(N=0), INVALID), (dict(V=0), INVALID), (dict(N=65536), UNSUPPORTED), (dict(V=(1 << 20) + 1, stride=1 << 21), UNSUPPORTED),
    (dict(dtype=7), INVALID), (dict(stride=999), INVALID), (dict(stride=1 << 41), UNSUPPORTED),
    (dict(temperature=AT + 2), INVALID), (dict(top_k=AT + 1), INVALID), (dict(top_p=AT + 3), INVALID), (dict(min_p=AT + 2), INVALID),
])
def test_draw_refusals(lib, kw, code):
    assert _sample(lib, _draw(**kw)) == code and lib.nacl_last_error_detail()
    assert lib.nacl_sample_workspace_bytes(ctypes.byref(_draw(**kw))) == 0


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), INVALID), (dict(u=None), INVALID), (dict(tok=None), INVALID), (dict(x=at(0, 2)), INVALID),
    (dict(u=at(1, 1)), INVALID), (dict(tok=at(2, 2)), INVALID), (dict(lp=at(3, 3)), INVALID), (dict(tok=at(0, 400)), INVALID),
    (dict(lp=at(1)), INVALID), (dict(lp=at(2, 8)), INVALID), (dict(ws=None), WORKSPACE), (dict(ws=at(4, 64)), WORKSPACE),
    (dict(ws=at(0)), INVALID), (dict(n=0), WORKSPACE), (dict(d=_draw(top_p=AT + 2 * SIZE)), INVALID),
])
def test_sample_pointer_refusals(lib, kw, code):
    assert _sample(lib, **kw) == code and lib.nacl_last_error_detail()
    assert lib.nacl_sample(None, at(0), at(1), at(2), at(3), at(4), 1 << 24, None) == INVALID


def test_the_binding_refuses_host_tensors():
    prob = nacl.Problem(1, 2, 64, 64, "bf16", [63])
    q = torch.zeros((1, 2, 1, 64), dtype=torch.bfloat16)
    k = torch.zeros((1, 2, 64, 64), dtype=torch.bfloat16)
    step = nacl.Step(prob)
    for call in (lambda: nacl.Step(prob, lens=torch.zeros(1, dtype=torch.int32)),
                 lambda: nacl.Rotation(prob, torch.ones(32)), lambda: nacl.Prefix(prob, k, k),
                 lambda: nacl.rotate_append(prob, step, nacl.Rotation(prob), None, q, q, q, k, k),
                 lambda: nacl.prefix_attention(prob, step, q, k, k),
                 lambda: nacl.sample(torch.zeros((2, 5)), torch.zeros(2))):
        with pytest.raises(ValueError, match="on the GPU"):
            call()


@pytest.mark.parametrize("i", [0, 1, 2])
@pytest.mark.parametrize("name", ["k_stride", "v_stride"])
def test_rotate_needs_cache_rows_apart(lib, name, i):
    st = [H * L * D, L * D, D]
    for low in (0, D - 8):
        st[i] = low
        assert _rotate(lib, _prob(**{name: tuple(st)})) == INVALID and lib.nacl_last_error_detail()


def test_rotate_in_place_needs_its_own_memory(lib):
    assert _rotate(lib, qo=at(0), kn=at(0)) == INVALID
    assert _rotate(lib, qo=at(0), vn=at(0)) == INVALID


def test_sizes_past_32_bits_are_refused():
    p = _prob()
    for kw in (dict(T=2 ** 32 + 1), dict(row0=2 ** 32), dict(row0=-2 ** 31 - 1)):
        with pytest.raises(ValueError, match="32 bits"):
            nacl.Step(p, **kw)
    for n, v in ((2 ** 32 + 1, 100), (1, 2 ** 32 + 100)):
        with pytest.raises(ValueError, match="32 bits"):
            nacl.sample_workspace(n, v)


def test_rows_and_groups_past_32_bits_are_refused():
    """2^32 + 1 of them would pass for one."""
    n = 2 ** 32 + 1
    with pytest.raises(ValueError, match="32 bits"):
        nacl.sample(torch.empty((n, 1), device="meta"), torch.empty(n, device="meta"))
    k = torch.empty((1, 2, 64, 64), dtype=torch.bfloat16, device="meta").expand(n, 2, 64, 64)
    with pytest.raises(ValueError, match="32 bits"):
        nacl.Prefix(nacl.Problem(1, 2, 64, 64, "bf16", [63]), k, k)
