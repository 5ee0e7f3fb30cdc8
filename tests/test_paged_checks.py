"""Refusals of the paged cache's and beam search's entry points, before any launch
(these calls never reach the HIP runtime, so they run without a GPU), and of the
binding."""

import ctypes

import pytest
import torch

nacl = pytest.importorskip("paper_2408_03675_amd.nacl")
from test_step_checks import AT, SIZE, _rotation, at, lib  # noqa: F401 (lib: the fixture)

INVALID, UNSUPPORTED, WORKSPACE = nacl.NACL_ERR_INVALID_ARG, nacl.NACL_ERR_UNSUPPORTED, nacl.NACL_ERR_WORKSPACE
B, H, G, T, L, D = 4, 2, 2, 3, 100, 128
N, PAGE, ENTRIES = 32, 16, 7


def _prob(**kw):
    return nacl.Problem(kw.get("B", B), H, kw.get("L", L), kw.get("D", D), kw.get("dtype", "bf16"), [0], q_group=G)


def _pages(**kw):
    x = nacl._Pages()
    x.n_pages, x.page, x.entries, x.table_stride = N, PAGE, ENTRIES, ENTRIES
    x.k_stride[:] = x.v_stride[:] = (H * PAGE * D, PAGE * D, D)
    x.k, x.v, x.table = AT + 4 * SIZE, AT + 5 * SIZE, AT + 6 * SIZE
    for key, value in kw.items():
        if key.endswith("_stride") and key != "table_stride":
            getattr(x, key)[:] = value
        else:
            setattr(x, key, value)
    return x


def _step(p, t=T):
    return nacl._Step.from_buffer_copy(nacl.Step(p, t).c)


def _assign(lib, p=None, s=None, x=None, held=at(10), shared=at(11), free=at(12), n_free=at(13), held_out=at(14),
            n_out=at(15), slots=at(16), missing=at(17)):
    p = p or _prob()
    return lib.nacl_pages_assign(p.ref(), ctypes.byref(s or _step(p)), ctypes.byref(x or _pages()), held, shared, free, n_free,
                                 held_out, n_out, slots, missing, None)


def _append(lib, p=None, s=None, r=None, x=None, pos=at(20), q=at(0), kn=at(1), vn=at(2), qo=at(3), slots=at(16)):
    p = p or _prob()
    return lib.nacl_paged_append(p.ref(), ctypes.byref(s or _step(p)), ctypes.byref(r or _rotation()), pos, q, kn, vn,
                                 ctypes.byref(x or _pages()), slots, qo, None)


def _attend(lib, p=None, s=None, x=None, q=at(0), out=at(1), lse=at(2), ws=at(8), n=None):
    p, x = p or _prob(), x or _pages()
    s = s or _step(p)
    if n is None:
        n = lib.nacl_paged_workspace_bytes(p.ref(), ctypes.byref(s), ctypes.byref(x)) or 1 << 30
    return lib.nacl_paged_attention(p.ref(), ctypes.byref(s), ctypes.byref(x), q, out, lse, ws, n, None)


def _reorder(lib, p=None, x=None, W=2, parents=at(20), lens=at(21), held=at(22), table=at(23), stride=ENTRIES, lens_out=at(24),
             held_out=at(25)):
    p = p or _prob()
    return lib.nacl_beam_reorder(p.ref(), ctypes.byref(x or _pages()), W, parents, lens, held, table, stride, lens_out, held_out,
                                 None)


@pytest.mark.parametrize("kw,code", [
    (dict(n_pages=0), INVALID), (dict(page=0), INVALID), (dict(entries=0), INVALID), (dict(page=-1), INVALID),
    (dict(entries=(1 << 20) + 1, table_stride=1 << 21), UNSUPPORTED),
    (dict(n_pages=1 << 20, page=1 << 11), UNSUPPORTED), (dict(table_stride=ENTRIES - 1), INVALID),
    (dict(table_stride=1 << 33), UNSUPPORTED), (dict(table=AT + 6 * SIZE + 2), INVALID),
])
def test_table_refusals(lib, kw, code):  # noqa: F811
    for call in (_assign, _append, _attend, _reorder):
        assert call(lib, x=_pages(**kw)) == code and lib.nacl_last_error_detail()
    p = _prob()
    assert lib.nacl_paged_workspace_bytes(p.ref(), ctypes.byref(_step(p)), ctypes.byref(_pages(**kw))) == 0


@pytest.mark.parametrize("kw,code", [
    (dict(k=None), INVALID), (dict(v=AT + 5 * SIZE + 8), INVALID), (dict(k_stride=(4096, 2048, 4)), INVALID),
    (dict(v_stride=(-8, 2048, 128)), INVALID), (dict(k_stride=(1 << 41, 2048, 128)), UNSUPPORTED),
    (dict(n_pages=1 << 26, v_stride=(1 << 33, 2048, 128)), UNSUPPORTED),
])
def test_pool_refusals(lib, kw, code):  # noqa: F811
    for call in (_append, _attend, _reorder):
        assert call(lib, x=_pages(**kw)) == code and lib.nacl_last_error_detail()


@pytest.mark.parametrize("kw", [
    dict(k_stride=(2048, 2048, 128)), dict(k_stride=(4096, 2048, 64)), dict(v_stride=(4096, 0, 128)),
    dict(v=AT + 4 * SIZE), dict(v=AT + 4 * SIZE + 4096), dict(v=AT + 4 * SIZE + 256, k_stride=(8192, 4096, 128)),
    # K and V in one buffer, with V's rows over K's.
    dict(v=AT + 4 * SIZE + 2 * 4096, k_stride=(4096, 2048, 128), v_stride=(4096, 2048, 128)),
    dict(v=AT + 4 * SIZE + 128, k_stride=(8192, 4096, 256), v_stride=(8192, 4096, 256)),
])
def test_written_pools_lie_apart(lib, kw):  # noqa: F811
    for call in (_append, _reorder):
        assert call(lib, x=_pages(**kw)) == INVALID and b"overlap" in lib.nacl_last_error_detail()


@pytest.mark.parametrize("kw", [
    dict(table=None), dict(held=None), dict(free=None), dict(n_free=None), dict(held_out=None), dict(n_out=None), dict(slots=None),
    dict(held=at(10, 2)), dict(missing=at(17, 1)), dict(free=at(6)), dict(held_out=at(10, 4)), dict(n_out=at(14)),
    dict(slots=at(12)), dict(missing=at(15)), dict(shared=at(14)), dict(n_out=at(13, -4), n_free=at(13, -4), missing=at(13, -4)),
])
def test_assign_refusals(lib, kw):  # noqa: F811
    x = _pages(**{k: v for k, v in kw.items() if k == "table"})
    assert _assign(lib, x=x, **{k: v for k, v in kw.items() if k != "table"}) == INVALID and lib.nacl_last_error_detail()


@pytest.mark.parametrize("kw", [
    dict(slots=None), dict(slots=at(16, 2)), dict(pos=None), dict(q=None), dict(q=at(0, 8)), dict(kn=at(4, 4096)),
    dict(vn=at(5)), dict(qo=at(4)), dict(qo=at(0, 256)), dict(qo=at(1)),
])
def test_append_refusals(lib, kw):  # noqa: F811
    assert _append(lib, **kw) == INVALID and lib.nacl_last_error_detail()


def test_append_rotation_refusals(lib):  # noqa: F811
    assert _append(lib, r=_rotation(rot=24)) == UNSUPPORTED
    assert _append(lib, p=_prob(D=96)) == UNSUPPORTED
    p = _prob()
    assert lib.nacl_paged_append(p.ref(), ctypes.byref(_step(p)), ctypes.byref(_rotation()), at(20), at(0), at(1), at(2), None,
                                 at(16), at(3), None) == INVALID


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), INVALID), (dict(out=None), INVALID), (dict(out=at(1, 8)), INVALID), (dict(lse=at(2, 2)), INVALID),
    (dict(n=0), WORKSPACE), (dict(ws=None), WORKSPACE), (dict(ws=at(8, 128)), WORKSPACE), (dict(out=at(0)), INVALID),
    (dict(out=at(4, 512)), INVALID), (dict(lse=at(5)), INVALID), (dict(lse=at(6)), INVALID), (dict(ws=at(1)), INVALID),
])
def test_attention_refusals(lib, kw, code):  # noqa: F811
    assert _attend(lib, **kw) == code and lib.nacl_last_error_detail()
    assert _attend(lib, x=_pages(table=None)) == INVALID


def test_attention_size_refusals(lib):  # noqa: F811
    p = nacl.Problem(60000, 1, 64, 128, "bf16", [0], q_group=64)
    assert _attend(lib, p, _step(p, 20)) == UNSUPPORTED


def _beams(lib, logits=at(0), scores=at(1), parents=at(2), tokens=at(3), out=at(4), ws=at(8), n=None, **kw):
    d = nacl._Beams(2, 3, 1000, 4, nacl.NACL_F32, 1000, 5, AT + 9 * SIZE)
    for key, value in kw.items():
        setattr(d, key, value)
    if n is None:
        n = lib.nacl_beam_workspace_bytes(ctypes.byref(d)) or 1 << 30
    return lib.nacl_beam_select(ctypes.byref(d), logits, scores, parents, tokens, out, ws, n, None)


@pytest.mark.parametrize("kw,code", [
    (dict(B=0), INVALID), (dict(W=0), INVALID), (dict(V=0), INVALID), (dict(K=0), INVALID), (dict(W=65), UNSUPPORTED),
    (dict(K=65), UNSUPPORTED), (dict(B=30000), UNSUPPORTED), (dict(V=(1 << 20) + 1, stride=1 << 21), UNSUPPORTED),
    (dict(W=64, V=1 << 18, stride=1 << 18), UNSUPPORTED), (dict(dtype=7), INVALID), (dict(stride=999), INVALID),
    (dict(stride=1 << 41), UNSUPPORTED), (dict(end_token=-1), INVALID), (dict(end_token=1000), INVALID),
    (dict(ended=AT + 9 * SIZE + 2), INVALID),
])
def test_beam_refusals(lib, kw, code):  # noqa: F811
    assert _beams(lib, **kw) == code and lib.nacl_last_error_detail()
    d = nacl._Beams(2, 3, 1000, 4, nacl.NACL_F32, 1000, 5, AT + 9 * SIZE)
    for key, value in kw.items():
        setattr(d, key, value)
    assert lib.nacl_beam_workspace_bytes(ctypes.byref(d)) == 0


@pytest.mark.parametrize("kw,code", [
    (dict(logits=None), INVALID), (dict(scores=None), INVALID), (dict(parents=None), INVALID), (dict(tokens=None), INVALID),
    (dict(out=None), INVALID), (dict(logits=at(0, 2)), INVALID), (dict(out=at(4, 2)), INVALID), (dict(n=255), WORKSPACE),
    (dict(ws=None), WORKSPACE), (dict(ws=at(8, 64)), WORKSPACE), (dict(tokens=at(2)), INVALID), (dict(out=at(0, 4096)), INVALID),
    (dict(parents=at(9)), INVALID), (dict(ws=at(1)), INVALID),
])
def test_beam_pointer_refusals(lib, kw, code):  # noqa: F811
    assert _beams(lib, **kw) == code and lib.nacl_last_error_detail()


@pytest.mark.parametrize("kw,code", [
    (dict(W=0), INVALID), (dict(W=3), INVALID), (dict(stride=ENTRIES - 1), INVALID), (dict(stride=1 << 33), UNSUPPORTED),
    (dict(parents=None), INVALID), (dict(lens=None), INVALID), (dict(table=None), INVALID), (dict(lens_out=None), INVALID),
    (dict(held=None), INVALID), (dict(held_out=None), INVALID), (dict(lens_out=at(24, 2)), INVALID), (dict(table=at(6)), INVALID),
    (dict(lens_out=at(21)), INVALID), (dict(held_out=at(22)), INVALID), (dict(lens_out=at(4)), INVALID),
    (dict(table=at(5, 64)), INVALID), (dict(held_out=at(24)), INVALID),
])
def test_reorder_refusals(lib, kw, code):  # noqa: F811
    assert _reorder(lib, **kw) == code and lib.nacl_last_error_detail()
    assert _reorder(lib, p=_prob(B=65), W=65) == UNSUPPORTED


def test_binding_refuses_host_tensors_and_wrong_shapes(lib):  # noqa: F811
    prob = nacl.Problem(2, 1, 32, 64, "bf16", [0])
    pool, table = torch.zeros((4, 1, 16, 64), dtype=torch.bfloat16), torch.zeros((2, 2), dtype=torch.int32)
    i32 = torch.zeros((2,), dtype=torch.int32)
    with pytest.raises(ValueError, match="on the GPU"):
        nacl.Pages(prob, pool, pool, table)
    with pytest.raises(ValueError, match="n_pages, H, page, D"):
        nacl.Pages(prob, pool[0], pool, table)
    with pytest.raises(ValueError, match="on the GPU"):
        nacl.pages_assign(nacl.Step(prob, 1), 16, table, i32, i32, i32[:1])
    with pytest.raises(ValueError, match="B, entries"):
        nacl.pages_assign(nacl.Step(prob, 1), 16, i32, i32, i32, i32[:1])
    with pytest.raises(ValueError, match="on the GPU"):
        nacl.beam_select(torch.zeros((2, 10)), torch.zeros((1, 2)), 2)
    with pytest.raises(ValueError, match="logits must be"):
        nacl.beam_select(torch.zeros((2, 10), dtype=torch.float16), torch.zeros((1, 2)), 2)
    with pytest.raises(ValueError, match="32 bits"):
        nacl.beam_workspace(1, 1, 1 << 31, 1)
    with pytest.raises(nacl.NaclError):
        nacl.beam_workspace(1, 65, 1000, 1, "cpu")
