"""Refusals of the serving entry points that need no GPU: descriptors,
frequencies, strides and null arguments through the C ABI, shapes and dtypes
through the binding."""
import ctypes

import pytest
import torch

from paper_2609_37988_gb300 import build as kbuild

INVALID, UNSUPPORTED = 1, 5


@pytest.fixture(scope="module")
def lib():
    kbuild.build()
    from paper_2609_37988_gb300 import _lib
    return _lib


def _paged(lib, **kw):
    d = dict(n_layers=2, n_q_heads=8, n_kv_heads=2, head_dim=128, page_size=16, n_pages=10, dtype=lib.DTYPE_BF16)
    d.update(kw)
    return lib.PagedDesc(*[d[n] for n, _ in lib.PagedDesc._fields_])


def _plan(lib, **kw):
    pool, ws = ctypes.c_size_t(), ctypes.c_size_t()
    st = lib.load().kvk_paged_plan(ctypes.byref(_paged(lib, **kw)), ctypes.byref(pool), ctypes.byref(ws))
    return st, pool.value, ws.value


def test_paged_plan(lib):
    st, pool, ws = _plan(lib)
    assert st == 0 and pool == 10 * 2 * 16 * 128 * 2 and 0 < ws < 64 << 20
    for kw, want in ((dict(n_layers=0), INVALID), (dict(n_pages=0), INVALID), (dict(page_size=8), UNSUPPORTED),
                     (dict(page_size=48), UNSUPPORTED), (dict(n_q_heads=7), INVALID), (dict(n_kv_heads=0), INVALID),
                     (dict(head_dim=96), UNSUPPORTED), (dict(n_q_heads=130), UNSUPPORTED), (dict(dtype=lib.DTYPE_F32), INVALID),
                     (dict(dtype=9), INVALID), (dict(head_dim=-1), INVALID)):
        assert _plan(lib, **kw)[0] == want, kw
    assert lib.load().kvk_paged_plan(None, None, None) == INVALID
    assert lib.load().kvk_paged_plan(ctypes.byref(_paged(lib)), None, None) == INVALID


def test_null_handles(lib):
    so = lib.load()
    b = ctypes.byref(lib.PagedBatch())
    r = ctypes.byref(lib.Rows(1, 128, 128))
    code = ctypes.c_int32()
    assert so.kvk_paged_create(ctypes.byref(_paged(lib)), None, None, None, 0, None) == INVALID
    h = ctypes.c_void_p()
    assert so.kvk_paged_create(ctypes.byref(_paged(lib)), None, None, None, 0, ctypes.byref(h)) == INVALID and not h.value
    assert so.kvk_paged_reset(None, None) == INVALID
    assert so.kvk_paged_append(None, 0, b, r, r, None, None, None, None, None) == INVALID
    assert so.kvk_paged_attention(None, 0, b, r, 1.0, 1, 0, None, None) == INVALID
    assert so.kvk_paged_get_device_error(None, None, ctypes.byref(code)) == INVALID
    assert so.kvk_paged_destroy(None) == 0 and so.kvk_rotary_destroy(None) == 0
    assert so.kvk_rotary_apply(None, r, r, 1, r, r, 1, 0, 1, None, None) == INVALID


def test_paged_create_refuses_pools_and_workspaces(lib):
    so = lib.load()
    h = ctypes.c_void_p()
    pools = lambda *p: (ctypes.c_void_p * 2)(*p)  # noqa: E731
    _, _, ws = _plan(lib)
    for k, v, w, n in ((pools(256, 0), pools(256, 256), 256, ws), (pools(256, 256), pools(256, 272), 256, ws),
                       (pools(256, 256), pools(256, 256), 128, ws), (pools(256, 256), pools(256, 256), 256, ws - 1),
                       (pools(256, 256), pools(256, 256), 0, ws)):
        assert so.kvk_paged_create(ctypes.byref(_paged(lib)), k, v, w, n, ctypes.byref(h)) == INVALID
        assert not h.value


def _rotary(lib, head_dim=64, rotary_dim=64, n_axes=1, freq=None, axis=None, adjacent=0, factor=1.0):
    n = max(rotary_dim // 2, 1)
    h = ctypes.c_void_p()
    st = lib.load().kvk_rotary_create(head_dim, rotary_dim, n_axes, (ctypes.c_double * n)(*(freq or [0.5] * n)),
                                      (ctypes.c_int32 * n)(*(axis or [0] * n)), adjacent, factor, ctypes.byref(h))
    return st, h


def test_rotary_create(lib):
    nan = float("nan")
    for kw in (dict(head_dim=63), dict(head_dim=258), dict(head_dim=0), dict(rotary_dim=66), dict(rotary_dim=0), dict(rotary_dim=31),
               dict(n_axes=0), dict(n_axes=9), dict(adjacent=2), dict(factor=nan), dict(freq=[nan] * 32), dict(axis=[1] * 32),
               dict(axis=[-1] * 32)):
        st, h = _rotary(lib, **kw)
        assert st == INVALID and not h.value, kw
    st, h = _rotary(lib)
    assert st == 0
    so = lib.load()
    rows = lambda *a: ctypes.byref(lib.Rows(*a))  # noqa: E731
    ok, apply = rows(256, 64, 64), so.kvk_rotary_apply
    assert apply(h, ok, ok, 1, None, None, 0, 7, 4, 256, None) == INVALID        # dtype
    assert apply(h, ok, ok, 1, None, None, 0, 1, -1, 256, None) == INVALID       # tokens
    assert apply(h, ok, ok, 1, None, None, 0, 1, 4, None, None) == INVALID       # positions
    assert apply(h, None, ok, 1, None, None, 0, 1, 4, 256, None) == INVALID      # q
    assert apply(h, ok, None, 1, None, None, 0, 1, 4, 256, None) == INVALID      # q_out
    assert apply(h, rows(256, 0, 64), ok, 1, None, None, 0, 1, 4, 256, None) == INVALID   # one row for all tokens
    assert apply(h, rows(256, 128, 0), ok, 2, None, None, 0, 1, 4, 256, None) == INVALID  # one row for all heads
    assert apply(h, ok, ok, 1, None, None, 0, 1, 0, None, None) == 0             # no tokens
    assert so.kvk_rotary_destroy(h) == 0


def test_rotary_refuses_misaligned_pointers(lib):
    _, h = _rotary(lib)
    so = lib.load()
    rows = lambda *a: ctypes.byref(lib.Rows(*a))  # noqa: E731
    ok = rows(256, 64, 64)
    for q, q_out, dtype, pos in ((rows(257, 64, 64), ok, 1, 256), (ok, rows(257, 64, 64), 1, 256), (rows(258, 64, 64), ok, 0, 256),
                                 (ok, ok, 1, 258)):
        assert so.kvk_rotary_apply(h, q, q_out, 1, None, None, 0, dtype, 4, pos, None) == INVALID
    assert so.kvk_rotary_destroy(h) == 0


def test_prompt_attention_refuses_subnormal_scales_and_misaligned_words(lib):
    so = lib.load()
    ok = ctypes.byref(lib.Rows(256, 1024, 128))
    for cu, scale, error in ((256, 1e-40, None), (258, 1.0, None), (256, 1.0, 257)):
        assert so.kvk_prompt_attention(ok, ok, ok, 4, 8, 8, 128, lib.DTYPE_BF16, cu, 1, scale, 0, 256, error, None) == INVALID


def test_prompt_attention_refusals(lib):
    so = lib.load()
    rows = lambda *a: ctypes.byref(lib.Rows(*a))  # noqa: E731
    ok = rows(256, 1024, 128)

    def call(q=ok, k=ok, v=ok, n=4, hq=8, hkv=8, d=128, dtype=lib.DTYPE_BF16, cu=256, B=1, scale=1.0, window=0, out=256):
        return so.kvk_prompt_attention(q, k, v, n, hq, hkv, d, dtype, cu, B, scale, window, out, None, None)

    for kw, want in ((dict(hq=7, hkv=2), INVALID), (dict(d=96), UNSUPPORTED), (dict(hq=130, hkv=2), UNSUPPORTED),
                     (dict(dtype=lib.DTYPE_F32), INVALID), (dict(cu=None), INVALID), (dict(out=None), INVALID), (dict(out=264), INVALID),
                     (dict(scale=0.0), INVALID), (dict(scale=float("inf")), INVALID), (dict(scale=float("nan")), INVALID),
                     (dict(window=-1), INVALID), (dict(n=-1), INVALID), (dict(B=-1), INVALID), (dict(n=2 ** 30), INVALID),
                     (dict(q=None), INVALID), (dict(k=rows(264, 1024, 128)), INVALID), (dict(v=rows(256, 1020, 128)), INVALID),
                     (dict(v=rows(256, 1024, 64)), INVALID), (dict(k=rows(256, -1024, 128)), INVALID)):
        assert call(**kw) == want, kw
    assert call(n=0, q=None, k=None, v=None, cu=None, out=None) == 0
    assert call(B=0, cu=None) == 0


def test_binding_checks_shapes():
    from paper_2609_37988_gb300.serving import PagedCache, Rotary, prompt_attention
    with pytest.raises(ValueError):
        Rotary(head_dim=64, sections=(16, 8))
    with pytest.raises(ValueError):
        Rotary(head_dim=64, sections=(32,), axes=[0] * 32)
    with pytest.raises(ValueError):
        Rotary(head_dim=64, inv_freq=[1.0])
    rot = Rotary(head_dim=64, sections=(16, 8, 8))
    assert rot.n_axes == 3
    x = torch.zeros((4, 2, 64))
    pos = torch.zeros((3, 4), dtype=torch.int32)
    for args in ((x, None, pos), (None, None, pos), (x[0], None, pos)):  # not on a GPU, nothing, no tokens
        with pytest.raises(ValueError):
            rot.apply(*args)
    with pytest.raises(ValueError):
        prompt_attention(x, x, x, torch.zeros((2,), dtype=torch.int32), 1.0)
    with pytest.raises(ValueError):
        PagedCache(n_q_heads=2)
    with pytest.raises(ValueError):
        PagedCache(n_q_heads=2, k_pages=[torch.zeros((1, 1, 16, 64))])
    with pytest.raises(ValueError):
        PagedCache(n_q_heads=2, k_pages=[torch.zeros((1, 1, 16, 64))], v_pages=[torch.zeros((1, 1, 16, 64))])
    with pytest.raises(TypeError):
        PagedCache(n_q_heads=2, n_layers=1, n_kv_heads=1, head_dim=64, n_pages=1, dtype=torch.float64, device="cuda:0")


def test_give_up_of_no_cache(lib):
    assert lib.load().kvk_paged_set_give_up(None, 0) == INVALID


def test_prompt_errors_need_a_place_and_give_up_a_truth_value(lib):
    assert lib.load().kvk_prompt_get_device_error(None, None) == INVALID
    assert lib.load().kvk_prompt_set_give_up(2) == INVALID
