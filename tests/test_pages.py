"""Refusals of the paged cache in 8 bits and of the operators on pages that need no
GPU, through the C ABI and the binding."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2609_37988_gb300 import build as kbuild

INVALID, UNSUPPORTED = 1, 5


@pytest.fixture(scope="module")
def lib():
    kbuild.build()
    from paper_2609_37988_gb300 import _lib
    return _lib


def _desc(lib, **kw):
    d = dict(n_layers=2, n_q_heads=8, n_kv_heads=2, head_dim=128, page_size=16, n_pages=10, dtype=lib.DTYPE_BF16)
    d.update(kw)
    return lib.PagedDesc(*[d[n] for n, _ in lib.PagedDesc._fields_])


def _plan(lib, **kw):
    pool, exps, ws = (ctypes.c_size_t() for _ in range(3))
    st = lib.load().kvk_paged_coded_plan(ctypes.byref(_desc(lib, **kw)), ctypes.byref(pool), ctypes.byref(exps), ctypes.byref(ws))
    return st, pool.value, exps.value, ws.value


def test_coded_plan(lib):
    st, pool, exps, ws = _plan(lib)
    assert st == 0 and pool == 10 * 2 * 16 * 128 and exps == 20 and ws > 0
    # what operators on pages keep grows with the pool
    assert _plan(lib, n_pages=10 ** 6)[3] >= ws + 4 * (10 ** 6 - 10)
    for kw, want in ((dict(n_layers=0), INVALID), (dict(n_pages=0), INVALID), (dict(page_size=8), UNSUPPORTED),
                     (dict(head_dim=96), UNSUPPORTED), (dict(n_q_heads=7), INVALID), (dict(dtype=lib.DTYPE_F32), INVALID)):
        assert _plan(lib, **kw)[0] == want, kw
    so, z = lib.load(), ctypes.c_size_t()
    assert so.kvk_paged_coded_plan(None, ctypes.byref(z), ctypes.byref(z), ctypes.byref(z)) == INVALID
    assert so.kvk_paged_coded_plan(ctypes.byref(_desc(lib)), ctypes.byref(z), None, ctypes.byref(z)) == INVALID


def test_coded_create_refuses_pools_exponents_and_workspaces(lib):
    so, h = lib.load(), ctypes.c_void_p()
    p = lambda *x: (ctypes.c_void_p * 2)(*x)  # noqa: E731
    ws = _plan(lib)[3]
    ok = p(256, 256)
    for k, v, ke, ve, w, n in ((p(256, 0), ok, ok, ok, 256, ws), (ok, p(256, 272), ok, ok, 256, ws), (ok, ok, p(256, 0), ok, 256, ws),
                               (ok, ok, ok, p(256, 257), 256, ws), (ok, ok, None, ok, 256, ws), (ok, ok, ok, None, 256, ws),
                               (ok, ok, ok, ok, 128, ws), (ok, ok, ok, ok, 256, ws - 1), (None, ok, ok, ok, 256, ws)):
        assert so.kvk_paged_coded_create(ctypes.byref(_desc(lib)), k, v, ke, ve, w, n, ctypes.byref(h)) == INVALID
        assert not h.value
    assert so.kvk_paged_coded_create(ctypes.byref(_desc(lib)), ok, ok, ok, ok, 256, ws, None) == INVALID


def test_null_handles(lib):
    so = lib.load()
    assert so.kvk_paged_copy(None, 256, 256, 1, None) == INVALID
    assert so.kvk_paged_fork(None, 256, 256, 256, 1, 1, 256, 256, 1, 256, 512, 1, None) == INVALID
    assert so.kvk_paged_compact(None, 256, 256, 256, 1, 1, 256, 256, 256, None, None) == INVALID


def test_chunks_hand_registers_over_as_they_were_launched(tmp_path):
    """512 x 128 = 256 x 168 + 256 x 88, allocated in units of 8 a thread."""
    csrc = os.path.join(os.path.dirname(kbuild.__file__), "csrc")
    src, exe = tmp_path / "split.cpp", tmp_path / "split"
    src.write_text('#include "regsplit.h"\n#include <cstdio>\n'
                   'int main() { for (int r = 1; r < 256; ++r) if (kvk::kTcCodesRegs.fits(r)) std::printf("%d ", r); }\n')
    subprocess.run(["g++", "-std=c++17", "-I", csrc, str(src), "-o", str(exe)], check=True)
    got = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()
    assert [int(x) for x in got] == list(range(121, 129))


def test_binding_checks_pools():
    from paper_2609_37988_gb300.serving import PagedCache
    x = torch.zeros((1, 1, 16, 64), dtype=torch.float8_e4m3fn)
    e = torch.zeros((1, 1), dtype=torch.int8)
    for kw in (dict(k_pages=[x], v_pages=[x], k_exps=[e]), dict(k_exps=[e], v_exps=[e]), dict(k_pages=[x], v_pages=[x], bits=16),
               dict(n_layers=1, n_kv_heads=1, head_dim=64, n_pages=1, bits=4)):
        with pytest.raises(ValueError):
            PagedCache(n_q_heads=2, **kw)


@pytest.mark.gpu
def test_refusals_with_a_cache(lib):
    from paper_2609_37988_gb300.serving import KVKError, PagedCache, Rotary
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    for bits in (8, 16):
        c = PagedCache(n_q_heads=2, n_layers=1, n_kv_heads=1, head_dim=64, n_pages=4, bits=bits)
        so, h = lib.load(), c.handle
        refs, table, lens = ints([1, 0, 0, 0]), ints([[0, 0]]), ints([5])
        r, t, l, w = (x.data_ptr() for x in (refs, table, lens, ints([0] * 8)))
        two = ints([0, 0, 0, 0]).data_ptr()
        assert so.kvk_paged_copy(h, r, r, -1, None) == INVALID and so.kvk_paged_copy(h, None, r, 1, None) == INVALID
        assert so.kvk_paged_copy(h, r + 2, r, 1, None) == INVALID and so.kvk_paged_copy(h, None, None, 0, None) == 0
        fork = lambda *a: so.kvk_paged_fork(h, *a, None)  # noqa: E731
        good = [r, t, l, 1, 2, l, l, 1, r, two, 2]
        assert fork(*good[:8], r + 4, *good[9:]) == INVALID  # beside itself
        for at, bad in ((0, None), (1, None), (2, None), (3, -1), (3, 2 ** 25), (4, -1), (4, 2 ** 23), (5, None), (6, l + 1), (7, -1), (7, 16385),
                        (8, None), (8, r + 2), (9, None), (9, t), (9, t + 4), (10, -1), (10, 2 ** 23)):
            assert fork(*good[:at], bad, *good[at + 1:]) == INVALID, at
        compact = lambda *a: so.kvk_paged_compact(h, *a, None)  # noqa: E731
        good = [r, t, l, 1, 2, r, t, w, None]
        for at, bad in ((0, None), (1, None), (2, None), (3, -1), (4, -1), (5, None), (6, None), (6, t + 4), (7, None), (7, w + 2), (8, w + 1), (7, r), (5, r + 4)):
            assert compact(*good[:at], bad, *good[at + 1:]) == INVALID, at
        for call in (lambda: c.copy(ints([0]), ints([0, 1])), lambda: c.copy(ints([[0]]), ints([[0]])),
                     lambda: c.fork(refs[:3], table, lens, lens), lambda: c.fork(refs, table[0], lens, lens),
                     lambda: c.fork(refs, table, lens, lens.long()), lambda: c.fork(refs, table, lens, lens, ints([1, 2])),
                     lambda: c.compact(refs, table, lens, used=ints([1, 2])), lambda: c.free(refs, table, lens, out=table),
                     lambda: c.fork(refs.cpu(), table, lens, lens)):
            with pytest.raises(ValueError):
                call()
        with pytest.raises(KVKError):
            c.fork(refs, table, lens, lens, out=(refs, table))
        # what a cache refuses in 16 bits it refuses in 8
        x = torch.zeros((1, 1, 64), dtype=torch.bfloat16, device="cuda")
        q = torch.zeros((1, 2, 64), dtype=torch.bfloat16, device="cuda")
        cu = ints([0, 1])
        for call in (lambda: c.append(1, x, x, cu, lens, table), lambda: c.append(0, x, x, cu, lens, table, q=q),
                     lambda: c.append(0, x, x, cu, lens, table, rotary=Rotary(head_dim=128)),
                     lambda: c.append(0, x, x, cu, lens, table, rotary=Rotary(head_dim=64, sections=(16, 16))),
                     lambda: c.attend(0, q, cu, lens, table, 0.0), lambda: c.attend(0, q, cu, lens, table, 1.0, window=-1),
                     lambda: c.attend(0, q, cu, lens, table, 1.0, max_new=0), lambda: c.attend(-1, q, cu, lens, table, 1.0)):
            with pytest.raises(KVKError):
                call()
        with pytest.raises(TypeError):
            c.append(0, x.half(), x.half(), cu, lens, table)
        assert c.device_error() == 0


@pytest.mark.gpu
def test_a_fork_of_more_entries_than_are_counted_is_refused(lib):
    """1025 rows of 2^22 pages: those that the rows before the last ask for are 2^32, 0 in 32 bits."""
    from paper_2609_37988_gb300.serving import PagedCache
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    c = PagedCache(n_q_heads=2, n_layers=1, n_kv_heads=1, head_dim=64, n_pages=4)
    refs, parents = ints([0] * 4), ints([-1] * 1025)
    r, p, out = refs.data_ptr(), parents.data_ptr(), ints([0] * 8).data_ptr()
    fork = lambda rows, width: lib.load().kvk_paged_fork(c.handle, r, None, None, 0, 0, p, None, rows, r, out, width, None)  # noqa: E731
    assert fork(1025, 2 ** 22) == INVALID and fork(257, 2 ** 22) == INVALID and fork(1025, 2 ** 21) == INVALID
    assert fork(1, 8) == 0 and fork(1025, 0) == 0
    torch.cuda.synchronize()
    assert c.device_error() == 0 and not refs.any()
