"""Host-side checks of the rotary and cache entry points, without a GPU: sizes
of the argument structures, workspace sizes, refusals (each made before
anything touches the device) and calls with nothing to do."""

from __future__ import annotations

import ctypes
import os
import shutil

import pytest

PTR, WS = 0x10000, 0x20000  # aligned addresses that nothing reads


@pytest.fixture(scope="module")
def lib():
    if shutil.which("nvcc") is None and not os.path.exists("/usr/local/cuda/bin/nvcc"):
        pytest.skip("nvcc not available")
    from paper_2605_29657_gb300 import build
    build.build()
    import paper_2605_29657_gb300 as occ
    return occ.library()


def codes():
    import paper_2605_29657_gb300._lib as L
    return L.OCCAM_ERR_INVALID_ARG, L.OCCAM_ERR_UNSUPPORTED, L.OCCAM_ERR_WORKSPACE


def cache(**kw):
    import paper_2605_29657_gb300._lib as L
    f = dict(layers=2, pages=10, heads=2, dim=64, page_tokens=16, max_seqs=4, max_pages=8, k=PTR, v=PTR, k_scale=PTR,
             v_scale=PTR, table=PTR, length=PTR, refs=PTR)
    f.update(kw)
    return L.CCache(**f)


def size(lib, c, tokens=0):
    n = ctypes.c_size_t(0)
    return lib.occam_cache_workspace_size(ctypes.byref(c), tokens, ctypes.byref(n)), n.value


def test_workspace_size(lib):
    rc, n = size(lib, cache())
    assert rc == 0 and n > 0 and n % 256 == 0
    assert size(lib, cache(), 100000)[1] >= n + 4 * 100000 - 256
    assert size(lib, cache(max_pages=1000))[1] > n
    assert size(lib, cache(), -1)[0] == codes()[0]


@pytest.mark.parametrize("change", [
    dict(layers=0), dict(pages=0), dict(pages=(1 << 24) + 1), dict(layers=65535, pages=1 << 24), dict(heads=0), dict(heads=1025),
    dict(max_seqs=0), dict(max_seqs=65536), dict(max_pages=0), dict(max_pages=1 << 27), dict(k=PTR + 8), dict(v=PTR + 4),
    dict(k=None), dict(k_scale=None), dict(table=None), dict(length=None), dict(refs=None),
    dict(dim=96), dict(dim=32), dict(page_tokens=48), dict(page_tokens=256)])
def test_caches_that_are_refused(lib, change):
    invalid, unsupported, _ = codes()
    want = unsupported if "dim" in change or "page_tokens" in change else invalid
    c = cache(**change)
    assert size(lib, c)[0] == want
    ref = ctypes.byref(c)
    assert lib.occam_cache_extend(ref, 1, PTR, PTR, WS, 1 << 40, None) == want
    assert lib.occam_cache_append(ref, 0, 0, 1, PTR, 128, PTR, 128, 1, PTR, PTR, WS, 1 << 40, None) == want
    assert lib.occam_cache_fork(ref, 1, PTR, PTR, WS, 1 << 40, None) == want
    assert lib.occam_cache_compact(ref, 0, 1, 1, PTR, PTR, PTR, 1, WS, 1 << 40, None) == want
    assert lib.occam_cache_release(ref, 1, PTR, WS, 1 << 40, None) == want
    assert lib.occam_cache_attend(ref, attend(), WS, 1 << 40, None) == want


def attend(**kw):
    import paper_2605_29657_gb300._cache as C
    f = dict(layer=0, dtype=0, heads=4, causal=1, rows=2, q_row=256, q=PTR, out=PTR, lse=None, n=1, max_rows=2, seqs=PTR,
             row_off=PTR, scale=0.0, keep=None, keep_off=None, total_keep=0)
    f.update(kw)
    return C._ATTEND_ARGS.pack(*[0 if x is None else x for x in f.values()])


@pytest.mark.parametrize("change,kind", [
    (dict(layer=2), 0), (dict(layer=-1), 0), (dict(dtype=2), 1), (dict(heads=3), 0), (dict(heads=0), 0), (dict(heads=130), 1),
    (dict(rows=-1), 0), (dict(n=5), 0), (dict(n=-1), 0), (dict(max_rows=-1), 0), (dict(q=PTR + 8), 0), (dict(out=PTR + 2), 0),
    (dict(q_row=255), 0), (dict(q_row=260), 0), (dict(q=None), 0), (dict(out=None), 0), (dict(seqs=None), 0),
    (dict(row_off=None), 0), (dict(scale=-1.0), 0), (dict(scale=float("inf")), 0), (dict(scale=float("nan")), 0),
    (dict(keep=PTR), 0), (dict(keep=PTR, keep_off=PTR, total_keep=-1), 0)])
def test_attend_refusals(lib, change, kind):
    c = cache()
    assert lib.occam_cache_attend(ctypes.byref(c), attend(**change), WS, 1 << 40, None) == codes()[kind]


def test_other_refusals(lib):
    invalid, unsupported, workspace = codes()
    c = cache()
    ref, big, small = ctypes.byref(c), 1 << 40, size(lib, c)[1] - 1
    append = lambda layer=0, dtype=0, rows=1, k=PTR, k_row=128, v=PTR, v_row=128, n=1, seqs=PTR, off=PTR, ws=WS, wn=big: \
        lib.occam_cache_append(ref, layer, dtype, rows, k, k_row, v, v_row, n, seqs, off, ws, wn, None)
    assert append(dtype=2) == unsupported
    for bad in (dict(layer=2), dict(layer=-1), dict(rows=-1), dict(rows=1 << 31), dict(k=None), dict(v=None), dict(k=PTR + 8),
                dict(v=PTR + 2), dict(k_row=120), dict(v_row=132), dict(n=5), dict(seqs=None), dict(off=None)):
        assert append(**bad) == invalid, bad
    for ws, wn in ((None, big), (WS + 128, big), (WS, small)):
        assert append(ws=ws, wn=wn) == workspace
        assert lib.occam_cache_extend(ref, 1, PTR, PTR, ws, wn, None) == workspace
        assert lib.occam_cache_fork(ref, 1, PTR, PTR, ws, wn, None) == workspace
        assert lib.occam_cache_release(ref, 1, PTR, ws, wn, None) == workspace
        assert lib.occam_cache_compact(ref, 0, 1, 1, PTR, PTR, PTR, 1, ws, wn, None) == workspace
        assert lib.occam_cache_attend(ref, attend(), ws, wn, None) == workspace
    # the workspace holds the keep flags' tokens
    assert lib.occam_cache_compact(ref, 0, 1, 1, PTR, PTR, PTR, 1 << 20, WS, small + 1, None) == workspace
    for l0, l1 in ((-1, 1), (0, 3), (2, 1)):
        assert lib.occam_cache_compact(ref, l0, l1, 1, PTR, PTR, PTR, 1, WS, big, None) == invalid
    assert lib.occam_cache_compact(ref, 0, 1, 1, PTR, None, PTR, 1, WS, big, None) == invalid
    assert lib.occam_cache_extend(ref, 5, PTR, PTR, WS, big, None) == invalid
    assert lib.occam_cache_extend(ref, 1, PTR, None, WS, big, None) == invalid
    assert lib.occam_cache_fork(ref, 1, None, PTR, WS, big, None) == invalid
    assert lib.occam_cache_release(ref, 1, None, WS, big, None) == invalid
    assert lib.occam_cache_extend(None, 1, PTR, PTR, WS, big, None) == invalid
    assert lib.occam_cache_attend(ref, None, WS, big, None) == invalid


def test_calls_with_nothing_to_do(lib):
    c = cache()
    ref, big = ctypes.byref(c), 1 << 40
    assert lib.occam_cache_extend(ref, 0, None, None, WS, big, None) == 0
    assert lib.occam_cache_append(ref, 0, 0, 0, None, 0, None, 0, 0, None, None, WS, big, None) == 0
    assert lib.occam_cache_attend(ref, attend(rows=0, n=0, q=None, out=None), WS, big, None) == 0
    assert lib.occam_cache_fork(ref, 0, None, None, WS, big, None) == 0
    assert lib.occam_cache_compact(ref, 0, 2, 0, None, None, None, 0, WS, big, None) == 0
    assert lib.occam_cache_release(ref, 0, None, WS, big, None) == 0
    assert lib.occam_last_call_kernels() == 0


def test_rope_refusals(lib):
    import paper_2605_29657_gb300._lib as L
    invalid, unsupported, _ = codes()

    def rope(dtype=0, rows=2, dim=64, rot=64, pairing=0, pos=PTR, pos_stride=2, axes=3, freq=PTR, axis=PTR, n=1, **t):
        f = dict(src=PTR, dst=PTR, heads=2, src_row=128, src_head=64, dst_row=128, dst_head=64)
        f.update(t)
        x = (L.CRopeTensor * 2)(L.CRopeTensor(**f), L.CRopeTensor(**f))
        return lib.occam_rope(dtype, rows, dim, rot, pairing, 0, pos, pos_stride, axes, freq, axis, n, bytes(x), None)

    assert rope(rows=0) == 0
    for bad in (dict(dtype=3), dict(dim=63), dict(dim=0), dict(dim=1026)):
        assert rope(**bad) == unsupported, bad
    for bad in (dict(rot=66), dict(rot=3), dict(rot=0), dict(rows=-1), dict(axes=0), dict(axes=9), dict(pairing=2), dict(pos=None),
                dict(freq=None), dict(axis=None), dict(n=0), dict(n=3), dict(pos_stride=-1), dict(src=None), dict(dst=None),
                dict(heads=0), dict(heads=65536), dict(src_row=-128), dict(src=PTR + 1), dict(dst=PTR + 1), dict(dtype=2, src=PTR + 2),
                dict(dst_row=256), dict(dst=PTR + 4096, dst_row=0), dict(dst=PTR + 4096, dst_head=32)):
        assert rope(**bad) == invalid, bad
    assert lib.occam_rope(0, 2, 64, 64, 0, 0, PTR, 2, 3, PTR, PTR, 1, None, None) == invalid


def test_rope_results_that_overlap_are_refused(lib):
    """bf16, 3 rows of 2 heads of 64 dims (4 of 2 in the last one), as [rows, heads, dim] unless said."""
    import paper_2605_29657_gb300._lib as L
    invalid, FAR = codes()[0], PTR + (1 << 20)

    def rope(*tensors, rows=3):
        full = [dict(dict(src=PTR, dst=FAR, heads=2, src_row=128, src_head=64, dst_row=128, dst_head=64), **t) for t in tensors]
        x = (L.CRopeTensor * 2)(*[L.CRopeTensor(**f) for f in full])
        return lib.occam_rope(0, rows, 64, 64, 0, 0, PTR, 4, 3, PTR, PTR, len(tensors), bytes(x), None)

    other = dict(src=PTR + (1 << 21), dst=PTR + (1 << 22))
    for bad in (
            [dict(dst_row=64)],                                  # row r's second head is row r + 1's first
            [dict(dst_row=64, dst_head=128)],                    # heads outside rows, rows 0 and 2 of neighbours meet
            [dict(dst_row=100, dst_head=90)],
            [dict(dst=PTR + 2)], [dict(dst=PTR + 128)],          # shifted by an element, by a head
            [dict(dst=PTR + 256)], [dict(dst=PTR - 256)],        # by a row
            [dict(dst=PTR + 64, dst_row=256)],                   # rows of other strides within the input
            [dict(src_row=0, dst=PTR - 256)],                    # onto a row that every row reads
            [dict(), dict(other, dst=FAR)],                      # the same result twice
            [dict(), dict(other, dst=FAR + 128)],
            [dict(dst_row=256), dict(other, dst=FAR + 192, dst_row=256)],  # half a head into the other's rows
            [dict(), dict(other, dst=PTR)], [dict(dst=PTR + (1 << 21)), other],  # onto the other's input
            [dict(dst=PTR), dict(other, src=PTR + 128, dst=PTR + 128)]):  # in place, inputs that share a head
        assert rope(*bad) == invalid, bad
    assert rope(dict(dst_row=200, dst_head=150), rows=4) == invalid
