"""Host-side checks of whole-prompt attention, its gradient, append with the rotation and attention over shared
pages, without a GPU: sizes of the argument structures, workspace sizes, refusals (each made before anything touches the
device) and calls with nothing to do."""

from __future__ import annotations

import ctypes
import subprocess

import pytest

from test_cache_abi_cpu import PTR, WS, attend, cache, codes, lib, size  # noqa: F401  (lib: the fixture)

BIG, FAR = 1 << 40, 1 << 32


def test_argument_structures_have_the_header_s_sizes(lib, tmp_path):
    import os
    import paper_2605_29657_gb300._lib as L
    import paper_2605_29657_gb300._prompt as P
    names = dict(occam_prompt_args=L.CPromptArgs, occam_prompt_grads=L.CPromptGrads, occam_append_rope_args=L.CAppendRopeArgs)
    lines = [f'printf("%zu\\n", sizeof({n}));' for n in names]
    fields = [("occam_prompt_args", L.CPromptArgs, f) for f in ("total_rows", "q", "q_row", "row_off", "scale")]
    fields += [("occam_prompt_grads", L.CPromptGrads, f) for f in ("lse", "dv", "dout_row", "dv_row")]
    fields += [("occam_append_rope_args", L.CAppendRopeArgs, f) for f in ("total_rows", "k_row", "positions", "axis", "q")]
    lines += [f'printf("%zu\\n", offsetof({n}, {f}));' for n, _, f in fields]
    src = tmp_path / "s.c"
    src.write_text("#include <stddef.h>\n#include <stdio.h>\n#include \"occam.h\"\nint main(void) {\n" + "\n".join(lines) + "\nreturn 0; }\n")
    include = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    subprocess.run(["gcc", "-I", include, str(src), "-o", str(tmp_path / "s")], check=True)
    got = [int(x) for x in subprocess.run([str(tmp_path / "s")], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [ctypes.sizeof(t) for t in names.values()] + [getattr(t, f).offset for _, t, f in fields]
    assert P._PROMPT_ARGS.size == got[0]


def prompt(**kw):
    import paper_2605_29657_gb300._prompt as P
    f = dict(dtype=0, heads=4, kv_heads=2, dim=64, causal=1, n=1, rows=3, keys=5, q=PTR, k=PTR + FAR, v=PTR + 2 * FAR, q_row=256,
             k_row=128, v_row=128, row_off=PTR, key_off=PTR, scale=0.0)
    f.update(kw)
    return P._PROMPT_ARGS.pack(*[0 if x is None else x for x in f.values()])


def grads(**kw):
    import paper_2605_29657_gb300._lib as L
    f = dict(out=PTR + 3 * FAR, lse=PTR + 4 * FAR, dout=PTR + 5 * FAR, dq=PTR + 6 * FAR, dk=PTR + 7 * FAR, dv=PTR + 8 * FAR, dout_row=256,
             dq_row=256, dk_row=128, dv_row=128)
    f.update(kw)
    return L.CPromptGrads(**f)


def prompt_size(lib, *a):
    n = ctypes.c_size_t(0)
    return lib.occam_prompt_workspace_size(*a, ctypes.byref(n)), n.value


def test_prompt_workspace_size(lib):
    invalid = codes()[0]
    rc, n = prompt_size(lib, 1000, 1000, 8, 2)
    assert rc == 0 and n > 0 and n % 256 == 0
    assert prompt_size(lib, 0, 0, 1, 1)[0] == 0
    assert prompt_size(lib, 100000, 1000, 8, 2)[1] > n and prompt_size(lib, 1000, 1000, 16, 2)[1] > n
    assert prompt_size(lib, 1000, 100000, 8, 2)[1] >= n
    assert prompt_size(lib, (1 << 31) - 1024, (1 << 31) - 1024, 1, 1)[0] == 0
    for bad in ((-1, 1, 1, 1), (1, -1, 1, 1), ((1 << 31) - 1023, 1, 1, 1), (1 << 31, 1, 1, 1), (1, 1 << 31, 1, 1), (1, 1, 0, 1), (1, 1, 1025, 1), (1, 1, 2, 0),
                (1, 1, 2, 3)):
        assert prompt_size(lib, *bad)[0] == invalid, bad
    assert lib.occam_prompt_workspace_size(1, 1, 1, 1, None) == invalid


@pytest.mark.parametrize("change,kind", [
    (dict(dtype=2), 1), (dict(dtype=-1), 1), (dict(dim=0), 1), (dict(dim=4), 1), (dict(dim=68), 1), (dict(dim=136), 1),
    (dict(heads=0), 0), (dict(heads=3), 0), (dict(heads=1026), 0), (dict(kv_heads=0), 0), (dict(kv_heads=8), 0), (dict(n=-1), 0),
    (dict(n=(1 << 20) + 1), 0), (dict(rows=-1), 0), (dict(rows=(1 << 31) - 1023), 0), (dict(keys=-1), 0), (dict(keys=(1 << 31) - 1023), 0),
    (dict(scale=-1.0), 0), (dict(scale=float("inf")), 0), (dict(scale=float("nan")), 0), (dict(row_off=None), 0),
    (dict(key_off=None), 0), (dict(q=None), 0), (dict(k=None), 0), (dict(v=None), 0), (dict(q=PTR + 8), 0), (dict(k=PTR + 2), 0),
    (dict(v=PTR + 4), 0), (dict(q_row=252), 0), (dict(q_row=248), 0), (dict(k_row=120), 0), (dict(v_row=132), 0),
    (dict(k_row=1 << 38), 0)])
def test_prompt_refusals(lib, change, kind):
    assert lib.occam_prompt_attend(prompt(**change), PTR + 3 * FAR, PTR + 4 * FAR, WS, BIG, None) == codes()[kind]
    assert lib.occam_prompt_attend_grad(prompt(**change), ctypes.byref(grads()), WS, BIG, None) == codes()[kind]


def test_prompt_other_refusals(lib):
    invalid, _, workspace = codes()
    a, out, lse = prompt(), PTR + 3 * FAR, PTR + 4 * FAR
    need = prompt_size(lib, 3, 5, 4, 2)[1]
    for ws, n in ((None, BIG), (WS + 128, BIG), (WS, need - 1)):
        assert lib.occam_prompt_attend(a, out, lse, ws, n, None) == workspace
        assert lib.occam_prompt_attend_grad(a, ctypes.byref(grads()), ws, n, None) == workspace
    assert lib.occam_prompt_attend(None, out, lse, WS, BIG, None) == invalid
    assert lib.occam_prompt_attend_grad(None, ctypes.byref(grads()), WS, BIG, None) == invalid
    assert lib.occam_prompt_attend_grad(a, None, WS, BIG, None) == invalid
    # results: missing, misaligned, over an input (3 rows of 4 heads of 64 dims in bf16 are 1536 bytes), out and lse over each other
    for o, l in ((None, lse), (out + 8, lse), (PTR, lse), (PTR + 1520, lse), (PTR + FAR - 1520, lse), (PTR + 2 * FAR, lse), (out, PTR),
                 (out, PTR + FAR + 16), (out, out), (out, out + 1532)):
        assert lib.occam_prompt_attend(a, o, l, WS, BIG, None) == invalid, (o, l)
    for bad in (dict(out=None), dict(lse=None), dict(dout=None), dict(dq=None), dict(dk=None), dict(dv=None), dict(out=PTR + 8),
                dict(dout=PTR + 8), dict(dq=out + FAR * 3 + 8), dict(dout_row=248), dict(dq_row=260), dict(dk_row=120), dict(dv_row=1 << 38),
                dict(dq=PTR), dict(dk=PTR + FAR), dict(dv=PTR + 2 * FAR), dict(dv=PTR), dict(dq=PTR + 3 * FAR), dict(dk=PTR + 4 * FAR),
                dict(dv=PTR + 5 * FAR), dict(dk=PTR + 6 * FAR), dict(dv=PTR + 7 * FAR + 16)):
        assert lib.occam_prompt_attend_grad(a, ctypes.byref(grads(**bad)), WS, BIG, None) == invalid, bad


def test_prompt_calls_with_nothing_to_do(lib):
    none = dict(q=None, k=None, v=None, row_off=None, key_off=None)
    for a in (prompt(n=0, **none), prompt(rows=0, keys=0, **none)):
        assert lib.occam_prompt_attend(a, None, None, WS, BIG, None) == 0
        assert lib.occam_prompt_attend_grad(a, ctypes.byref(grads(out=None, lse=None, dout=None, dq=None, dk=None, dv=None)), WS, BIG, None) == 0
    assert lib.occam_prompt_attend(prompt(rows=0, q=None), None, None, WS, BIG, None) == 0
    assert lib.occam_last_call_kernels() == 0


def enter(lib, c=None, ws=WS, wn=BIG, q=None, **kw):
    import paper_2605_29657_gb300._lib as L
    f = dict(layer=0, dtype=0, n=1, rot=64, pairing=0, axes=3, total_rows=2, k=PTR, k_row=128, v=PTR, v_row=128, seqs=PTR, row_off=PTR,
             positions=PTR, pos_stride=2, inv_freq=PTR, axis=PTR)
    f.update(kw)
    t = dict(src=PTR + FAR, dst=PTR + 2 * FAR, heads=4, src_row=256, src_head=64, dst_row=256, dst_head=64)
    a = L.CAppendRopeArgs(**f, q=None if q is None else bytes(L.CRopeTensor(**dict(t, **q))))
    return lib.occam_cache_append_rope(ctypes.byref(c or cache()), ctypes.byref(a), ws, wn, None)


def test_append_rope_refusals(lib):
    invalid, unsupported, workspace = codes()
    c = cache()
    for bad in (dict(dtype=2), dict(dtype=-1)):
        assert enter(lib, **bad) == unsupported
    for bad in (dict(layer=2), dict(layer=-1), dict(total_rows=-1), dict(total_rows=1 << 31), dict(n=-1), dict(n=5), dict(rot=0), dict(rot=3),
                dict(rot=66), dict(axes=0), dict(axes=9), dict(pos_stride=-1), dict(pairing=2), dict(positions=None), dict(inv_freq=None),
                dict(axis=None), dict(k=None), dict(v=None), dict(seqs=None), dict(row_off=None), dict(k=PTR + 8), dict(v=PTR + 2),
                dict(k_row=120), dict(v_row=132)):
        assert enter(lib, **bad) == invalid, bad
    for bad in (dict(src=None), dict(dst=None), dict(heads=0), dict(heads=65536), dict(src_row=-1), dict(dst_head=-64), dict(src=PTR + 1),
                dict(dst=PTR + 1), dict(dst_row=32), dict(dst_head=32), dict(dst=PTR), dict(dst=PTR + FAR + 128), dict(dst_row=128),
                dict(dst=PTR + FAR, dst_row=512)):
        assert enter(lib, q=bad) == invalid, bad
    for ws, wn in ((None, BIG), (WS + 128, BIG), (WS, size(lib, c)[1] - 1)):
        assert enter(lib, ws=ws, wn=wn) == workspace
    for change in (dict(layers=0), dict(dim=96), dict(k=None), dict(max_seqs=0), dict(page_tokens=48)):
        want = unsupported if "dim" in change or "page_tokens" in change else invalid
        assert enter(lib, cache(**change)) == want
    assert lib.occam_cache_append_rope(None, None, WS, BIG, None) == invalid
    assert lib.occam_cache_append_rope(ctypes.byref(c), None, WS, BIG, None) == invalid
    assert enter(lib, total_rows=0, k=None, v=None, positions=None, seqs=None, row_off=None) == 0
    assert enter(lib, n=0, k=None, v=None, seqs=None, row_off=None) == 0


def shared_size(lib, c, rows, heads):
    n = ctypes.c_size_t(0)
    return lib.occam_cache_shared_workspace_size(ctypes.byref(c), rows, heads, ctypes.byref(n)), n.value


def test_attend_shared_refusals(lib):
    invalid, unsupported, workspace = codes()
    c = cache()
    ref = ctypes.byref(c)
    call = lambda a=None, off=PTR, groups=1, most=2, ws=WS, wn=BIG: \
        lib.occam_cache_attend_shared(ref, a or attend(), off, groups, most, ws, wn, None)
    rc, need = shared_size(lib, c, 2, 4)
    assert rc == 0 and need > size(lib, c)[1] + 2 * 4 * 65 * 4 and need % 256 == 0
    for bad in ((-1, 4), (1 << 31, 4), (1, 0), (1, 129)):
        assert shared_size(lib, c, *bad)[0] == invalid
    assert shared_size(lib, cache(dim=96), 1, 4)[0] == unsupported
    for ws, wn in ((None, BIG), (WS + 128, BIG), (WS, need - 1), (WS, size(lib, c)[1] - 1)):
        assert call(ws=ws, wn=wn) == workspace
    assert call(attend(keep=PTR, keep_off=PTR)) == unsupported
    for bad in (dict(layer=2), dict(heads=3), dict(heads=0), dict(rows=-1), dict(n=5), dict(max_rows=-1), dict(q=PTR + 8), dict(out=None),
                dict(q_row=255), dict(seqs=None), dict(row_off=None), dict(scale=float("nan"))):
        assert call(attend(**bad)) == invalid, bad
    assert call(attend(dtype=2)) == unsupported
    for bad in (dict(off=None), dict(groups=-1), dict(groups=0), dict(groups=5), dict(most=-1)):
        assert call(**bad) == invalid, bad
    assert lib.occam_cache_attend_shared(ref, None, PTR, 1, 2, WS, BIG, None) == invalid
    assert lib.occam_cache_attend_shared(None, attend(), PTR, 1, 2, WS, BIG, None) == invalid
    assert call(attend(rows=0, n=0, q=None, out=None), off=None, groups=0, most=0) == 0
    assert lib.occam_last_call_kernels() == 0
