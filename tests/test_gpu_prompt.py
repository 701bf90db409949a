"""Attention of packed prompts against its definition in 64 bits, within bounds derived from the data
(prompt_reference)."""

from __future__ import annotations

import math

import pytest
import torch

import prompt_reference as P

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f16": torch.float16}


def offs(rows, at=0):
    out = [at]
    for r in rows:
        out.append(out[-1] + r)
    return out


def dev(x, dt=torch.int64):
    return torch.tensor(x, dtype=dt, device="cuda")


def inputs(rows, keys, H, Hkv, D, dtype, seed=0, gain=1.5, fused=False, first=0, behind=0):
    """q, k, v with `first` rows before and `behind` rows after the sequences', NaN in those."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    r, m = sum(rows) + first + behind, sum(keys if keys is not None else rows) + first + behind

    def normal(n, h):
        x = torch.randn((n, h, D), generator=g, device="cuda") * gain
        x[:first] = math.nan
        if behind:
            x[-behind:] = math.nan
        return x.to(dtype)

    if fused:
        qkv = normal(r, H + 2 * Hkv)
        return qkv.split((H, Hkv, Hkv), 1)
    return normal(r, H), normal(m, Hkv), normal(m, Hkv)


def check(q, k, v, off, koff=None, scale=0.0, causal=True, where=""):
    import paper_2605_29657_gb300 as occ
    ws = occ.alloc_prompt_workspace(q.shape[0], q.shape[1], k.shape[0], k.shape[1])
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    occ.occam_prompt_attend(q, k, v, dev(off), ws, key_off=None if koff is None else dev(koff), scale=scale, causal=causal, out=out,
                            lse=lse)
    assert occ.occam_get_status(ws) == 0
    want, wlse, tol, ltol = P.attend(q, k, v, off, koff, scale, causal)
    for x in (out, lse):  # rows of no sequence are left as they were
        assert bool((x[:off[0]] == 7.0).all()) and bool((x[off[-1]:] == 7.0).all())
    a = slice(off[0], off[-1])
    P.assert_near(out[a], want[a], tol[a], q.dtype, where + " out")
    P.assert_near(lse[a], wlse[a], ltol[a], torch.float32, where + " lse")
    return out, lse


# rows of each sequence, heads, key heads, dims
CASES = [
    ([1], 4, 1, 64), ([37], 32, 8, 128), ([128], 2, 2, 128), ([129, 127], 3, 1, 64), ([256, 1, 0, 300, 5], 8, 2, 128),
    ([0, 0, 3], 7, 1, 80), ([580], 4, 4, 72), ([64, 65, 63, 200], 16, 1, 64), ([391, 130], 6, 1, 128), ([33, 700], 12, 2, 8),
    ([5, 1100], 5, 5, 40), ([513], 4, 2, 96), ([90, 2, 260], 64, 1, 64), ([70, 140], 128, 1, 16), ([1030], 28, 4, 104),
    ([257, 255], 10, 2, 120),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n", range(len(CASES)))
def test_prompt(n, dtype):
    rows, H, Hkv, D = CASES[n]
    q, k, v = inputs(rows, None, H, Hkv, D, DT[dtype], n, fused=n % 2 == 0, first=n % 3, behind=(n + 1) % 3)
    off = offs(rows, n % 3)
    check(q, k, v, off, where="causal")
    check(q, k, v, off, scale=0.3, causal=False, where="full")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rows,keys", [([1, 7, 130], [200, 7, 1000]), ([40, 300, 3], [5, 130, 0]), ([0, 2], [9, 0]), ([260], [1]),
                                       ([17], [129]), ([300, 2], [299, 64])])
def test_prompt_with_other_keys(rows, keys, dtype):
    """Chunks of longer prompts; fewer keys than rows leave rows that see nothing."""
    for D, H, Hkv in ((128, 8, 2), (64, 3, 3)):
        q, k, v = inputs(rows, keys, H, Hkv, D, DT[dtype], 5)
        out, lse = check(q, k, v, offs(rows), offs(keys), where="causal")
        check(q, k, v, offs(rows), offs(keys), causal=False, where="full")
        if rows == [40, 300, 3]:
            assert bool((out[:35] == 0).all()) and bool((lse[:35] == -math.inf).all()) and bool((out[-3:] == 0).all())


def test_prompt_without_keys():
    q, k, v = inputs([5, 200], [0, 0], 4, 2, 64, torch.bfloat16)
    out, lse = check(q, k, v, [0, 5, 205], [0, 0, 0])
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())


@pytest.mark.parametrize("causal", [True, False])
def test_prompt_long(causal):
    q, k, v = inputs([2900, 1], None, 4, 1, 128, torch.bfloat16, 3, fused=True)
    check(q, k, v, [0, 2900, 2901], causal=causal)
    q, k, v = inputs([3500], None, 2, 2, 64, torch.float16, 4)
    check(q, k, v, [0, 3500], causal=causal)


def test_prompt_many_sequences():
    """More sequences than are listed one by one, some of them empty."""
    rows = [(7 * i) % 23 if i % 5 else 0 for i in range(700)]
    q, k, v = inputs(rows, None, 4, 2, 64, torch.bfloat16, 1, first=2)
    check(q, k, v, offs(rows, 2))
    rows = [3] * 5000
    q, k, v = inputs(rows, None, 1, 1, 8, torch.float16, 2)
    check(q, k, v, offs(rows))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("gain", [0.01, 6.0])
def test_prompt_flat_and_peaked(gain, dtype):
    q, k, v = inputs([300, 77], None, 4, 2, 128, DT[dtype], 9, gain=gain)
    check(q, k, v, [0, 300, 377])
    # scores that climb along the keys, so that references move many times
    k = (torch.linspace(0, 4, 377, device="cuda")[:, None, None] * torch.ones_like(k.float())).to(DT[dtype])
    check(q.abs(), k, v, [0, 300, 377])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("H,Hkv,D", [(4, 1, 128), (2, 2, 64), (3, 3, 72)])
def test_prompt_values_that_are_not_finite(H, Hkv, D, dtype):
    """A value counts for the rows that see it; other sequences and earlier rows never meet it."""
    rows = [200, 150, 90]
    q, k, v = (x.clone() for x in inputs(rows, None, H, Hkv, D, DT[dtype], 11))
    v[60, 0, 3], v[70, 0, 3], v[130, 0, 5] = math.inf, -math.inf, math.nan
    v[199, 0, D - 1], v[199, 0, 0] = -math.inf, math.inf
    v[200, 0, 7] = math.nan
    v[350:] = math.nan  # the last sequence's
    check(q, k, v, offs(rows), where="values")
    k[140] = math.nan  # a key: its score counts for the rows that see it
    k[210] = math.inf
    q[5] = math.nan
    q[100], q[101, 0, 0] = 0.0, math.inf
    q[200:350] = 0.0
    import paper_2605_29657_gb300 as occ
    out, lse = occ.occam_prompt_attend(q, k, v, dev(offs(rows)), occ.alloc_prompt_workspace(440, H))
    want, wl, _, _ = P.attend(q, k, v, offs(rows))
    fine = torch.isfinite(wl)  # rows without a score that is not finite
    assert torch.equal(torch.isfinite(lse), fine) and torch.equal(torch.isnan(out[fine]), torch.isnan(want[fine]))


def test_prompt_rows_of_another_stride():
    """Rows far apart, odd offsets between q, k and v, more keys' rows than queries'."""
    big = torch.randn((500, 30, 64), device="cuda", generator=torch.Generator(device="cuda").manual_seed(2)).half()
    q, k, v = big[::3, 5:13], big[1:, 20:22][:333], big[:333, 2:4]
    check(q[:160], k, v, [0, 100, 160], [3, 103, 333])


def test_prompt_offsets_that_do_not_fit_are_recorded():
    import paper_2605_29657_gb300 as occ
    from paper_2605_29657_gb300 import _lib as L
    q, k, v = inputs([40, 40], None, 4, 2, 64, torch.bfloat16)
    ws = occ.alloc_prompt_workspace(80, 4)
    want, wl = occ.occam_prompt_attend(q, k, v, dev([0, 40, 80]), ws)
    for off, koff in (([0, 40, 81], None), ([-1, 40, 80], None), ([0, 40, 30], None), ([0, 40, 80], [0, 40, 1 << 40]),
                      ([0, 40, 80], [0, 40, 39])):
        out, lse = torch.zeros_like(q), torch.zeros_like(wl)
        occ.occam_prompt_attend(q, k, v, dev(off), ws, key_off=None if koff is None else dev(koff), out=out, lse=lse)
        assert occ.occam_get_status(ws) == L.OCCAM_ERR_INVALID_ARG
        if off[0] == 0:
            assert torch.equal(out[:40], want[:40]) and bool((out[40:] == 0).all())
    out, lse = occ.occam_prompt_attend(q, k, v, dev([0, 40, 80]), ws)
    assert occ.occam_get_status(ws) == 0 and torch.equal(out, want) and torch.equal(lse, wl)


def test_prompt_streams_and_graph():
    """Two calls at once with a workspace each, a captured call replayed on new values, results bit for bit the same."""
    import paper_2605_29657_gb300 as occ
    rows = [300, 20, 513]
    q, k, v = inputs(rows, None, 8, 2, 128, torch.bfloat16, 21)
    q2, k2, v2 = inputs(rows, None, 8, 2, 128, torch.bfloat16, 22)
    off = dev(offs(rows))
    ws = [occ.alloc_prompt_workspace(833, 8) for _ in range(2)]
    want = [occ.occam_prompt_attend(*x, off, ws[0]) for x in ((q, k, v), (q2, k2, v2))]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(5):
        for n, x in enumerate(((q, k, v), (q2, k2, v2))):
            got[n].append(occ.occam_prompt_attend(*x, off, ws[n], stream=streams[n]))
    torch.cuda.synchronize()
    for n in range(2):
        for o, l in got[n]:
            assert torch.equal(o, want[n][0]) and torch.equal(l, want[n][1])
    out, lse = torch.zeros_like(want[0][0]), torch.zeros_like(want[0][1])
    a = [x.contiguous() for x in (q, k, v)]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        occ.occam_prompt_attend(*a, off, ws[0], out=out, lse=lse)
        occ.occam_prompt_attend(*a, off, ws[0], out=out, lse=lse)
    for n, x in enumerate(((q, k, v), (q2, k2, v2))):
        for to, y in zip(a, x):
            to.copy_(y)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[n][0]) and torch.equal(lse, want[n][1])
    assert occ.occam_get_status(ws[0]) == 0


def test_prompt_refusals():
    import paper_2605_29657_gb300 as occ
    q, k, v = inputs([8], None, 4, 2, 64, torch.bfloat16)
    off, ws = dev([0, 8]), occ.alloc_prompt_workspace(8, 4)
    odd = torch.zeros((8, 4, 68), dtype=torch.bfloat16, device="cuda")
    for call in (
        lambda: occ.occam_prompt_attend(q.float(), k.float(), v.float(), off, ws),
        lambda: occ.occam_prompt_attend(q, k.half(), v, off, ws),
        lambda: occ.occam_prompt_attend(q, k, v[:7], off, ws),
        lambda: occ.occam_prompt_attend(q[:, :3], k, v, off, ws),
        lambda: occ.occam_prompt_attend(q, k, v, off.int(), ws),
        lambda: occ.occam_prompt_attend(q, k, v, off, ws, key_off=off[:1]),
        lambda: occ.occam_prompt_attend(q, k, v, off[:0], ws),
        lambda: occ.occam_prompt_attend(q, k, v, off, ws[:256]),
        lambda: occ.occam_prompt_attend(q, k, v, off, ws[8:]),
        lambda: occ.occam_prompt_attend(q, k, v, off, ws, scale=-1.0),
        lambda: occ.occam_prompt_attend(q, k, v, off, ws, scale=math.nan),
        lambda: occ.occam_prompt_attend(q, k, v, off, ws, out=q),
        lambda: occ.occam_prompt_attend(q, k, v, off, ws, out=q[:4]),
        lambda: occ.occam_prompt_attend(q, k, v, off, ws, lse=torch.zeros(8, device="cuda")),
        lambda: occ.occam_prompt_attend(odd, odd, odd, off, ws),
        lambda: occ.occam_prompt_attend(q.cpu(), k, v, off, ws),
        lambda: occ.occam_prompt_attend(q.transpose(0, 1), k, v, off, ws),
        lambda: occ.occam_prompt_attend(q, k, v, off, None),
    ):
        with pytest.raises(occ.OccamError):
            call()
    none = occ.occam_prompt_attend(q[:0], k[:0], v[:0], dev([0]), ws)
    assert none[0].shape == (0, 4, 64)


def test_prompt_values_near_the_end_of_bf16():
    """Sums before their division stay finite: results are means of the values."""
    q, k, v = (x.clone() for x in inputs([300, 40, 2], None, 4, 2, 128, torch.bfloat16, 12))
    v[:300] = v[:300].sign() * 3.3e38
    v[300:] = 3.3e38
    k[:300] = 0.0  # all weights the same
    q[300:340], k[300:340] = 1.0, (torch.arange(40, device="cuda")[:, None, None] / 80).bfloat16()  # scores that climb by 5.5
    check(q, k, v, [0, 300, 340, 342])
    check(q, k, v, [0, 300, 340, 342], causal=False)
    # and small ones are what they were
    check(q, k, torch.where(v > 0, 1e-30, -3e-31).bfloat16(), [0, 300, 340, 342])
