"""The gradient of a prompt's attention against its formulas in 64 bits, within bounds derived from
the data (prompt_reference.grad), and against differences."""

from __future__ import annotations

import math

import pytest
import torch

import prompt_reference as P
from test_gpu_prompt import CASES, DT, dev, inputs, offs

pytestmark = pytest.mark.gpu


def gradient_of(q, dtype, seed=0, spread=1.0):
    g = torch.Generator(device="cuda").manual_seed(1000 + seed)
    size = 0.02 * torch.exp(spread * torch.randn((q.shape[0], 1, 1), generator=g, device="cuda"))
    return (torch.randn(q.shape, generator=g, device="cuda") * size).to(dtype)


def check(q, k, v, dout, off, koff=None, scale=0.0, causal=True, where="", fused=False):
    """The three gradients, into tensors whose other rows keep what they hold (fused: views of one)."""
    import paper_2605_29657_gb300 as occ
    H, Hkv = q.shape[1], k.shape[1]
    ws = occ.alloc_prompt_workspace(q.shape[0], H, k.shape[0], Hkv)
    kw = dict(key_off=None if koff is None else dev(koff), scale=scale, causal=causal)
    out, lse = occ.occam_prompt_attend(q, k, v, dev(off), ws, **kw)
    if fused:
        whole = torch.full((q.shape[0], H + 2 * Hkv, q.shape[2]), 7.0, dtype=q.dtype, device="cuda")
        to = whole.split((H, Hkv, Hkv), 1)
    else:
        to = [torch.full(x.shape, 7.0, dtype=q.dtype, device="cuda") for x in (q, k, v)]
    got = occ.occam_prompt_attend_grad(q, k, v, out, lse, dout, dev(off), ws, dq=to[0], dk=to[1], dv=to[2], **kw)
    assert occ.occam_get_status(ws) == 0
    ko = off if koff is None else koff
    want = P.grad(q, k, v, dout, off, koff, scale, causal)
    for n, name in enumerate(("dq", "dk", "dv")):
        o = off if n == 0 else ko
        assert got[n].data_ptr() == to[n].data_ptr()
        assert bool((got[n][:o[0]] == 7.0).all()) and bool((got[n][o[-1]:] == 7.0).all())
        a = slice(o[0], o[-1])
        P.assert_near(got[n][a], want[n][a], want[3 + n][a], q.dtype, f"{where} {name}")
    return got


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n", range(len(CASES)))
def test_grad(n, dtype):
    rows, H, Hkv, D = CASES[n]
    fused = n % 2 == 0
    q, k, v = inputs(rows, None, H, Hkv, D, DT[dtype], n, fused=fused, first=n % 3, behind=(n + 1) % 3)
    dout = gradient_of(q, DT[dtype], n)
    if n % 3:
        dout[:n % 3] = math.nan  # rows of no sequence
    off = offs(rows, n % 3)
    check(q, k, v, dout, off, where="causal", fused=fused)
    check(q, k, v, dout, off, scale=0.3, causal=False, where="full")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rows,keys", [([1, 7, 130], [200, 7, 1000]), ([40, 300, 3], [5, 130, 0]), ([0, 2, 0, 0, 0, 70, 0], [9, 0, 200, 1, 300, 70, 4]),
                                       ([260], [1]), ([17], [129]), ([300, 2], [299, 64]), ([0, 0], [130, 500])])
def test_grad_with_other_keys(rows, keys, dtype):
    """Chunks of longer prompts, rows that see nothing, keys without rows (in a row: more than are known ahead)."""
    for D, H, Hkv in ((128, 8, 2), (64, 3, 3)):
        q, k, v = inputs(rows, keys, H, Hkv, D, DT[dtype], 5)
        dout = gradient_of(q, DT[dtype])
        for causal in (True, False):
            dq, dk, dv = check(q, k, v, dout, offs(rows), offs(keys), causal=causal, where=str(causal))
            if sum(rows) == 0:
                assert not dk.any() and not dv.any()


def test_grad_without_keys():
    q, k, v = inputs([5, 200], [0, 0], 4, 2, 64, torch.bfloat16)
    dq, _, _ = check(q, k, v, gradient_of(q, torch.bfloat16), [0, 5, 205], [0, 0, 0])
    assert not dq.any()


@pytest.mark.parametrize("causal", [True, False])
def test_grad_long(causal):
    q, k, v = inputs([2900, 1], None, 4, 1, 128, torch.bfloat16, 3, fused=True)
    check(q, k, v, gradient_of(q, torch.bfloat16), [0, 2900, 2901], causal=causal)
    q, k, v = inputs([3500], None, 2, 2, 64, torch.float16, 4)
    check(q, k, v, gradient_of(q, torch.float16), [0, 3500], causal=causal)


def test_grad_many_sequences():
    rows = [(7 * i) % 23 if i % 5 else 0 for i in range(700)]
    q, k, v = inputs(rows, None, 4, 2, 64, torch.bfloat16, 1, first=2)
    check(q, k, v, gradient_of(q, torch.bfloat16), offs(rows, 2))
    rows = [3, 1] * 600
    q, k, v = inputs(rows, None, 1, 1, 8, torch.float16, 2)
    check(q, k, v, gradient_of(q, torch.float16), offs(rows))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("gain,size,spread", [(0.01, 1.0, 1.0), (3.0, 1.0, 0.0), (1.5, 1e-4, 3.0), (1.5, 3000.0, 1.0)])
def test_grad_of_many_sizes(gain, size, spread, dtype):
    """Flat and peaked attention, tiny gradients (most of an f16 step's range) and large ones, rows of very different size."""
    q, k, v = inputs([300, 77], None, 4, 2, 128, DT[dtype], 9, gain=gain)
    dout = gradient_of(q, torch.float32, spread=spread) * size
    check(q, k, v, dout.clamp(-6e4, 6e4).to(DT[dtype]), [0, 300, 377])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_grad_against_differences(dtype):
    """Moving q, k or v by a small step changes sum(out * dout) as the gradient says, the attention itself in 64 bits."""
    rows = [70, 9, 130]
    q, k, v = inputs(rows, None, 4, 2, 64, DT[dtype], 31)
    dout = gradient_of(q, DT[dtype], 31)
    off = offs(rows)
    got = check(q, k, v, dout, off)
    tol = P.grad(q, k, v, dout, off)[3:]
    g = torch.Generator(device="cuda").manual_seed(5)

    def loss(q, k, v):
        total = 0.0
        for a, b in zip(off, off[1:]):
            for h in range(4):
                s = (q[a:b, h] @ k[a:b, h // 2].T / 8.0).masked_fill(torch.ones((b - a, b - a), dtype=torch.bool, device="cuda").triu(1), -math.inf)
                total = total + (torch.softmax(s, -1) @ v[a:b, h // 2] * dout[a:b, h].double()).sum()
        return total

    x = [y.double() for y in (q, k, v)]
    for n in range(3):
        d = torch.randn(x[n].shape, generator=g, device="cuda", dtype=torch.float64)
        hi, lo = ([y + s * d if i == n else y for i, y in enumerate(x)] for s in (1e-5, -1e-5))
        diff = (loss(*hi) - loss(*lo)) / 2e-5
        mine = got[n].double()
        # every gradient within its bound, so their sum along d within the sum of the bounds
        slack = ((tol[n] + P.UNIT[DT[dtype]] * mine.abs() * 1.01 + P.TINY[DT[dtype]]) * d.abs()).sum() + 1e-6 * (mine * d).abs().sum()
        assert abs(float(diff - (mine * d).sum())) <= float(slack)


def test_grad_repeats_and_other_sequences_do_not_matter():
    """Bit for bit the same every time, and a sequence's own whatever lies beside it, not finite included."""
    import paper_2605_29657_gb300 as occ
    for dtype in (torch.bfloat16, torch.float16):
        rows = [200, 333, 90]
        q, k, v = (x.clone() for x in inputs(rows, None, 8, 2, 128, dtype, 41))
        dout = gradient_of(q, dtype, 41)
        off, ws = dev(offs(rows)), occ.alloc_prompt_workspace(623, 8)
        out, lse = occ.occam_prompt_attend(q, k, v, off, ws)
        want = occ.occam_prompt_attend_grad(q, k, v, out, lse, dout, off, ws)
        for _ in range(3):
            assert all(torch.equal(x, y) for x, y in zip(occ.occam_prompt_attend_grad(q, k, v, out, lse, dout, off, ws), want))
        for t in (q, k, v, dout):
            t[200] = math.nan
            t[532] = math.inf
        got = occ.occam_prompt_attend_grad(q, k, v, *occ.occam_prompt_attend(q, k, v, off, ws), dout, off, ws)
        for x, y in zip(got, want):
            assert torch.equal(x[:200], y[:200]) and torch.equal(x[533:], y[533:])
        assert occ.occam_get_status(ws) == 0


def test_grad_offsets_that_do_not_fit_are_recorded():
    import paper_2605_29657_gb300 as occ
    from paper_2605_29657_gb300 import _lib as L
    q, k, v = inputs([40, 40], None, 4, 2, 64, torch.bfloat16)
    dout, off, ws = gradient_of(q, torch.bfloat16), dev([0, 40, 80]), occ.alloc_prompt_workspace(80, 4)
    out, lse = occ.occam_prompt_attend(q, k, v, off, ws)
    want = occ.occam_prompt_attend_grad(q, k, v, out, lse, dout, off, ws)
    for bad in ([0, 40, 81], [-1, 40, 80], [0, 40, 30]):
        to = [torch.zeros_like(x) for x in (q, k, v)]
        occ.occam_prompt_attend_grad(q, k, v, out, lse, dout, dev(bad), ws, dq=to[0], dk=to[1], dv=to[2])
        assert occ.occam_get_status(ws) == L.OCCAM_ERR_INVALID_ARG
        for x, y in zip(to, want):
            assert torch.equal(x[:40], y[:40]) if bad[0] == 0 else not x[:40].any()


def test_grad_streams_and_graph():
    """Steps at once with a workspace each; a captured step of forward and gradient replayed on new values while eager
    calls go on."""
    import paper_2605_29657_gb300 as occ
    rows = [300, 20, 513]
    sets = []
    for seed in (21, 22):
        q, k, v = inputs(rows, None, 8, 2, 64, torch.float16, seed)
        sets.append((q, k, v, gradient_of(q, torch.float16, seed)))
    off = dev(offs(rows))
    ws = [occ.alloc_prompt_workspace(833, 8) for _ in range(3)]

    def step(x, ws, stream=None, to=(None,) * 5):
        o, l = occ.occam_prompt_attend(*x[:3], off, ws, out=to[0], lse=to[1], stream=stream)
        return o, l, *occ.occam_prompt_attend_grad(*x[:3], o, l, x[3], off, ws, dq=to[2], dk=to[3], dv=to[4], stream=stream)

    want = [step(x, ws[0]) for x in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [step(sets[i % 2], ws[i % 2], streams[i % 2]) for i in range(6)]
    torch.cuda.synchronize()
    for i, r in enumerate(got):
        assert all(torch.equal(x, y) for x, y in zip(r, want[i % 2]))
    a = [x.clone() for x in sets[0]]
    to = [torch.zeros_like(x) for x in want[0]]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(a, ws[2], to=to)
    for n in (1, 0):
        for x, y in zip(a, sets[n]):
            x.copy_(y)
        g.replay()
        eager = step(sets[1 - n], ws[0])
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(to, want[n])) and all(torch.equal(x, y) for x, y in zip(eager, want[1 - n]))
    assert all(occ.occam_get_status(w) == 0 for w in ws)


def test_grad_refusals():
    import paper_2605_29657_gb300 as occ
    q, k, v = inputs([8], None, 4, 2, 64, torch.bfloat16)
    off, ws = dev([0, 8]), occ.alloc_prompt_workspace(8, 4)
    out, lse = occ.occam_prompt_attend(q, k, v, off, ws)
    dout = torch.ones_like(q)
    whole = torch.zeros((8, 8, 64), dtype=torch.bfloat16, device="cuda")

    def call(q=q, k=k, v=v, out=out, lse=lse, dout=dout, off=off, ws=ws, **kw):
        return occ.occam_prompt_attend_grad(q, k, v, out, lse, dout, off, ws, **kw)

    for bad in (
        dict(out=out[:4]), dict(out=out.float()), dict(lse=lse[:4]), dict(lse=lse.double()), dict(dout=dout.half()), dict(dout=dout[:4]),
        dict(dout=dout[:, :2]), dict(ws=ws[:512]), dict(off=off.int()), dict(dq=q), dict(dk=v), dict(dv=out[:, :2]), dict(dq=dout),
        dict(dk=whole[:, :2], dv=whole[:, 1:3]), dict(dq=whole[:, :4], dk=whole[:, 3:5]), dict(dq=torch.zeros((8, 4, 128), device="cuda").bfloat16()[..., ::2]),
        dict(dk=torch.zeros((7, 2, 64), device="cuda").bfloat16()), dict(scale=math.inf), dict(dout=dout.cpu()),
    ):
        with pytest.raises(occ.OccamError):
            call(**bad)
    call(dq=whole[:, :4], dk=whole[:, 4:6], dv=whole[:, 6:])


# rows, keys (None: the same), heads, key heads, dims
ONE_KEY = [
    ([1], None, 8, 1, 128), ([1], None, 3, 3, 64), ([1] * 70, None, 32, 8, 128), ([300, 1, 2], None, 5, 1, 72), ([5, 300, 70], [1, 1, 3], 8, 2, 128),
    ([200, 129], [70, 129], 128, 1, 16), ([1000], None, 8, 1, 64),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n", range(len(ONE_KEY)))
def test_grad_of_rows_that_see_one_key(n, dtype):
    """Their softmax is 1 whatever q and k are: dq is 0, and dk does not depend on them. Exactly."""
    import paper_2605_29657_gb300 as occ
    rows, keys, H, Hkv, D = ONE_KEY[n]
    q, k, v = inputs(rows, keys, H, Hkv, D, DT[dtype], n)
    dout = gradient_of(q, DT[dtype], n)
    keys = rows if keys is None else keys
    off, koff, ws = offs(rows), offs(keys), occ.alloc_prompt_workspace(sum(rows), H, sum(keys), Hkv)
    for causal in (True, False):
        check(q, k, v, dout, off, koff, causal=causal, where=str(causal))
        sees = [max(m - r + j + 1, 0) if causal else m for r, m in zip(rows, keys) for j in range(r)]
        one = torch.tensor([s == 1 for s in sees], device="cuda")
        most = [max([min(sees[a + j], m) for j in range(r)]) for a, r, m in zip(off, rows, keys)]
        kw = dict(key_off=dev(koff), causal=causal)
        got = []
        for x in (q, torch.where(one[:, None, None], -0.5 * q, q)):
            out, lse = occ.occam_prompt_attend(x, k, v, dev(off), ws, **kw)
            got.append(occ.occam_prompt_attend_grad(x, k, v, out, lse, dout, dev(off), ws, **kw))
        for dq, dk, _ in got:
            assert not dq[one].any()
            for i, s in enumerate(most):
                assert s > 1 or not dk[koff[i]:koff[i + 1]].any()
        assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    assert occ.occam_get_status(ws) == 0


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("H,Hkv,D", [(4, 2, 64), (3, 3, 128), (8, 1, 72)])
def test_grad_of_many_items_of_one_step(H, Hkv, D, dtype):
    """Each of the two issuing warps passes by every second item: no wait runs out, and results repeat."""
    import paper_2605_29657_gb300 as occ
    rows = [1 + (5 * i) % 8 for i in range(3000)]
    q, k, v = inputs(rows, None, H, Hkv, D, DT[dtype], 6)
    dout, off, ws = gradient_of(q, DT[dtype]), dev(offs(rows)), occ.alloc_prompt_workspace(sum(rows), H, sum(rows), Hkv)
    out, lse = occ.occam_prompt_attend(q, k, v, off, ws)
    want = occ.occam_prompt_attend_grad(q, k, v, out, lse, dout, off, ws)
    for _ in range(30):
        got = occ.occam_prompt_attend_grad(q, k, v, out, lse, dout, off, ws)
        assert all(torch.equal(x, y) for x, y in zip(got, want))
    assert occ.occam_get_status(ws) == 0
    first = offs(rows[:100])
    for x, y, tol in zip(want, *(lambda r: (r[:3], r[3:]))(P.grad(*(t[:first[-1]] for t in (q, k, v, dout)), first))):
        P.assert_near(x[:first[-1]], y, tol, DT[dtype])
