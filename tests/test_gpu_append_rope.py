"""occam_cache_append_rope against its definition in 64 bits: values and page state as
occam_cache_append, queries as occam_rope, keys within what fp32 turning may move a value before its one
rounding to a code.

Bound of a turned value before that rounding: 2^-21 (|a| + |b|), as for occam_rope. A code
is the nearest to the fp32 value, so its distance from the exact value is at most the
nearest code's plus twice the bound."""

from __future__ import annotations

import math

import pytest
import torch

import cache_reference as R
from test_gpu_cache import dev, make, offs
from test_gpu_rope import close as close_finite

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f16": torch.float16}
I64 = torch.int64


def case(rows, hq, hk, dim, rot, axes, dtype, seed=0, gain=1.0, max_pos=4000):
    g = torch.Generator().manual_seed(seed)
    qkv = (gain * torch.randn((rows, hq + 2 * hk, dim), generator=g) * torch.exp(torch.randn((rows, 1, 1), generator=g))).to(DT[dtype]).cuda()
    pos = torch.randint(0, max_pos, (axes, rows), generator=g, dtype=torch.int32).cuda()
    freq = (10000.0 ** (-torch.arange(rot // 2).double() * 2 / rot)).float().cuda()
    axis = torch.randint(0, axes, (rot // 2,), generator=g, dtype=torch.int32).cuda()
    return *qkv.split((hq, hk, hk), 1), pos, freq, axis


def close(got, x, pos, freq, axis, pairing, inverse):
    """As for occam_rope. A value of half a step past the type's largest or more (f16: 65520) rounds to infinity, and what is
    not finite in x stays so by the formula."""
    want, mag = R.rope(x, pos, freq, axis, pairing, inverse)
    g = got.double().cpu()
    u, top = R.UNIT[got.dtype], torch.finfo(got.dtype).max
    end = top * (1 + u / 2) if got.dtype == torch.bfloat16 else 65520.0  # where rounding to infinity begins
    slack = (1 + u) * 2.0 ** -21 * mag
    assert torch.equal(torch.isnan(g), torch.isnan(want))
    out = torch.isinf(g)
    assert bool((want.abs()[out] >= end - slack.nan_to_num()[out]).all()) and torch.equal(g[out].sign(), want[out].sign())
    fine = ~out & ~torch.isnan(want)
    err, bound = (g - want).abs(), u * want.abs() + R.TINY[got.dtype] + slack
    assert bool((err <= bound)[fine].all())


def assert_turned(c, ref, layer, mag, seqs, off):
    """The state after an append, `ref` being the reference's with exactly turned keys. mag: of each new key's pair."""
    assert torch.equal(c.table.cpu(), ref.table) and c.length.cpu().tolist() == ref.length and c.refs.cpu().tolist() == ref.refs
    for got, want in ((c.v, ref.v), (c.v_scale, ref.vs), (c.k_scale, ref.ks)):
        torch.testing.assert_close(got.cpu().double(), want, rtol=0, atol=0, equal_nan=True)
    got, want = c.k.cpu().double(), ref.k
    bound = torch.zeros_like(want)
    for i, s in enumerate(seqs):
        for r in range(off[i], off[i + 1]):
            p = ref.length[s] - (off[i + 1] - r)
            page = int(ref.table[s, p // c.page_tokens])
            bound[layer, page, :, p % c.page_tokens] = mag[r] / ref.ks[layer, page][:, None]
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    assert bool((same | (bound > 0)).all())
    # where the codes differ, both are about as near: neighbours around the exact value
    x = ref.exact[layer] if hasattr(ref, "exact") else want
    near = (got - x).abs() <= (want - x).abs() + 2.0 ** -20 * bound
    assert bool((same | near).all())
    assert float((~same).double().mean()) < 1e-3


def append(c, ref, layer, q, k, v, pos, freq, axis, pairing, seqs, counts, first=0, behind=0):
    """The call, and the reference's append of exactly turned keys; returns (turned queries, mag of the keys)."""
    import paper_2605_29657_gb300 as occ
    off = offs(counts)
    off = [first + x for x in off]
    occ.occam_cache_extend(c, dev(seqs), dev(counts))
    out = occ.occam_cache_append_rope(c, layer, q, k, v, dev(seqs), dev(off, I64), pos, freq, axis, pairing=pairing)
    ref.extend(seqs, counts)
    turned, mag = R.rope(k, pos, freq, axis, pairing, False)
    ref.append(layer, turned, v, seqs, off)
    # the exact values in units of their blocks' scales
    ref.exact = ref.k.clone()
    for i, s in enumerate(seqs):
        for r in range(off[i], off[i + 1]):
            p = ref.length[s] - (off[i + 1] - r)
            page = int(ref.table[s, p // c.page_tokens])
            ref.exact[layer, page, :, p % c.page_tokens] = turned[r] / ref.ks[layer, page][:, None]
    assert c.status() == 0
    assert_turned(c, ref, layer, mag, seqs, off)
    ref.k = c.k.cpu().double()  # (codes that went the other way are what the next call finds)
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("pairing", ["half", "adjacent"])
@pytest.mark.parametrize("T,dim,heads,hq,rot", [(16, 64, 2, 2, 64), (32, 128, 1, 4, 128), (64, 128, 3, 6, 64), (128, 64, 2, 8, 24),
                                                (128, 128, 1, 1, 128), (16, 128, 5, 5, 10), (64, 64, 9, 9, 2)])
def test_append_rope(T, dim, heads, hq, rot, pairing, dtype):
    c = make(heads=heads, dim=dim, T=T, max_pages=9)
    ref = R.Cache(c)
    # fresh pages, then single tokens and ragged runs into half-filled ones; later tokens larger, so scales grow
    for n, (seqs, counts, gain) in enumerate([
            ([4, 1, 2], [T + 1, 3, 2 * T], 1.0), ([1, 4], [1, 1], 30.0), ([2, 0, 1], [0, 5, T], 1e-3), ([4, 1, 0, 2], [1, 2 * T - 1, 1, 1], 1e3)]):
        q, k, v, pos, freq, axis = case(sum(counts), hq, heads, dim, rot, 3, dtype, n, gain)
        out = append(c, ref, n % 2, q, k, v, pos, freq, axis, pairing, seqs, counts)
        close(out, q, pos, freq, axis, pairing, False)
        if gain <= 1.0:
            close_finite(out, q, pos, freq, axis, pairing, False)
        assert out.is_contiguous()


def test_append_rope_is_rope_and_append_but_for_one_rounding():
    """Values, scales and queries bit for bit those of the two calls; keys within their rounding to 16 bits."""
    import paper_2605_29657_gb300 as occ
    a, b = make(heads=4, dim=128, T=64, stale=False), make(heads=4, dim=128, T=64, stale=False)
    q, k, v, pos, freq, axis = case(150, 8, 4, 128, 128, 3, "f16", 3, max_pos=1 << 20)
    seqs, off = dev([2, 0]), dev([0, 100, 150], I64)
    for c in (a, b):
        occ.occam_cache_extend(c, seqs, dev([100, 50]))
    tq, tk = occ.occam_rope(q, k, pos, freq, axis)
    occ.occam_cache_append(a, 1, tk, v, seqs, off)
    out = occ.occam_cache_append_rope(b, 1, q, k, v, seqs, off, pos, freq, axis)
    assert torch.equal(out, tq) and torch.equal(a.v.view(torch.uint8), b.v.view(torch.uint8))
    assert torch.equal(a.v_scale, b.v_scale) and torch.equal(a.k_scale, b.k_scale)
    x, y = (c.k.double() * c.k_scale.double()[..., None, None] for c in (a, b))
    assert bool(((x - y).abs() <= 2.0 ** -3 * x.abs() + 2.0 ** -9 * a.k_scale.double()[..., None, None]).all())
    # in place, and repeating the call changes nothing
    codes = b.k.view(torch.uint8).clone()
    q2 = q.contiguous().clone()
    got = occ.occam_cache_append_rope(b, 1, q2, k, v, seqs, off, pos, freq, axis, out_q=q2)
    assert got.data_ptr() == q2.data_ptr() and torch.equal(q2, tq) and torch.equal(codes, b.k.view(torch.uint8))
    # in place inside the projection that keys and values are views of
    whole = torch.cat((q, k, v), 1)
    wq, wk, wv = whole.split((8, 4, 4), 1)
    occ.occam_cache_append_rope(b, 1, wq, wk, wv, seqs, off, pos, freq, axis, out_q=wq)
    assert torch.equal(whole[:, :8], tq) and torch.equal(whole[:, 8:], torch.cat((k, v), 1))
    assert torch.equal(codes, b.k.view(torch.uint8)) and b.status() == 0
    # without queries
    assert occ.occam_cache_append_rope(b, 1, None, k, v, seqs, off, pos, freq, axis) is None
    assert torch.equal(codes, b.k.view(torch.uint8))


def test_append_rope_special_values():
    c = make(layers=1, T=16, dim=64, heads=2)
    ref = R.Cache(c)
    q, k, v, pos, freq, axis = case(21, 2, 2, 64, 32, 2, "bf16", 5)
    k, v = k.clone(), v.clone()
    k[0, 0], k[3, 0, 40] = 0.0, math.inf         # (past the turned dims: an infinity stays one)
    k[4, 0, 41], v[5, 1, 6] = math.nan, 3.3e38
    v[6, 0, 3], v[7, 0, 3] = -math.inf, math.nan
    k[16:, 1] = 0.0
    append(c, ref, 0, q, k, v, pos, freq, axis, "half", [3], [21])


def test_append_rope_many_sequences_and_rows_outside():
    import paper_2605_29657_gb300 as occ
    n = 150
    c = make(layers=1, pages=400, heads=2, dim=64, T=16, seqs=n, max_pages=3)
    ref = R.Cache(c)
    g = torch.Generator().manual_seed(3)
    seqs = torch.randperm(n, generator=g).tolist()
    counts = torch.randint(0, 40, (n,), generator=g).tolist()
    q, k, v, pos, freq, axis = case(sum(counts) + 12, 2, 2, 64, 64, 1, "f16", 8)
    out = append(c, ref, 0, q, k, v, pos, freq, axis, "half", seqs, counts, first=7)
    close(out, q, pos, freq, axis, "half", False)  # every row, those of no sequence too
    # nothing to append: the queries alone
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    assert torch.equal(occ.occam_cache_append_rope(c, 0, q, k, v, none, dev([0], I64), pos, freq, axis), out)


def test_append_rope_many_heads_share_a_page():
    """Heads enough that CTAs take several."""
    n = 40
    c = make(layers=1, pages=n * 3 + 4, heads=32, dim=128, T=64, seqs=n, max_pages=3)
    ref = R.Cache(c)
    counts = [64 + 3 * i % 50 for i in range(n)]
    q, k, v, pos, freq, axis = case(sum(counts), 32, 32, 128, 128, 3, "bf16", 2)
    out = append(c, ref, 0, q, k, v, pos, freq, axis, "adjacent", list(range(n)), counts)
    close(out, q, pos, freq, axis, "adjacent", False)


def test_append_rope_errors_change_nothing():
    import paper_2605_29657_gb300 as occ
    c = make(layers=1, pages=12, heads=1, dim=64, T=16, seqs=4, max_pages=4)
    ref = R.Cache(c)
    q, k, v, pos, freq, axis = case(20, 1, 1, 64, 64, 1, "bf16")
    append(c, ref, 0, q, k, v, pos, freq, axis, "half", [0], [20])
    want, _ = occ.occam_rope(q, None, pos, freq, axis)
    for seqs, off in (([0], [0, 4]), ([9], [0, 20]), ([-1], [0, 20]), ([0], [0, 21]), ([0], [-1, 5]), ([1], [0, 1])):
        out = occ.occam_cache_append_rope(c, 0, q[:3] if off == [0, 4] else q, k[:3] if off == [0, 4] else k, v[:3] if off == [0, 4] else v,
                                          dev(seqs), dev(off, I64), pos[:, :3].contiguous() if off == [0, 4] else pos, freq, axis)
        assert c.status() == 1, (seqs, off)
        R.assert_codes(c, ref)
        assert torch.equal(out, want[:out.shape[0]])  # the queries are turned all the same
    # a shared page, and behind a refused extend
    occ.occam_cache_fork(c, dev([0]), dev([1]))
    ref.fork([0], [1])
    occ.occam_cache_append_rope(c, 0, q, k, v, dev([0]), dev([0, 20], I64), pos, freq, axis)
    assert c.status() == 1
    R.assert_codes(c, ref)
    occ.occam_cache_extend(c, dev([2]), dev([1000]))
    occ.occam_cache_append_rope(c, 0, q[:4], k[:4], v[:4], dev([1]), dev([0, 4], I64), pos[:, :4].contiguous(), freq, axis)
    assert c.status() == 2
    R.assert_codes(c, ref)


def test_append_rope_stream_and_graph():
    import paper_2605_29657_gb300 as occ
    c = make(layers=1, T=16, dim=64, heads=2, stale=False)
    occ.occam_cache_extend(c, dev([1]), dev([33]))
    q, k, v, pos, freq, axis = case(33, 4, 2, 64, 64, 3, "bf16", 1)
    q2, k2, v2, pos2, _, _ = case(33, 4, 2, 64, 64, 3, "bf16", 2)
    seqs, off = dev([1]), dev([0, 33], I64)
    want = []
    for x in ((q, k, v, pos), (q2, k2, v2, pos2)):
        c.k_scale.fill_(1.0), c.v_scale.fill_(1.0)
        out = occ.occam_cache_append_rope(c, 0, *x[:3], seqs, off, x[3], freq, axis)
        want.append((out, c.k.view(torch.uint8).clone(), c.v.view(torch.uint8).clone()))
    a = [x.contiguous().clone() for x in (q2, k2, v2, pos2)]
    out = torch.zeros_like(a[0])
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    occ.occam_cache_append_rope(c, 0, *a[:3], seqs, off, a[3], freq, axis, out_q=out, ws=c.alloc_workspace(), stream=st)
    torch.cuda.synchronize()
    assert torch.equal(out, want[1][0]) and torch.equal(c.k.view(torch.uint8), want[1][1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        occ.occam_cache_append_rope(c, 0, *a[:3], seqs, off, a[3], freq, axis, out_q=out)
    for n, x in enumerate(((q, k, v, pos), (q2, k2, v2, pos2))):
        for to, y in zip(a, x):
            to.copy_(y)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[n][0]) and torch.equal(c.k.view(torch.uint8), want[n][1]) and torch.equal(c.v.view(torch.uint8), want[n][2])
    assert c.status() == 0


def test_append_rope_refusals():
    import paper_2605_29657_gb300 as occ
    c = make(layers=1, T=16, dim=64, heads=2)
    q, k, v, pos, freq, axis = case(5, 4, 2, 64, 64, 3, "bf16")
    s, off = dev([0]), dev([0, 5], I64)

    def call(layer=0, q=q, k=k, v=v, s=s, off=off, pos=pos, freq=freq, axis=axis, **kw):
        return occ.occam_cache_append_rope(c, layer, q, k, v, s, off, pos, freq, axis, **kw)

    wide = torch.ones(33, device="cuda")
    far = torch.zeros((5, 4, 128), dtype=torch.bfloat16, device="cuda")[..., :64]
    overlap = torch.zeros((6, 4, 64), dtype=torch.bfloat16, device="cuda")
    for bad in (
        dict(layer=1), dict(layer=-1), dict(q=q.half()), dict(k=k.half()), dict(v=v.half()), dict(q=q[:4]), dict(v=v[:4]), dict(k=k[:, :1]),
        dict(s=s.long()), dict(off=off[:1]), dict(pos=pos[:, :4]), dict(pos=pos.long()), dict(pos=torch.zeros((9, 5), dtype=torch.int32, device="cuda")),
        dict(freq=wide, axis=wide.int()), dict(freq=freq.double()), dict(axis=axis[:3]), dict(pairing="other"), dict(q=None, out_q=q),
        dict(out_q=far[:4]), dict(q=q.cpu()), dict(ws=c.ws[:256]), dict(q=overlap[:5], out_q=overlap[1:]),
        dict(q=q.clone(), out_q=k.as_strided((5, 4, 64), k.stride(), k.storage_offset())),  # over the keys
    ):
        with pytest.raises(occ.OccamError):
            call(**bad)


@pytest.mark.parametrize("dim,rot,pairing", [(128, 128, "half"), (64, 64, "half"), (128, 24, "half"), (128, 128, "adjacent")])
def test_append_rope_codes_do_not_depend_on_the_queries(dim, rot, pairing):
    """The same keys beside queries of every alignment, and none: the same codes, and queries turned to the same bits."""
    import paper_2605_29657_gb300 as occ
    rows, heads = 4096, 16
    c = make(layers=1, pages=rows // 64 + 1, heads=heads, dim=dim, T=64, seqs=1, max_pages=rows // 64, stale=False)
    seqs, off = dev([0]), dev([0, rows], I64)
    occ.occam_cache_extend(c, seqs, dev([rows]))
    q, k, v, pos, freq, axis = case(rows, 2, heads, dim, rot, 3, "f16", 4)
    odd = torch.zeros(rows * (2 * dim + 6) + 1, dtype=torch.float16, device="cuda")
    some = [None, q, odd[1:].view(rows, 2 * dim + 6)[:, :2 * dim].unflatten(1, (2, dim)), odd[:-1].view(rows, 2 * dim + 6)[:, 4:2 * dim + 4].unflatten(1, (2, dim))]
    codes, turned = [], []
    for x in some:
        if x is not None:
            x.copy_(q)
        c.k_scale.fill_(1.0), c.v_scale.fill_(1.0)
        out = occ.occam_cache_append_rope(c, 0, x, k, v, seqs, off, pos, freq, axis, pairing=pairing)
        codes.append((c.k.view(torch.uint8).clone(), c.v.view(torch.uint8).clone(), c.k_scale.clone(), c.v_scale.clone()))
        if x is not None:
            turned.append(out)
    assert c.status() == 0
    for x in codes[1:]:
        assert all(torch.equal(a, b) for a, b in zip(x, codes[0]))
    assert all(torch.equal(x, turned[0]) for x in turned[1:])


@pytest.mark.parametrize("n", [255, 256, 700])
def test_append_rope_of_many_conversations(n):
    """Fewer sequences than a CTA has threads, as many, and more; empty ones, rows before and behind."""
    c = make(layers=1, pages=2 * n, heads=1, dim=64, T=16, seqs=n, max_pages=3)
    ref = R.Cache(c)
    g = torch.Generator().manual_seed(n)
    seqs = torch.randperm(n, generator=g).tolist()
    for _ in range(2):
        counts = torch.randint(-3, 10, (n,), generator=g).clamp(min=0).tolist()
        q, k, v, pos, freq, axis = case(sum(counts) + 30, 2, 1, 64, 64, 2, "bf16", n)
        out = append(c, ref, 0, q, k, v, pos, freq, axis, "half", seqs, counts, first=19)
        close(out, q, pos, freq, axis, "half", False)


@pytest.mark.parametrize("more", [0, 300])
@pytest.mark.parametrize("off", [[0, 640, 0, 640], [0, 320, 192, 400], [300, 640, 0, 300]])
def test_append_offsets_that_go_back_are_recorded(off, more):
    """Also where no page of the sequence between them is looked at, or sequences take each other's places."""
    import paper_2605_29657_gb300 as occ
    n = 3 + more
    c = make(layers=1, pages=64, heads=1, dim=64, T=64, seqs=n, max_pages=10, stale=False)
    seqs = dev(list(range(n)))
    counts = [max(b - a, 0) for a, b in zip(off, off[1:])]
    occ.occam_cache_extend(c, dev([0, 1, 2]), dev(counts))
    assert c.status() == 0
    q, k, v, pos, freq, axis = case(640, 1, 1, 64, 64, 1, "bf16")
    all_off = dev(off + off[-1:] * more, I64)
    occ.occam_cache_append_rope(c, 0, q, k, v, seqs, all_off, pos, freq, axis)
    assert c.status() == 1
    occ.occam_cache_append(c, 0, k, v, seqs, all_off)
    assert c.status() == 1
