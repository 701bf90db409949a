"""The paged 8-bit cache against its definition in 64 bits: append and the page
calls exactly, attention within bounds derived from the data
(cache_reference.Cache.attend)."""

from __future__ import annotations

import math

import pytest
import torch

import cache_reference as R

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f16": torch.float16}


def make(layers=2, pages=40, heads=2, dim=64, T=16, seqs=6, max_pages=12, seed=0, stale=True):
    """A cache whose unused codes are random bytes (NaN codes among them) and whose scales are wild."""
    import paper_2605_29657_gb300 as occ
    c = occ.PagedCache(layers, pages, heads, dim, seqs, max_pages, page_tokens=T)
    if stale:
        g = torch.Generator().manual_seed(seed)
        for x in (c.k, c.v):
            x.view(torch.uint8).copy_(torch.randint(0, 256, x.shape, generator=g, dtype=torch.uint8))
        for x in (c.k_scale, c.v_scale):
            x.copy_(torch.randn(x.shape, generator=g) * 1e30)
    return c


def dev(x, dt=torch.int32):
    return torch.tensor(x, dtype=dt, device="cuda")


def offs(rows):
    out = [0]
    for r in rows:
        out.append(out[-1] + r)
    return out


def grow(c, ref, seqs, counts, seed, dtype=torch.bfloat16, gain=1.0, layers=None):
    """Extends sequences and appends random rows to every layer, in the cache and in the reference."""
    import paper_2605_29657_gb300 as occ
    occ.occam_cache_extend(c, dev(seqs), dev(counts))
    ref.extend(seqs, counts)
    off = offs(counts)
    g = torch.Generator().manual_seed(seed)
    for layer in range(c.layers if layers is None else layers):
        kv = (torch.randn((off[-1], 2 * c.heads, c.dim), generator=g) * gain *
              torch.exp(torch.randn((off[-1], 2 * c.heads, 1), generator=g))).to(dtype).cuda()
        k, v = kv[:, :c.heads], kv[:, c.heads:]  # strided rows
        occ.occam_cache_append(c, layer, k, v, dev(seqs), dev(off, torch.int64))
        ref.append(layer, k, v, seqs, off)
    assert c.status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("T,dim,heads", [(16, 64, 2), (32, 128, 1), (64, 128, 3), (128, 64, 2), (128, 128, 1), (16, 128, 5)])
def test_append(dtype, T, dim, heads):
    c = make(heads=heads, dim=dim, T=T, max_pages=9)
    ref = R.Cache(c)
    # fresh pages, then single tokens and ragged runs into half-filled ones; later tokens larger, so scales grow
    for n, (seqs, counts, gain) in enumerate([
            ([4, 1, 2], [T + 1, 3, 2 * T], 1.0), ([1, 4], [1, 1], 30.0), ([2, 0, 1], [0, 5, T], 1e-3), ([4, 1, 0, 2], [1, 2 * T - 1, 1, 1], 1e3)]):
        grow(c, ref, seqs, counts, n, DT[dtype], gain)
        R.assert_codes(c, ref)


def test_append_special_values_and_repeat():
    import paper_2605_29657_gb300 as occ
    c = make(layers=1, T=16, dim=64, heads=2)
    ref = R.Cache(c)
    x = torch.randn((21, 2, 64), generator=torch.Generator().manual_seed(1)).bfloat16()
    x[0, 0] = 0.0
    x[1:17, 1] = 0.0                       # a block of zeros
    x[2, 0, 3], x[3, 0, 4] = float("inf"), float("-inf")
    x[4, 0, 5] = float("nan")
    x[5, 0, 6] = 3.3e38                    # the largest values
    x[18, 1, 7] = 1e-40                    # a subnormal among zeros
    x[17, 1], x[19:, 1] = 0.0, 0.0
    x[18, 1, 8:] = 0.0
    # every tie between neighbouring codes, both signs
    x[20, 0] = torch.tensor([(1 + (2 * i + 1) / 16) * 2.0 ** (j - 6) * s for s in (1, -1) for j in range(4) for i in range(8)]).bfloat16()
    x = x.cuda()
    occ.occam_cache_extend(c, dev([3]), dev([21]))
    ref.extend([3], [21])
    ref.append(0, x, -x, [3], [0, 21])
    for _ in range(2):  # repeating a call changes nothing
        occ.occam_cache_append(c, 0, x, -x, dev([3]), dev([0, 21], torch.int64))
        R.assert_codes(c, ref)
    # a held block whose scale is no power of two, and one that is larger than needed
    c.k_scale[0, int(c.table[3, 1])] = 0.37
    c.v_scale[0, int(c.table[3, 1])] = 5e5
    ref = R.Cache(c)
    y = (40 * torch.randn((3, 2, 64), generator=torch.Generator().manual_seed(2))).half().cuda()
    occ.occam_cache_extend(c, dev([3]), dev([3]))
    occ.occam_cache_append(c, 0, y, y, dev([3]), dev([0, 3], torch.int64))
    ref.extend([3], [3])
    ref.append(0, y, y, [3], [0, 3])
    R.assert_codes(c, ref)
    assert c.status() == 0


def test_append_many_sequences_and_rows_outside():
    """More sequences than one warp searches at a time; rows before row_off[0] and after row_off[n] belong to none."""
    import paper_2605_29657_gb300 as occ
    n = 150
    c = make(layers=1, pages=400, heads=1, dim=64, T=16, seqs=n, max_pages=3)
    ref = R.Cache(c)
    g = torch.Generator().manual_seed(3)
    seqs = torch.randperm(n, generator=g).tolist()
    counts = torch.randint(0, 40, (n,), generator=g).tolist()
    occ.occam_cache_extend(c, dev(seqs), dev(counts))
    ref.extend(seqs, counts)
    off = [7 + x for x in offs(counts)]
    x = torch.randn((off[-1] + 5, 1, 64), generator=g).bfloat16().cuda()
    occ.occam_cache_append(c, 0, x, x, dev(seqs), dev(off, torch.int64))
    ref.append(0, x, x, seqs, off)
    R.assert_codes(c, ref)
    assert c.status() == 0


@pytest.mark.parametrize("T,dim,heads,layers", [(16, 64, 2, 3), (64, 128, 5, 2), (32, 64, 1, 1), (128, 128, 2, 1)])
def test_pages(T, dim, heads, layers):
    """A life of a pool: grow, fork, prune, grow the forks, release, reuse."""
    import paper_2605_29657_gb300 as occ
    c = make(layers=layers, pages=60, heads=heads, dim=dim, T=T, seqs=9, max_pages=8)
    ref = R.Cache(c)
    grow(c, ref, [0, 5, 7], [3 * T + 5, 4 * T, 1], 0)
    occ.occam_cache_fork(c, dev([0, 5, 0, 7, 8]), dev([1, 2, 3, 4, 6]))  # 8 is empty
    ref.fork([0, 5, 0, 7, 8], [1, 2, 3, 4, 6])
    R.assert_codes(c, ref)
    grow(c, ref, [3, 1, 4, 2, 6], [1, T, 0, 2, 3], 1, gain=20.0)
    R.assert_codes(c, ref)
    g = torch.Generator().manual_seed(4)
    for n, (seqs, rate, lead, short) in enumerate([([1, 3], 0.3, T + 2, 0), ([2, 0, 8], 0.9, 2 * T, 3), ([4, 6], 0.0, 0, 0), ([5, 3], 1.1, 0, 7)]):
        flags, off = [], [0]
        for s in seqs:
            m = max(ref.length[s] - short, 0)
            f = torch.rand(m, generator=g) < rate
            f[:lead] = True
            flags += f.tolist()
            off.append(off[-1] + m)
        layer_range = (0, layers) if n != 1 else (0, max(1, layers - 1))
        occ.occam_cache_compact(c, dev(seqs), dev(flags or [0], torch.uint8), dev(off, torch.int64), layers=layer_range)
        ref.compact(seqs, flags, off, layer_range)
        assert c.status() == 0
        R.assert_codes(c, ref)
    grow(c, ref, [2, 4, 1], [T + 1, 3, 1], 2)
    R.assert_codes(c, ref)
    occ.occam_cache_release(c, dev([5, 8, 1, 5]))  # an empty one, and one listed twice
    ref.release([5, 8, 1])
    R.assert_codes(c, ref)
    grow(c, ref, [8, 5], [2 * T, 5], 3)
    R.assert_codes(c, ref)
    occ.occam_cache_release(c, dev(list(range(9))))
    ref.release(range(9))
    R.assert_codes(c, ref)
    assert sum(ref.refs) == 0 and c.status() == 0


def test_pages_many_sequences():
    """More sequences than the bookkeeping kernel has threads, more pages than it scans at once."""
    import paper_2605_29657_gb300 as occ
    n = 1100
    c = make(layers=1, pages=9000, heads=1, dim=64, T=16, seqs=2 * n, max_pages=6, stale=False)
    ref = R.Cache(c)
    g = torch.Generator().manual_seed(0)
    counts = torch.randint(0, 60, (n,), generator=g).tolist()
    a, b = list(range(0, 2 * n, 2)), list(range(1, 2 * n, 2))
    occ.occam_cache_extend(c, dev(a), dev(counts))
    ref.extend(a, counts)
    occ.occam_cache_fork(c, dev(a), dev(b))
    ref.fork(a, b)
    flags = (torch.rand(sum(counts), generator=g) < 0.5).tolist()
    occ.occam_cache_compact(c, dev(b), dev(flags, torch.uint8), dev(offs(counts), torch.int64))
    ref.compact(b, flags, offs(counts), (0, 0))
    assert torch.equal(c.table.cpu(), ref.table) and c.refs.cpu().tolist() == ref.refs and c.length.cpu().tolist() == ref.length
    assert c.status() == 0


def attend_case(c, seqs, rows, heads, dtype=torch.bfloat16, seed=0, gain=1.5, **kw):
    import paper_2605_29657_gb300 as occ
    off = offs(rows)
    g = torch.Generator().manual_seed(seed)
    fused = (gain * torch.randn((off[-1], heads + 2, c.dim), generator=g)).to(dtype).cuda()
    q = fused[:, :heads]  # strided rows
    ref = R.Cache(c)
    args = dict(kw)
    for name, dt in (("keep", torch.uint8), ("keep_off", torch.int64)):
        if args.get(name) is not None:
            args[name] = dev(args[name], dt)
    out, lse = occ.occam_cache_attend(c, 0, q, dev(seqs), dev(off, torch.int64), max(rows + [0]), **args)
    want, wlse, tol, ltol = ref.attend(0, q, seqs, off, kw.get("scale", 0.0), kw.get("causal", True), kw.get("keep"), kw.get("keep_off"))
    assert c.status() == 0
    nan = torch.isnan(want)
    got = out.double().cpu()
    assert torch.equal(torch.isnan(got), nan)
    u = R.UNIT[dtype]
    bound = u * want.abs() + R.TINY[dtype] + (1 + u) * tol
    over = ((got - want).abs() - bound)[~nan]
    assert over.numel() == 0 or float(over.max()) <= 0, float(over.max())
    l = lse.double().cpu()
    assert torch.equal(torch.isinf(l) & (l < 0), torch.isinf(wlse) & (wlse < 0))
    assert torch.equal(torch.isnan(l), torch.isnan(wlse))
    fin = torch.isfinite(wlse)
    assert bool(((l - wlse).abs() <= ltol)[fin].all())
    return out, lse


ATTEND = [
    # T, dim, kv heads, group, lengths, rows
    (16, 64, 1, 1, [1], [1]),
    (64, 128, 2, 4, [33, 1, 64, 200], [1, 1, 1, 1]),
    (16, 128, 1, 8, [170, 16, 31], [1, 0, 1]),
    (32, 64, 3, 2, [100, 5, 77], [4, 5, 2]),
    (128, 128, 1, 5, [129, 300], [3, 1]),
    (16, 128, 2, 7, [40, 190], [9, 33]),
    (64, 128, 1, 4, [300, 70, 129, 2], [130, 70, 65, 1]),
    (32, 64, 2, 1, [333, 128], [333, 100]),
    (16, 128, 1, 64, [90], [2]),
]


def filled(T, dim, hkv, lengths, seed=0, pages=None, gain=1.0):
    c = make(layers=1, pages=pages or sum(-(-n // T) for n in lengths) + 2, heads=hkv, dim=dim, T=T, seqs=len(lengths) + 1,
             max_pages=max(-(-n // T) for n in lengths) + 1, seed=seed)
    seqs = list(range(len(lengths), 0, -1))
    grow(c, R.Cache(c), seqs, lengths, seed + 1, gain=gain)
    return c, seqs


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n", range(len(ATTEND)))
def test_attend(n, dtype):
    T, dim, hkv, G, lengths, rows = ATTEND[n]
    c, seqs = filled(T, dim, hkv, lengths, n)
    attend_case(c, seqs, rows, hkv * G, DT[dtype], n)
    attend_case(c, seqs, rows, hkv * G, DT[dtype], n + 50, causal=False, scale=0.3)


@pytest.mark.parametrize("n", range(len(ATTEND)))
@pytest.mark.parametrize("causal", [True, False])
def test_attend_hidden_tokens(n, causal):
    """Keep flags at every rate, shorter and longer than the sequence; some rows see nothing."""
    T, dim, hkv, G, lengths, rows = ATTEND[n]
    c, seqs = filled(T, dim, hkv, lengths, n)
    g = torch.Generator().manual_seed(n)
    for rate, extra in ((0.5, 0), (0.05, 3), (0.0, 0), (0.0, -2), (1.0, -5)):
        keep, off = [], [0]
        for x in lengths:
            m = max(x + extra, 0)
            keep += (torch.rand(m, generator=g) < rate).int().tolist()
            off.append(off[-1] + m)
        attend_case(c, seqs, rows, hkv * G, seed=n, causal=causal, keep=keep or [0], keep_off=off)


def test_attend_nothing_seen_is_zero():
    c, seqs = filled(16, 64, 2, [40, 20], 0)
    out, lse = attend_case(c, seqs, [3, 20], 4, keep=[0] * 60, keep_off=[0, 40, 60])
    assert not out.any() and bool((lse == -float("inf")).all())


@pytest.mark.parametrize("T,dim,G,lengths,rows", [(16, 128, 1, [90], [1]), (64, 64, 4, [200, 70], [40, 70]), (32, 128, 2, [300], [300])])
def test_attend_nan_counts_for_rows_that_see_it(T, dim, G, lengths, rows):
    """NaN codes in keys and values of hidden tokens, of later tokens, and of seen ones."""
    c, seqs = filled(T, dim, 1, lengths, 9)
    ref = R.Cache(c)
    raw_k, raw_v = c.k.view(torch.uint8), c.v.view(torch.uint8)

    def put(raw, i, p, d, x):
        raw[0, int(ref.table[seqs[i], p // T]), 0, p % T, d] = x

    keep = []
    for i, n in enumerate(lengths):
        f = [1] * n
        for p in (0, 17, n // 2):
            f[p] = 0
            put(raw_v, i, p, p % dim, 0xFF)
            put(raw_k, i, p, 3, 0x7F)
        keep += f
    attend_case(c, seqs, rows, G, keep=keep, keep_off=offs(lengths))
    for i, n in enumerate(lengths):  # values of tokens that only the later rows see
        put(raw_v, i, n - 1, 5, 0x7F)
        put(raw_v, i, n - 1 - rows[i] // 2, 6, 0xFF)
        put(raw_v, i, max(0, n - 1 - rows[i]), 7, 0xFF)
    attend_case(c, seqs, rows, G, keep=keep, keep_off=offs(lengths))
    put(raw_k, 0, lengths[0] - 1 - rows[0] // 3, 2, 0x7F)  # a key: whole rows
    attend_case(c, seqs, rows, G, keep=keep, keep_off=offs(lengths))


@pytest.mark.parametrize("T,dim", [(16, 128), (64, 128), (128, 64)])
@pytest.mark.parametrize("rows", [1, 7, 70])
def test_attend_long_caches_mostly_hidden(T, dim, rows):
    """Many tiles with few seen tokens, whole tiles without one, flags that end inside the sequence."""
    lengths, g = [1500, 700, 129], torch.Generator().manual_seed(T + rows)
    c, seqs = filled(T, dim, 1, lengths, T)
    keep, off = [], [0]
    for n in lengths:
        m = n - rows // 2
        f = torch.rand(m, generator=g) < 0.1
        f[m // 4:m // 2] = False
        keep += f.int().tolist()
        off.append(off[-1] + m)
    for causal in (True, False):
        attend_case(c, seqs, [rows] * 3, 4, seed=T, causal=causal, keep=keep, keep_off=off)


@pytest.mark.parametrize("T,rows", [(16, 1), (64, 1), (16, 60), (128, 200)])
def test_attend_scales_far_apart(T, rows):
    """Scales of v far apart, the large ones where the probabilities are 0: what is seen keeps its digits."""
    c, seqs = filled(T, 128, 1, [260], 3)
    pages = c.table[seqs[0], :-(-260 // T)].long()
    n = pages.shape[0]
    c.v_scale[0, pages, 0] = torch.tensor([2.0 ** ((-1) ** i * (i * 29 // n)) for i in range(n)], device="cuda")
    attend_case(c, seqs, [rows], 4)
    c.k_scale[0, pages, 0] = torch.tensor([0.02 if i % 2 else 0.3 for i in range(n)], device="cuda")
    c.v_scale[0, pages, 0] = torch.tensor([0.37 if i % 2 else 1e5 for i in range(n)], device="cuda")
    attend_case(c, seqs, [rows], 4)
    # one page's values dwarf the others, and its keys are never chosen
    c.v_scale[0, pages[0], 0] = 2.0 ** 50
    keep = [0] * T + [1] * (260 - T)
    attend_case(c, seqs, [rows], 4, keep=keep, keep_off=[0, 260])


def test_attend_large_and_small_queries():
    c, seqs = filled(32, 64, 2, [150], 3)
    for gain in (1e-30, 1e-4, 30.0):
        attend_case(c, seqs, [2], 4, gain=gain)
        attend_case(c, seqs, [70], 4, gain=gain)


@pytest.mark.parametrize("rows", [[1, 1, 1], [20, 1, 300]])
def test_attend_long_splits_many_ways(rows):
    """Few items over many keys: every item is split between CTAs; two runs agree bit for bit."""
    c, seqs = filled(64, 128, 1, [5000, 100, 3000], 5, gain=0.7)
    a, la = attend_case(c, seqs, rows, 2)
    b, lb = attend_case(c, seqs, rows, 2)
    assert torch.equal(a, b) and torch.equal(la, lb)


def test_attend_many_sequences():
    n = 700
    g = torch.Generator().manual_seed(1)
    lengths = torch.randint(1, 50, (n,), generator=g).tolist()
    c, seqs = filled(16, 64, 1, lengths, 5)
    attend_case(c, seqs, [1 if i % 5 else 0 for i in range(n)], 2)
    attend_case(c, seqs, [min(x, 1 + i % 9) for i, x in enumerate(lengths)], 2)


def test_offsets_past_32_bits():
    """A pool of more than 2^32 codes a tensor: pages at its end."""
    import paper_2605_29657_gb300 as occ
    pages = (1 << 32) // (2 * 128 * 128) + 50  # 4.3 GB a tensor
    c = occ.PagedCache(1, pages, 2, 128, 3, 3, page_tokens=128)
    c.refs[:pages - 9] = 1
    small = make(layers=1, pages=9, heads=2, dim=128, T=128, seqs=3, max_pages=3)
    g = torch.Generator().manual_seed(0)
    off = dev([0, 200, 330], torch.int64)
    x, y = (torch.randn((330, 2, 128), generator=g).bfloat16().cuda() for _ in range(2))
    q = torch.randn((330, 4, 128), generator=g).bfloat16().cuda()
    got = []
    for cc in (c, small):
        occ.occam_cache_extend(cc, dev([0, 1]), dev([200, 130]))
        occ.occam_cache_append(cc, 0, x, y, dev([0, 1]), off)
        occ.occam_cache_fork(cc, dev([1]), dev([2]))
        keep = dev([i % 3 != 0 for i in range(130)], torch.uint8)
        occ.occam_cache_compact(cc, dev([2]), keep, dev([0, 130], torch.int64))
        res = list(occ.occam_cache_attend(cc, 0, q, dev([0, 1]), off, 200))
        res += occ.occam_cache_attend(cc, 0, q[:2], dev([2, 0]), dev([0, 1, 2], torch.int64), 1)
        assert cc.status() == 0
        got.append(res)
    assert c.table[:2].min() >= -1 and int(c.table.max()) >= pages - 9
    for a, b in zip(*got):
        assert torch.equal(a, b)


def test_streams_and_graph():
    """A call on a stream of its own, and a captured sequence of calls replayed."""
    import paper_2605_29657_gb300 as occ
    c, seqs = filled(64, 128, 2, [300, 100], 5)
    q = torch.randn((2, 8, 128), generator=torch.Generator().manual_seed(0)).bfloat16().cuda()
    s, off = dev(seqs), dev([0, 1, 2], torch.int64)
    want, wl = occ.occam_cache_attend(c, 0, q, s, off, 1)
    st = torch.cuda.Stream()
    ws = c.alloc_workspace()
    st.wait_stream(torch.cuda.current_stream())
    out, lse = torch.empty_like(want), torch.empty_like(wl)
    occ.occam_cache_attend(c, 0, q, s, off, 1, out=out, lse=lse, ws=ws, stream=st)
    st.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, wl)
    ref = R.Cache(c)
    k = torch.randn((2, 2, 128), generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    one = dev([1, 1])
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        occ.occam_cache_extend(c, s, one)
        occ.occam_cache_append(c, 0, k, k, s, off)
        occ.occam_cache_attend(c, 0, q, s, off, 1, out=out, lse=lse)
    for _ in range(3):
        graph.replay()
        ref.extend(seqs, [1, 1])
        ref.append(0, k, k, seqs, [0, 1, 2])
    torch.cuda.synchronize()
    R.assert_codes(c, ref)
    got, gl = occ.occam_cache_attend(c, 0, q, s, off, 1)
    assert torch.equal(out, got) and torch.equal(lse, gl)


def test_device_errors_change_nothing():
    """Wrong slots, counts and full pools are recorded, and no state moves."""
    import paper_2605_29657_gb300 as occ
    c = make(layers=1, pages=6, heads=1, dim=64, T=16, seqs=4, max_pages=4)
    ref = R.Cache(c)
    grow(c, ref, [0, 1], [20, 16], 0)
    INV, CAP = 1, 2
    i64 = torch.int64
    calls = [
        (CAP, lambda: occ.occam_cache_extend(c, dev([2]), dev([64]))),            # the pool: 4 pages wanted, 3 free
        (CAP, lambda: occ.occam_cache_extend(c, dev([2, 0]), dev([1, 45]))),      # the table: 65 tokens in 4 pages
        (INV, lambda: occ.occam_cache_extend(c, dev([2, 2]), dev([1, 1]))),       # listed twice
        (INV, lambda: occ.occam_cache_extend(c, dev([4]), dev([1]))),
        (INV, lambda: occ.occam_cache_extend(c, dev([-1]), dev([1]))),
        (INV, lambda: occ.occam_cache_extend(c, dev([2]), dev([-1]))),
        (INV, lambda: occ.occam_cache_fork(c, dev([0]), dev([1]))),               # not empty
        (INV, lambda: occ.occam_cache_fork(c, dev([2]), dev([2]))),               # itself
        (INV, lambda: occ.occam_cache_fork(c, dev([9]), dev([2]))),
        (INV, lambda: occ.occam_cache_fork(c, dev([0, 0]), dev([2, 2]))),
        (INV, lambda: occ.occam_cache_compact(c, dev([0, 0]), dev([1] * 40, torch.uint8), dev([0, 20, 40], i64))),
        (INV, lambda: occ.occam_cache_compact(c, dev([0]), dev([1] * 20, torch.uint8), dev([0, 21], i64))),
        (INV, lambda: occ.occam_cache_compact(c, dev([0]), dev([1] * 20, torch.uint8), dev([5, 2], i64))),
        (INV, lambda: occ.occam_cache_release(c, dev([7]))),
        (INV, lambda: occ.occam_cache_append(c, 0, torch.ones(21, 1, 64).bfloat16().cuda(), torch.ones(21, 1, 64).bfloat16().cuda(), dev([0]), dev([0, 21], i64))),
        (INV, lambda: occ.occam_cache_append(c, 0, torch.ones(3, 1, 64).bfloat16().cuda(), torch.ones(3, 1, 64).bfloat16().cuda(), dev([0]), dev([0, 4], i64))),
        (INV, lambda: occ.occam_cache_append(c, 0, torch.ones(3, 1, 64).bfloat16().cuda(), torch.ones(3, 1, 64).bfloat16().cuda(), dev([5]), dev([0, 3], i64))),
        (INV, lambda: occ.occam_cache_attend(c, 0, torch.ones(21, 2, 64).bfloat16().cuda(), dev([0]), dev([0, 21], i64), 21)),
        (INV, lambda: occ.occam_cache_attend(c, 0, torch.ones(1, 2, 64).bfloat16().cuda(), dev([6]), dev([0, 1], i64), 1)),
        (INV, lambda: occ.occam_cache_attend(c, 0, torch.ones(1, 2, 64).bfloat16().cuda(), dev([0]), dev([0, 1], i64), 1, keep=dev([1] * 9, torch.uint8), keep_off=dev([0, 20], i64))),
    ]
    for n, (code, f) in enumerate(calls):
        f()
        assert c.status() == code, n
        R.assert_codes(c, ref)
    # a pool that is too full for a prune of shared pages, and the same once there is room
    occ.occam_cache_extend(c, dev([2]), dev([48]))
    ref.extend([2], [48])
    flags = dev([i % 2 for i in range(20)], torch.uint8)
    occ.occam_cache_compact(c, dev([0]), flags, dev([0, 20], i64))
    assert c.status() == CAP
    R.assert_codes(c, ref)
    occ.occam_cache_release(c, dev([2]))
    ref.release([2])
    occ.occam_cache_compact(c, dev([0]), flags, dev([0, 20], i64))
    ref.compact([0], flags.tolist(), [0, 20], (0, 1))
    assert c.status() == 0
    R.assert_codes(c, ref)


def test_max_rows_is_only_a_hint():
    import paper_2605_29657_gb300 as occ
    c, seqs = filled(64, 128, 1, [300, 90, 50], 5)
    rows = [100, 1, 7]
    off = dev(offs(rows), torch.int64)
    q = torch.randn((108, 4, 128), generator=torch.Generator().manual_seed(0)).bfloat16().cuda()
    want, _, tol, _ = R.Cache(c).attend(0, q, seqs, offs(rows))
    for hint in (0, 1, 3, 100, 5000):
        out, _ = occ.occam_cache_attend(c, 0, q, dev(seqs), off, hint)
        assert bool(((out.double().cpu() - want).abs() <= R.UNIT[q.dtype] * want.abs() + 1.01 * tol).all()), hint


def test_refusals():
    import paper_2605_29657_gb300 as occ
    c, seqs = filled(16, 64, 2, [40, 20], 0)
    s, off = dev(seqs), dev([0, 1, 2], torch.int64)
    q, k = torch.ones(2, 4, 64).bfloat16().cuda(), torch.ones(2, 2, 64).bfloat16().cuda()
    wide = torch.ones(2, 2 * 64 + 4).bfloat16().cuda()
    bad = [
        lambda: occ.PagedCache(1, 4, 1, 96, 2, 2),
        lambda: occ.PagedCache(1, 4, 1, 64, 2, 2, page_tokens=48),
        lambda: occ.PagedCache.wrap(c.k, c.v[:, :3], c.k_scale, c.v_scale, c.table, c.length, c.refs),
        lambda: occ.PagedCache.wrap(c.k, c.v, c.k_scale, c.v_scale, c.table, c.length, c.refs[:3]),
        lambda: occ.occam_cache_attend(c, 1, q, s, off, 1),
        lambda: occ.occam_cache_attend(c, 0, q[:, :3], s, off, 1),
        lambda: occ.occam_cache_attend(c, 0, q.float(), s, off, 1),
        lambda: occ.occam_cache_attend(c, 0, q, s.long(), off, 1),
        lambda: occ.occam_cache_attend(c, 0, q, s, off[:2], 1),
        lambda: occ.occam_cache_attend(c, 0, q, s, off, 1, scale=float("nan")),
        lambda: occ.occam_cache_attend(c, 0, q, s, off, 1, scale=-1.0),
        lambda: occ.occam_cache_attend(c, 0, q, s, off, 1, keep=dev([1], torch.uint8)),
        lambda: occ.occam_cache_attend(c, 0, q, s, off, 1, out=q[:1]),
        lambda: occ.occam_cache_attend(c, 0, q, s, off, 1, ws=c.ws[:256]),
        lambda: occ.occam_cache_attend(c, 0, torch.ones(2, 130, 64).bfloat16().cuda(), s, off, 1),
        lambda: occ.occam_cache_append(c, 0, k, k.half(), s, off),
        lambda: occ.occam_cache_append(c, 0, k, k[:1], s, off),
        lambda: occ.occam_cache_append(c, -1, k, k, s, off),
        lambda: occ.occam_cache_append(c, 0, torch.as_strided(wide, (2, 2, 64), (132, 64, 1), 2), k, s, off),
        lambda: occ.occam_cache_append(c, 0, torch.as_strided(wide, (2, 2, 64), (132, 64, 1)), k, s, off),
        lambda: occ.occam_cache_extend(c, s, dev([1])),
        lambda: occ.occam_cache_extend(c, dev([0, 1, 2, 3]), dev([1, 1, 1, 1])),
        lambda: occ.occam_cache_fork(c, s, dev([0])),
        lambda: occ.occam_cache_compact(c, s, dev([1] * 60, torch.uint8), dev([0, 40, 60], torch.int64), layers=(0, 2)),
        lambda: occ.occam_cache_compact(c, s, torch.ones(4096, dtype=torch.uint8, device="cuda"), dev([0, 40, 60], torch.int64)),
        lambda: occ.occam_cache_release(c, s.cpu()),
    ]
    before = R.Cache(c)
    for n, f in enumerate(bad):
        with pytest.raises(occ.OccamError):
            f()
            print("not refused", n)
    R.assert_codes(c, before)


def rows_of(n, heads, dim, seed):
    return torch.randn((n, heads, dim), generator=torch.Generator().manual_seed(seed)).bfloat16().cuda()


def test_append_behind_a_refused_extend_changes_nothing():
    """A full pool: the extend is refused for all its sequences, and the calls queued behind it write
    nothing, whether the page at the end is a sequence's own or shared, until the status is read."""
    import paper_2605_29657_gb300 as occ
    c = make(layers=2, pages=5, heads=2, dim=64, T=16, seqs=4, max_pages=4)
    ref = R.Cache(c)
    grow(c, ref, [0, 1], [32, 20], 0)
    occ.occam_cache_fork(c, dev([0]), dev([2]))
    ref.fork([0], [2])
    occ.occam_cache_extend(c, dev([3]), dev([10]))  # the last page
    ref.extend([3], [10])
    x, one = rows_of(3, 2, 64, 1), dev([1, 1, 1])
    s, off = dev([0, 1, 2]), dev([0, 1, 2, 3], torch.int64)
    for _ in range(2):  # a step that does not fit, and the next one
        occ.occam_cache_extend(c, s, one)
        for layer in range(2):
            occ.occam_cache_append(c, layer, x, x, s, off)
    occ.occam_cache_release(c, dev([3]))  # room again, but nobody has looked
    ref.release([3])
    occ.occam_cache_extend(c, dev([1]), dev([1]))
    occ.occam_cache_append(c, 0, x[:1], x[:1], dev([1]), dev([0, 1], torch.int64))
    assert c.status() == 2
    R.assert_codes(c, ref)
    grow(c, ref, [1, 2], [1, 1], 2)
    R.assert_codes(c, ref)


def test_append_writes_no_shared_page():
    import paper_2605_29657_gb300 as occ
    c = make(layers=1, pages=8, heads=2, dim=64, T=16, seqs=4, max_pages=4)
    ref = R.Cache(c)
    grow(c, ref, [0, 3], [32, 5], 0)
    occ.occam_cache_fork(c, dev([0, 3]), dev([1, 2]))
    ref.fork([0, 3], [1, 2])
    x = rows_of(3, 2, 64, 1)
    for seqs, off in (([1], [0, 1]), ([0, 1], [0, 1, 2]), ([1], [0, 3])):  # not extended: the last rows are shared
        occ.occam_cache_append(c, 0, x[:off[-1]], x[:off[-1]], dev(seqs), dev(off, torch.int64))
        assert c.status() == 1
        R.assert_codes(c, ref)
    grow(c, ref, [1, 0, 2], [1, 2, 12], 2)
    R.assert_codes(c, ref)


def test_page_counts_past_32_bits():
    """1024 sequences that want 2^21 pages each, as many as the pool has: more than 32 bits count. The
    calls record that the pool is too small and change nothing (the table alone is 8.6 GB)."""
    import paper_2605_29657_gb300 as occ
    n, pages, T = 1 << 10, 1 << 21, 16
    c = occ.PagedCache(1, pages, 1, 64, n, pages, page_tokens=T, max_tokens=n)
    seqs = dev(list(range(n)))
    occ.occam_cache_extend(c, seqs, torch.full((n,), pages * T, dtype=torch.int32, device="cuda"))
    assert c.status() == 2
    assert not c.length.any() and not c.refs.any() and int(c.table.max()) == -1
    # every sequence holds the whole pool and drops its first token
    c.table.copy_(torch.arange(pages, dtype=torch.int32, device="cuda").expand(n, -1))
    c.length.fill_(pages * T)
    c.refs.fill_(n)
    occ.occam_cache_compact(c, seqs, torch.zeros(n, dtype=torch.uint8, device="cuda"),
                            torch.arange(n + 1, dtype=torch.int64, device="cuda"))
    assert c.status() == 2
    assert bool((c.length == pages * T).all()) and bool((c.refs == n).all())
    assert all(torch.equal(row, torch.arange(pages, dtype=torch.int32, device="cuda")) for row in c.table[::93])


def test_attention_leaves_its_counters_zero():
    """Arrivals that an unfinished call would leave behind: the counters (they follow the status
    word's 256 bytes) are zero after the next call of the tensor-core kernel, and the call after it is right."""
    import paper_2605_29657_gb300 as occ
    c, seqs = filled(64, 128, 1, [5000, 3000], 5, gain=0.7)
    q = torch.randn((500, 4, 128), generator=torch.Generator().manual_seed(0)).bfloat16().cuda()
    off = dev([0, 200, 500], torch.int64)
    want, wl = occ.occam_cache_attend(c, 0, q, dev(seqs), off, 300)
    counters = c.ws[256:256 + 4 * 513].view(torch.int32)
    assert not counters.any()
    counters[:152] = 1
    occ.occam_cache_attend(c, 0, q, dev(seqs), off, 300)
    assert not counters.any()
    out, lse = occ.occam_cache_attend(c, 0, q, dev(seqs), off, 300)
    assert torch.equal(out, want) and torch.equal(lse, wl)
    assert c.status() == 0


@pytest.mark.parametrize("rows,branches", [(1, 600), (4, 200), (2048, 1)])
def test_attend_sums_many_small_probabilities(rows, branches):
    """One key with a probability near 1 and a value of 0, 8,191 keys with a probability of 2^-27 each and a
    value of 1: the result is the sum of the small ones. (As many items as keep each on few CTAs, so
    that the small ones meet the large one's maximum.)

    Bound: a probability is held in f16, 2^15 (few rows) or 2^7 (many rows, whose reference is at most
    the maximum) times as large: 2^-11 relative or 2^-32 absolute; the exponent, 27 log 2 and a
    power of two away, is exact to 2^-20; half an ulp of the f16 result, 2^-11, or 2^-25."""
    import paper_2605_29657_gb300 as occ
    n, T, D, G = 1 << 13, 128, 64, 32 if rows > 4 else 1
    c = make(layers=1, pages=n // T, heads=1, dim=D, T=T, seqs=branches, max_pages=n // T, stale=False)
    k, v = torch.zeros((n, 1, D)), torch.zeros((n, 1, D))
    k[0, 0, 0], v[1:] = 1.0, 1.0
    occ.occam_cache_extend(c, dev([0]), dev([n]))
    occ.occam_cache_append(c, 0, k.bfloat16().cuda(), v.bfloat16().cuda(), dev([0]), dev([0, n], torch.int64))
    if branches > 1:
        occ.occam_cache_fork(c, dev([0] * (branches - 1)), dev(list(range(1, branches))))
    q = torch.zeros((rows * branches, G, D), device="cuda", dtype=torch.float16)
    q[:, :, 0] = 1.0
    off = torch.arange(branches + 1, dtype=torch.int64, device="cuda") * rows
    p = 2.0 ** -27
    l = 1 + (n - 1) * p
    want = (n - 1) * p / l
    bound = (n - 1) * ((2.0 ** -11 + 2.0 ** -20) * p + 2.0 ** -32) / l + 2.0 ** -11 * want + 2.0 ** -25
    for keep in (None, torch.ones(n * branches, dtype=torch.uint8, device="cuda")):
        out, lse = occ.occam_cache_attend(c, 0, q, dev(list(range(branches))), off, rows, scale=27 * math.log(2.0), causal=False,
                                          keep=keep, keep_off=None if keep is None else torch.arange(branches + 1, device="cuda") * n)
        assert c.status() == 0
        assert float((out.double() - want).abs().max()) <= bound, (float(out.min()), float(out.max()), want)
        # log l of a score of 27 log 2: its 2^-20 and the logarithm's own
        assert float((lse.double() - 27 * math.log(2.0) - math.log(l)).abs().max()) <= 2.0 ** -19 + 2.0 ** -22 * 27


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_compact_keeps_the_largest_values(dtype):
    """Values near the type's end, beside ordinary ones and alone, in blocks that are moved."""
    import paper_2605_29657_gb300 as occ
    c = make(layers=1, T=16, dim=64, heads=2)
    ref = R.Cache(c)
    x = torch.randn((40, 2, 64), generator=torch.Generator().manual_seed(3))
    big = 3.3e38 if dtype == "bf16" else 65504.0
    x[5, 0, 6], x[20, 1, 7] = big, -big
    x[16:24, 0] = 0.0
    x[17, 0, 1] = big  # with zeros only
    x = x.to(DT[dtype]).cuda()
    occ.occam_cache_extend(c, dev([3]), dev([40]))
    occ.occam_cache_append(c, 0, x, -x, dev([3]), dev([0, 40], torch.int64))
    ref.extend([3], [40])
    ref.append(0, x, -x, [3], [0, 40])
    R.assert_codes(c, ref)
    flags = [i % 3 != 0 for i in range(40)]
    occ.occam_cache_compact(c, dev([3]), dev(flags, torch.uint8), dev([0, 40], torch.int64))
    ref.compact([3], flags, [0, 40], (0, 1))
    R.assert_codes(c, ref)
    assert c.status() == 0


@pytest.mark.parametrize("off", [[1000, 1003], [4, 4], [-3, 0], [0, 2, 1], [0, 4, 4], [3, 2, 2]])
def test_append_offsets_outside_the_rows_are_recorded(off):
    import paper_2605_29657_gb300 as occ
    c = make(layers=1, pages=8, heads=2, dim=64, T=16, seqs=4, max_pages=4)
    ref = R.Cache(c)
    grow(c, ref, [0, 1], [32, 20], 0)
    x = rows_of(3, 2, 64, 1)
    x[2] = float("nan")  # (only good ranges of rows may be written: [0, 2) of [0, 2, 1])
    occ.occam_cache_append(c, 0, x, x, dev(list(range(len(off) - 1))), dev(off, torch.int64))
    assert c.status() == 1
    if off[:2] == [0, 2]:
        ref.append(0, x, x, [0], [0, 2])
    R.assert_codes(c, ref)


@pytest.mark.parametrize("op", ["attend", "rope"])
def test_new_results_belong_to_the_stream_that_writes_them(op):
    """Memory that the current stream has freed, with writes to it still queued there, is no place for
    the results of a call on another stream."""
    import paper_2605_29657_gb300 as occ
    c, seqs = filled(64, 128, 2, [300, 100], 5)
    rows = [200, 100]
    q = torch.randn((300, 32, 128), generator=torch.Generator().manual_seed(0)).bfloat16().cuda()  # 2.4 MB
    s, off = dev(seqs), dev(offs(rows), torch.int64)
    pos, freq, axis = torch.zeros((1, 300), dtype=torch.int32, device="cuda"), torch.ones(64, device="cuda"), dev([0] * 64)
    ws, st = c.alloc_workspace(), torch.cuda.Stream()

    def call(stream):
        if op == "attend":
            return occ.occam_cache_attend(c, 0, q, s, off, 200, ws=ws, stream=stream)[0]
        return occ.occam_rope(q, None, pos, freq, axis, stream=stream)[0]

    want = call(None)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    freed = [torch.empty_like(q) for _ in range(8)]
    torch.cuda._sleep(200_000_000)  # about 0.1 s
    for x in freed:
        x.fill_(7.0)
    del freed, x
    got = call(st)
    st.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(got, want)
