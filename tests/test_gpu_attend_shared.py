"""occam_cache_attend_shared against attention's definition in 64 bits (cache_reference.Cache.attend), over
caches that forks, appends and prunes have left.

Bound: that of attention over the cache, and the join of the two parts: their logarithms L are off by 2 fp32
roundings, their weights by that and the exponential's 2^-20, so a result moves by at most
(2^-20 + 2^-21 |L|) of sum p |v|, of which attention's own bound is at least 2^11 times 2^-11."""

from __future__ import annotations

import math

import pytest
import torch

import cache_reference as R
from test_gpu_cache import DT, dev, grow, make, offs

pytestmark = pytest.mark.gpu


def branches(T, dim, hkv, groups, seed=0, gain=1.0):
    """A cache with a prefix for each of groups [(prefix tokens, [own tokens of each fork])]; (cache, slots in order, lengths)."""
    import paper_2605_29657_gb300 as occ
    n = sum(len(own) for _, own in groups)
    parents = list(range(len(groups)))
    kids = [len(groups) + i for i in range(n)]
    lengths = [pre + x for pre, own in groups for x in own]
    pages = sum(-(-pre // T) for pre, _ in groups) + sum(-(-x // T) + 1 for _, own in groups for x in own) + 2
    c = make(layers=1, pages=pages, heads=hkv, dim=dim, T=T, seqs=len(groups) + n + 1, max_pages=max(-(-x // T) for x in lengths + [p for p, _ in groups]) + 1, seed=seed)
    ref = R.Cache(c)
    grow(c, ref, parents, [pre for pre, _ in groups], seed + 1, gain=gain)
    src = [g for g, (_, own) in enumerate(groups) for _ in own]
    occ.occam_cache_fork(c, dev(src), dev(kids))
    ref.fork(src, kids)
    grow(c, ref, kids, [x for _, own in groups for x in own], seed + 2, gain=gain)
    return c, kids, lengths


def check(c, seqs, rows, group_sizes, heads, dtype=torch.bfloat16, seed=0, gain=1.5, hints=None, scale=0.0, causal=True, known=None):
    import paper_2605_29657_gb300 as occ
    off, goff = offs(rows), offs(group_sizes)
    g = torch.Generator().manual_seed(seed)
    fused = (gain * torch.randn((off[-1], heads + 2, c.dim), generator=g)).to(dtype).cuda()
    q = fused[:, :heads]  # strided rows
    ws = c.alloc_workspace(off[-1], heads)
    most = max(sum(rows[a:b]) for a, b in zip(goff, goff[1:]))
    hints = hints or (max(rows), most)
    out, lse = occ.occam_cache_attend_shared(c, 0, q, dev(seqs), dev(off, torch.int64), hints[0], dev(goff), hints[1], ws, scale=scale,
                                             causal=causal)
    assert c.status(ws=ws) == 0
    if not known:  # (a list: what an earlier call with the same arguments is held against)
        known = [] if known is None else known
        known.extend(R.Cache(c).attend(0, q, seqs, off, scale, causal))
    want, wlse, tol, ltol = known
    tol = tol * (1 + 2.0 ** -9 + 2.0 ** -9 * wlse.nan_to_num(0, 0, 0).abs()[..., None])
    u, got = R.UNIT[dtype], out.double().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    over = ((got - want).abs() - (u * want.abs() + R.TINY[dtype] + (1 + u) * tol))[~torch.isnan(want)]
    assert over.numel() == 0 or float(over.max()) <= 0, float(over.max())
    fin = torch.isfinite(wlse)
    l = lse.double().cpu()
    assert torch.equal(torch.isfinite(l), fin)
    assert bool(((l - wlse).abs() <= ltol + 2.0 ** -20 + 2.0 ** -21 * wlse.abs())[fin].all())
    return q, out, lse, ws


def shared_tokens(c, ws, groups):
    """What the last call on a workspace shared in each group (the first thing behind the other calls' scratch)."""
    import ctypes
    import paper_2605_29657_gb300 as occ
    n = ctypes.c_size_t(0)
    assert occ.library().occam_cache_workspace_size(c._ref, 0, ctypes.byref(n)) == 0
    return ws[n.value:n.value + 4 * groups].view(torch.int32).tolist()


PAYS = [
    # T, dim, key heads, group, [(prefix, own tokens of each fork)], rows of each, full pages' tokens that are shared
    (64, 128, 8, 4, [(1100, [1, 3, 70, 2] * 10)], [1] * 40, [1088]),
    (16, 64, 16, 1, [(700, [1, 9] * 20)], [1, 2] * 20, [688]),
    (128, 128, 8, 2, [(1000, [20] * 24), (700, [5] * 30), (900, [2])], [20] * 24 + [1] * 30 + [2], [896, 640, 0]),
    (32, 128, 4, 8, [(1600, [9, 40] * 24)], [9] * 48, [1600]),
    (16, 128, 2, 7, [(4000, [1] * 50)], [1] * 50, [4000]),
    (64, 64, 4, 16, [(2900, [12, 13, 14] * 8), (2700, [12] * 24)], [12] * 48, [0, 0]),
    # (192 rows a fork and key head fill three quarters of a tile of 256 without the others': 24 tiles against 18 over 22.5 x 128
    # keys, 2 us each for 8 (group, head)s over 152 SMs: 14 us saved, and the two parts' joins cost 18 beside the launches' 15)
    (64, 64, 4, 16, [(2900, [5, 6] * 12), (2700, [4] * 24)], [3] * 48, [2880, 2688]),
    (32, 64, 8, 1, [(2000, [40, 35, 64, 129] * 8)], [35] * 32, [1984]),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n", range(len(PAYS)))
def test_attend_shared_where_it_pays(n, dtype):
    """Groups large enough that the pages are read once: single tokens and rows of more than one tile, prefixes split over
    all CTAs."""
    T, dim, hkv, G, groups, rows, tokens = PAYS[n]
    c, seqs, _ = branches(T, dim, hkv, groups, n)
    sizes = [len(own) for _, own in groups]
    known = []
    q, out, lse, ws = check(c, seqs, rows, sizes, hkv * G, DT[dtype], n, known=known)
    assert shared_tokens(c, ws, len(sizes)) == tokens
    import paper_2605_29657_gb300 as occ
    off, goff = offs(rows), dev(offs(sizes))
    most = max(sum(rows[a:b]) for a, b in zip(offs(sizes), offs(sizes)[1:]))
    for _ in range(3):  # the same every time
        o, l = occ.occam_cache_attend_shared(c, 0, q, dev(seqs), dev(off, torch.int64), max(rows), goff, most, ws)
        assert torch.equal(o, out) and torch.equal(l, lse)
    # the hints choose kernels only
    for hints in ((0, 0), (1, 10000), (max(rows), 1)):
        check(c, seqs, rows, sizes, hkv * G, DT[dtype], n, hints=hints, known=known)
    if dtype == "bf16":
        check(c, seqs, rows, sizes, hkv * G, DT[dtype], n + 50, causal=False, scale=0.3)


def test_attend_shared_values_that_are_nan_where_it_pays():
    c, seqs, _ = branches(64, 128, 8, [(1100, [3, 40] * 20)], 3)
    c.v.view(torch.uint8)[0, int(c.table[seqs[1], 17]), 2, 20, 9] = 0x7f   # an own token of the second fork
    c.v.view(torch.uint8)[0, int(c.table[seqs[2], 5]), 3, 7, 3] = 0xff     # a token of the prefix
    for rows in ([1] * 40, [3, 20] * 20):
        check(c, seqs, rows, [40], 16)


SHARED = [
    # T, dim, key heads, group, [(prefix, own tokens of each fork)], rows of each
    (16, 64, 1, 1, [(40, [1, 1])], [1, 1]),
    (64, 128, 2, 4, [(200, [1, 5, 70])], [1, 1, 1]),
    (16, 128, 1, 8, [(33, [3, 20, 1, 2]), (160, [9])], [1, 2, 0, 1, 3]),
    (32, 64, 3, 2, [(100, [1] * 12), (31, [40, 2]), (64, [64, 65])], [1] * 16),
    (128, 128, 1, 5, [(300, [7, 130])], [7, 100]),
    (16, 128, 2, 7, [(500, [1] * 9)], [1] * 9),
    (64, 128, 1, 4, [(700, [40, 1, 90, 33]), (128, [20, 20])], [40, 1, 64, 33, 3, 20]),
    (32, 64, 2, 1, [(333, [260, 20])], [260, 20]),
    (16, 128, 1, 64, [(90, [2, 3])], [2, 1]),
    (64, 64, 1, 16, [(1900, [1] * 30)], [1] * 30),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n", range(len(SHARED)))
def test_attend_shared(n, dtype):
    T, dim, hkv, G, groups, rows = SHARED[n]
    c, seqs, _ = branches(T, dim, hkv, groups, n)
    sizes = [len(own) for _, own in groups]
    check(c, seqs, rows, sizes, hkv * G, DT[dtype], n)
    check(c, seqs, rows, sizes, hkv * G, DT[dtype], n + 50, causal=False, scale=0.3)


def test_attend_shared_whatever_the_groups():
    """Groups that share nothing, one sequence each, all in one, groups of none, a sequence listed twice: the same results."""
    import paper_2605_29657_gb300 as occ
    groups = [(130, [1, 9, 33]), (70, [2, 2])]
    c, seqs, _ = branches(16, 128, 2, groups, 4)
    rows = [1, 4, 20, 2, 1]
    for sizes in ([3, 2], [5], [1, 1, 1, 1, 1], [2, 3], [0, 3, 0, 2, 0], [1, 4]):
        check(c, seqs, rows, sizes, 8, seed=3)
    check(c, [seqs[0], seqs[0], seqs[3]], [1, 1, 2], [2, 1], 8)
    # the hints choose kernels only
    for hints in ((0, 0), (1, 500), (500, 1), (20, 28)):
        check(c, seqs, rows, [3, 2], 8, seed=3, hints=hints)
    # against attention over each sequence by itself
    q, out, lse, ws = check(c, seqs, rows, [3, 2], 8, seed=7)
    o, l = occ.occam_cache_attend(c, 0, q, dev(seqs), dev(offs(rows), torch.int64), 20)
    assert float((out.float() - o.float()).abs().max()) <= 2.0 ** -6 * float(o.float().abs().max())
    torch.testing.assert_close(lse, l, rtol=1e-5, atol=1e-5)


def test_attend_shared_rows_inside_the_shared_pages():
    """Forks that have not grown: their last tokens, which ask, lie in pages that all of them hold."""
    import paper_2605_29657_gb300 as occ
    for pre in (64, 70, 16, 5):
        c = make(layers=1, pages=20, heads=2, dim=64, T=16, seqs=5, max_pages=8)
        ref = R.Cache(c)
        grow(c, ref, [0], [pre], 1)
        occ.occam_cache_fork(c, dev([0, 0, 0]), dev([1, 2, 3]))
        for rows in ([1, 1, 1, 1], [pre, 1, pre // 2, 3]):
            check(c, [0, 1, 2, 3], rows, [4], 4)


def test_attend_shared_after_one_fork_was_pruned():
    import paper_2605_29657_gb300 as occ
    c, seqs, lengths = branches(16, 64, 2, [(100, [3, 4, 5])], 9)
    occ.occam_cache_release(c, dev([0]))  # the parent goes, its pages stay
    keep = torch.ones(lengths[1], dtype=torch.uint8)
    keep[40:60] = 0  # its first two pages stay shared
    occ.occam_cache_compact(c, dev([seqs[1]]), keep.cuda(), dev([0, lengths[1]], torch.int64))
    assert c.status() == 0
    check(c, seqs, [1, 2, 3], [3], 4)


def test_attend_shared_nan_counts_for_rows_that_see_it():
    c, seqs, _ = branches(16, 64, 1, [(48, [5, 6]), (40, [5, 40])], 2)
    c.v.view(torch.uint8)[0, int(c.table[seqs[1], 3]), 0, 2, 9] = 0x7f   # the second fork's own token
    c.v.view(torch.uint8)[0, int(c.table[seqs[2], 0]), 0, 7, 3] = 0xff   # a token of the second group's prefix
    check(c, seqs, [5, 6, 3, 40], [2, 2], 2)
    check(c, seqs, [1, 1, 1, 1], [2, 2], 2)


@pytest.mark.parametrize("rows", [1, 30])
def test_attend_shared_long_prefix_repeats(rows):
    c, seqs, _ = branches(64, 128, 2, [(4100, [30, 31, 64, 65, 90])], 6)
    q, a, la, ws = check(c, seqs, [rows] * 5, [5], 8)
    import paper_2605_29657_gb300 as occ
    off = dev(offs([rows] * 5), torch.int64)
    for _ in range(3):
        b, lb = occ.occam_cache_attend_shared(c, 0, q, dev(seqs), off, rows, dev([0, 5]), 5 * rows, ws)
        assert torch.equal(a, b) and torch.equal(la, lb)


def test_attend_shared_streams_graph_and_other_calls_on_its_workspace():
    import paper_2605_29657_gb300 as occ
    c, seqs, _ = branches(16, 64, 2, [(150, [3, 4, 20])], 1)
    s, off, goff = dev(seqs), dev([0, 1, 3, 10], torch.int64), dev([0, 3])
    q = torch.randn((10, 8, 64), generator=torch.Generator().manual_seed(5)).half().cuda()
    ws = [c.alloc_workspace(10, 8) for _ in range(2)]
    want, wl = occ.occam_cache_attend_shared(c, 0, q, s, off, 7, goff, 10, ws[0])
    plain, _ = occ.occam_cache_attend(c, 0, q, s, off, 7, ws=ws[0])  # the workspace serves the other calls too
    torch.cuda.synchronize()
    st = [torch.cuda.Stream() for _ in range(2)]
    got = [occ.occam_cache_attend_shared(c, 0, q, s, off, 7, goff, 10, ws[i % 2], stream=st[i % 2]) for i in range(6)]
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) and torch.equal(l, wl) for o, l in got)
    out, lse = torch.zeros_like(want), torch.zeros_like(wl)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        occ.occam_cache_attend_shared(c, 0, q, s, off, 7, goff, 10, ws[0], out=out, lse=lse)
    for _ in range(2):
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, wl)
    # the captured call on a cache that has moved on since: one fork lost its pages
    occ.occam_cache_release(c, s[:1])
    occ.occam_cache_fork(c, s[1:2], s[:1])
    g.replay()
    torch.cuda.synchronize()
    assert c.status() == 0 and c.status(ws=ws[0]) == 0
    w, _, tol, _ = R.Cache(c).attend(0, q, seqs, [0, 1, 3, 10])
    assert bool(((out.double().cpu() - w).abs() <= 2.0 ** -11 * w.abs() + 1.2 * tol).all())
    assert torch.isfinite(plain).all()


def test_attend_shared_device_errors():
    import paper_2605_29657_gb300 as occ
    c, seqs, _ = branches(16, 64, 1, [(50, [3, 4])], 1)
    q = torch.randn((4, 2, 64), generator=torch.Generator().manual_seed(5)).bfloat16().cuda()
    ws = c.alloc_workspace(4, 2)
    off = [0, 2, 4]
    want, wl = occ.occam_cache_attend(c, 0, q, dev(seqs), dev(off, torch.int64), 2)
    for s, o, goff in ((seqs, off, [0, 1]), (seqs, off, [1, 2]), (seqs, off, [0, 3]), (seqs, off, [0, 2, 1, 2]), (seqs, off, [-1, 2]),
                       ([seqs[0], 99], off, [0, 2]), ([seqs[0], -1], off, [0, 2]), (seqs, [0, 2, 5], [0, 2]), (seqs, [0, 2, 1], [0, 2])):
        out, lse = torch.zeros_like(q), torch.zeros_like(wl)
        occ.occam_cache_attend_shared(c, 0, q, dev(s), dev(o, torch.int64), 2, dev(goff), 4, ws, out=out, lse=lse)
        assert c.status(ws=ws) == 1, (s, o, goff)
        # what fits is right all the same
        assert float((out[:2].float() - want[:2].float()).abs().max()) < 0.05, (s, o, goff)
    out, lse = occ.occam_cache_attend_shared(c, 0, q, dev(seqs), dev(off, torch.int64), 2, dev([0, 2]), 4, ws)
    assert c.status(ws=ws) == 0 and float((out.float() - want.float()).abs().max()) < 0.05


def test_attend_shared_refusals():
    import paper_2605_29657_gb300 as occ
    c, seqs, _ = branches(16, 64, 1, [(50, [3, 4])], 1)
    q = torch.ones((4, 2, 64), device="cuda").bfloat16()
    ws, s, off, goff = c.alloc_workspace(4, 2), dev(seqs), dev([0, 2, 4], torch.int64), dev([0, 2])
    call = occ.occam_cache_attend_shared
    for f in (
        lambda: call(c, 1, q, s, off, 2, goff, 4, ws), lambda: call(c, 0, q.float(), s, off, 2, goff, 4, ws),
        lambda: call(c, 0, q, s, off[:2], 2, goff, 4, ws), lambda: call(c, 0, q, s, off, 2, goff.long(), 4, ws),
        lambda: call(c, 0, q, s, off, 2, goff[:0], 4, ws), lambda: call(c, 0, q, s, off, 2, goff[:1], 4, ws),
        lambda: call(c, 0, q, s, off, 2, dev(list(range(c.max_seqs + 2))), 4, ws), lambda: call(c, 0, q, s, off, 2, goff, -1, ws),
        lambda: call(c, 0, q, s, off, 2, goff, 4, c.ws[:-256] if c.ws.numel() > ws.numel() else c.alloc_workspace()[:256]),
        lambda: call(c, 0, torch.ones((400, 2, 64), device="cuda").bfloat16(), s, off, 2, goff, 4, ws),  # more rows than it was made for
        lambda: call(c, 0, q, s, off, 2, goff, 4, ws, scale=math.nan), lambda: call(c, 0, q, s, off, 2, goff, 4, ws, out=q[:1]),
        lambda: call(c, 0, q, s, off, 2, goff, 4, None and ws or torch.zeros(10, device="cuda")),
    ):
        with pytest.raises(occ.OccamError):
            f()
