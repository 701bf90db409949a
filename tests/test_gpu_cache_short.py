"""Attention over the cache for many short sequences with 33 to 128 query rows a key head: one row tile, one or two key tiles
an item, several items a CTA, between items of two row tiles."""

from __future__ import annotations

import pytest
import torch

import cache_reference as R
from test_gpu_cache import attend_case, filled

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lo,hi,rows_lo,rows_hi", [(30, 150, 9, 32), (40, 260, 16, 70), (33, 64, 33, 33)])
def test_attend_many_short_items(lo, hi, rows_lo, rows_hi):
    import paper_2605_29657_gb300 as occ
    g = torch.Generator().manual_seed(lo)
    n = 64
    rows = torch.randint(rows_lo, rows_hi + 1, (n,), generator=g).tolist()
    lengths = [max(r, int(x)) for r, x in zip(rows, torch.randint(lo, hi + 1, (n,), generator=g))]
    c, seqs = filled(64, 128, 8, lengths, 3)
    q = torch.randn((sum(rows), 32, 128), generator=g).bfloat16().cuda()
    off = [0]
    for r in rows:
        off.append(off[-1] + r)
    s, o = torch.tensor(seqs, dtype=torch.int32, device="cuda"), torch.tensor(off, device="cuda")
    want, wlse, tol, ltol = R.Cache(c).attend(0, q, seqs, off)
    for _ in range(20):
        out, lse = occ.occam_cache_attend(c, 0, q, s, o, rows_hi)
        assert c.status() == 0
        assert bool(((lse.double().cpu() - wlse).abs() <= ltol).all())
        u = R.UNIT[q.dtype]
        assert bool(((out.double().cpu() - want).abs() <= u * want.abs() + R.TINY[q.dtype] + (1 + u) * tol).all())


def test_attend_nan_notes_of_short_items():
    """NaN values in many short items of a CTA: each counts for the rows of its own item that see it."""
    n = 48
    lengths = [40 + 3 * i % 90 for i in range(n)]
    rows = [20 + i % 12 if i % 3 else 40 for i in range(n)]
    lengths = [max(a, b) for a, b in zip(lengths, rows)]
    c, seqs = filled(16, 64, 4, lengths, 5)
    for i in range(0, n, 2):
        p = lengths[i] - 5
        c.v.view(torch.uint8)[0, int(c.table[seqs[i], p // 16]), i % 4, p % 16, i] = 0x7f
    for _ in range(5):
        attend_case(c, seqs, rows, 16)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("length", [256, 1500])
def test_attend_results_are_the_same_each_time(dim, length):
    """100 rows of 16 heads over 4 key heads: items of two row tiles, whose products take most of the shared memory's reads
    while the next pages come in. The results depend on no timing, and are those of the kernel for few rows to f16's and
    the result's roundings (2^-8 relative at most where nothing cancels; a tenth of a row's largest value is far off)."""
    import paper_2605_29657_gb300 as occ
    g = torch.Generator().manual_seed(dim + length)
    n, rows = 8, 100
    c, seqs = filled(64, dim, 4, [length] * n, 7)
    q = (0.2 * torch.randn((n * rows, 64, dim), generator=g)).bfloat16().cuda()
    s, off = torch.tensor(seqs, dtype=torch.int32, device="cuda"), torch.arange(0, n * rows + 1, rows, device="cuda")
    few, few_lse = occ.occam_cache_attend(c, 0, q, s, off, 1)
    first, first_lse = occ.occam_cache_attend(c, 0, q, s, off, rows)
    assert bool(((first.float() - few.float()).abs().amax(-1) <= 0.1 * few.float().abs().amax(-1)).all())
    assert bool(((first_lse - few_lse).abs() <= 0.01).all())
    for _ in range(60):
        out, lse = occ.occam_cache_attend(c, 0, q, s, off, rows)
        assert torch.equal(out, first) and torch.equal(lse, first_lse)
    assert c.status() == 0
