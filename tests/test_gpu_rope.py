"""occam_rope against its definition in 64 bits.

Bound: the angle's product carries its rounding error along, so a value is off
by the fp32 sine and cosine (2 ulp each) and three fp32 operations: 2^-21 (|a|
+ |b|), then half an ulp of the output's type."""

from __future__ import annotations

import pytest
import torch

import cache_reference as R

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def case(rows, hq, hk, dim, rot, axes, dtype, seed=0, max_pos=4000, fused=False):
    g = torch.Generator().manual_seed(seed)
    if fused:
        qkv = torch.randn((rows, hq + 2 * hk, dim), generator=g).to(DT[dtype]).cuda()
        q, k = qkv[:, :hq], qkv[:, hq:hq + hk]
    else:
        q = torch.randn((rows, hq, dim), generator=g).to(DT[dtype]).cuda()
        k = torch.randn((rows, hk, dim), generator=g).to(DT[dtype]).cuda()
    pos = torch.randint(0, max_pos, (axes, rows), generator=g, dtype=torch.int32).cuda()
    freq = (10000.0 ** (-torch.arange(rot // 2).double() * 2 / rot)).float().cuda()
    axis = torch.randint(0, axes, (rot // 2,), generator=g, dtype=torch.int32).cuda()
    return q, k, pos, freq, axis


def close(got, x, pos, freq, axis, pairing, inverse):
    want, mag = R.rope(x, pos, freq, axis, pairing, inverse)
    err = (got.double().cpu() - want).abs()
    u = R.UNIT[got.dtype]
    bound = u * want.abs() + R.TINY[got.dtype] + (1 + u) * 2.0 ** -21 * mag
    assert bool((err <= bound).all()), float((err - bound).max())


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("pairing", ["half", "adjacent"])
@pytest.mark.parametrize("rows,hq,hk,dim,rot", [
    (1, 32, 8, 128, 128), (33, 16, 16, 72, 72), (7, 3, 1, 80, 40), (257, 5, 5, 64, 64), (19, 1, 1, 6, 2),
    (12, 2, 1, 70, 30), (300, 28, 4, 128, 64), (3, 1, 2, 2, 2)])
def test_rope(dtype, pairing, rows, hq, hk, dim, rot):
    import paper_2605_29657_gb300 as occ
    for fused in (False, True):
        for inverse in (False, True):
            q, k, pos, freq, axis = case(rows, hq, hk, dim, rot, 3, dtype, fused=fused)
            a, b = occ.occam_rope(q, k, pos, freq, axis, pairing=pairing, inverse=inverse)
            close(a, q, pos, freq, axis, pairing, inverse)
            close(b, k, pos, freq, axis, pairing, inverse)


def test_large_positions_and_many_rows():
    import paper_2605_29657_gb300 as occ
    q, k, pos, freq, axis = case(9001, 8, 2, 128, 128, 3, "f32", max_pos=1 << 20)
    a, b = occ.occam_rope(q, k, pos, freq, axis)
    close(a, q, pos, freq, axis, "half", False)
    close(b, k, pos, freq, axis, "half", False)


def test_in_place_queries_alone_and_odd_addresses():
    import paper_2605_29657_gb300 as occ
    q, k, pos, freq, axis = case(65, 6, 2, 128, 96, 2, "bf16")
    want, _ = occ.occam_rope(q, k, pos, freq, axis)
    mine = q.clone()
    got, none = occ.occam_rope(mine, None, pos, freq, axis, out_q=mine)
    assert none is None and got.data_ptr() == mine.data_ptr()
    assert torch.equal(got, want)
    # the same values at an address that is a multiple of 2 bytes only, rows of odd size
    wide = torch.zeros((65, 6, 131), dtype=torch.bfloat16, device="cuda")
    wide[..., 1:129] = q
    odd, _ = occ.occam_rope(wide[..., 1:129], None, pos, freq, axis)
    assert torch.equal(odd, want)
    # positions that are a view of a wider tensor
    both = torch.cat([pos, pos], 1)
    again, _ = occ.occam_rope(q, None, both[:, :65], freq, axis)
    assert torch.equal(again, want)


def test_gradient():
    """The inverse map is the gradient: against autograd of the definition, and against differences."""
    import paper_2605_29657_gb300 as occ
    q, _, pos, freq, axis = case(11, 4, 1, 64, 48, 2, "f32", max_pos=50)
    gy = torch.randn(q.shape, generator=torch.Generator().manual_seed(5)).cuda()
    for pairing in ("half", "adjacent"):
        gx, _ = occ.occam_rope(gy, None, pos, freq, axis, pairing=pairing, inverse=True)
        x = q.double().cpu().requires_grad_(True)
        half = freq.numel()
        t = pos.cpu().double()[axis.cpu().long()].T * freq.cpu().double()
        c, s = torch.cos(t)[:, None], torch.sin(t)[:, None]
        if pairing == "half":
            a, b = x[..., :half], x[..., half:2 * half]
            y = torch.cat([a * c - b * s, b * c + a * s, x[..., 2 * half:]], -1)
        else:
            a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
            y = torch.cat([torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2), x[..., 2 * half:]], -1)
        (y * gy.double().cpu()).sum().backward()
        _, mag = R.rope(gy, pos, freq, axis, pairing, True)
        assert bool(((gx.double().cpu() - x.grad).abs() <= 2.0 ** -21 * mag + 2.0 ** -23 * x.grad.abs()).all())
        # differences of the kernel's own forward: it is linear, so one step of 1 is exact up to rounding
        for n, h, d in ((0, 0, 0), (5, 3, 47), (10, 1, 50), (3, 2, 23)):
            e = torch.zeros_like(q)
            e[n, h, d] = 1.0
            up, _ = occ.occam_rope(e, None, pos, freq, axis, pairing=pairing)
            diff = float((up.double() * gy.double()).sum())
            assert abs(diff - float(gx[n, h, d])) <= 2.0 ** -20 * (float(gy[n, h].abs().sum()) + 1)


def test_axis_outside_reads_axis_zero_and_empty_call():
    import paper_2605_29657_gb300 as occ
    q, k, pos, freq, axis = case(5, 2, 1, 64, 64, 2, "f32")
    zero = torch.zeros_like(axis)
    want, _ = occ.occam_rope(q, k, pos, freq, zero)
    wild = torch.where(torch.arange(32, device="cuda") % 2 == 0, 7, -3).int()
    got, _ = occ.occam_rope(q, k, pos, freq, wild)
    assert torch.equal(got, want)
    a, b = occ.occam_rope(q[:0], k[:0], pos[:, :0], freq, axis)
    assert a.shape == (0, 2, 64) and b.shape == (0, 1, 64)


def test_rope_axes():
    import paper_2605_29657_gb300 as occ
    assert occ.rope_axes((2, 1, 1)).tolist() == [0, 0, 1, 2]
    assert occ.rope_axes((3, 2, 2), interleaved=True).tolist() == [0, 1, 2, 0, 1, 2, 0]
    with pytest.raises(occ.OccamError):
        occ.rope_axes((1, 4), interleaved=True)


def test_refusals():
    import paper_2605_29657_gb300 as occ
    q, k, pos, freq, axis = case(5, 2, 1, 64, 64, 2, "f32")
    bad = [
        lambda: occ.occam_rope(q.cpu(), k, pos, freq, axis),
        lambda: occ.occam_rope(q, k.bfloat16(), pos, freq, axis),
        lambda: occ.occam_rope(q, k[:4], pos, freq, axis),
        lambda: occ.occam_rope(q, k, pos.long(), freq, axis),
        lambda: occ.occam_rope(q, k, pos[:, :4], freq, axis),
        lambda: occ.occam_rope(q, k, pos, freq.double(), axis),
        lambda: occ.occam_rope(q, k, pos, freq, axis[:3]),
        lambda: occ.occam_rope(q, k, pos, torch.ones(33, device="cuda"), torch.zeros(33, dtype=torch.int32, device="cuda")),
        lambda: occ.occam_rope(q, k, pos, freq, axis, pairing="other"),
        lambda: occ.occam_rope(q.transpose(1, 2), k, pos, freq, axis),
        lambda: occ.occam_rope(q, k, torch.zeros((9, 5), dtype=torch.int32, device="cuda"), freq, axis),
    ]
    for f in bad:
        with pytest.raises(occ.OccamError):
            f()


def test_results_in_every_layout_that_does_not_overlap():
    """In place on views of one projection, heads outside rows, rows between the heads of another tensor, results in the
    gaps of the input: all give what new dense tensors get."""
    import paper_2605_29657_gb300 as occ
    rows, hq, hk, dim = 33, 4, 2, 64
    q, k, pos, freq, axis = case(rows, hq, hk, dim, dim, 2, "bf16")
    want_q, want_k = occ.occam_rope(q, k, pos, freq, axis)

    def empty(*shape):
        return torch.zeros(shape, dtype=torch.bfloat16, device="cuda")

    def check(q, k, out_q, out_k):
        a, b = occ.occam_rope(q, k, pos, freq, axis, out_q=out_q, out_k=out_k)
        assert a is out_q and b is out_k and torch.equal(a, want_q) and torch.equal(b, want_k)

    fused = empty(rows, hq + 2 * hk, dim)
    fused[:, :hq], fused[:, hq:hq + hk] = q, k
    check(fused[:, :hq], fused[:, hq:hq + hk], fused[:, :hq], fused[:, hq:hq + hk])
    fused[:, :hq], fused[:, hq:hq + hk] = q, k  # keys in place of the values' rows, queries in place
    check(fused[:, :hq], fused[:, hq:hq + hk], fused[:, :hq], fused[:, hq + hk:])
    both = empty(hq + hk, rows, dim)
    check(q, k, both[:hq].transpose(0, 1), both[hq:].transpose(0, 1))
    woven = empty(rows, 2 * hq, dim)
    check(q, k, woven[:, ::2], woven[:, 1:2 * hk:2])
    woven[:, ::2] = q
    check(woven[:, ::2], k, woven[:, 1::2], empty(rows, hk, dim))
    apart = empty(2 * hq, rows, dim).transpose(0, 1)  # heads outside rows, other head strides
    apart[:, ::2] = q
    check(apart[:, ::2], k, apart[:, 1::2], apart[:, 0:2 * hk:2].clone())
    odd = empty(rows * 3 * dim + hq * 100 * dim)  # rows 3 and heads 34 widths apart: rows and heads cross, and no two meet
    out = torch.as_strided(odd, (rows, hq, dim), (3 * dim, 34 * dim, 1))
    check(q, k, out, empty(rows, hk, dim))


def test_overlapping_results_are_refused():
    import paper_2605_29657_gb300 as occ
    q, k, pos, freq, axis = case(5, 4, 2, 64, 64, 2, "bf16")
    buf = torch.zeros(4096, dtype=torch.bfloat16, device="cuda")
    rows = torch.zeros((6, 6, 64), dtype=torch.bfloat16, device="cuda")
    for kw in (dict(out_q=torch.as_strided(buf, (5, 4, 64), (64, 64, 1))), dict(out_q=rows[:5, :4], out_k=rows[:5, 3:5]),
               dict(out_q=rows[:5, :4], out_k=rows[1:, :2])):
        with pytest.raises(occ.OccamError):
            occ.occam_rope(q, k, pos, freq, axis, **kw)
    with pytest.raises(occ.OccamError):
        occ.occam_rope(rows[:5, :4], k, pos, freq, axis, out_q=rows[1:, :4])
    with pytest.raises(occ.OccamError):
        occ.occam_rope(rows[:5, :4], rows[:5, 4:], pos, freq, axis, out_q=rows[:5, 2:])
    assert not rows.any() and not buf.any()
