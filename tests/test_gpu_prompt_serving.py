"""Whole-prompt attention, append with the rotation, forks and attention over shared pages together, as a server
runs them, and the forward and backward pass of a layer's attention, as a trainer does; tensors past 32 bits of
offsets. Bounds as in the operators' own tests."""

from __future__ import annotations

import pytest
import torch

import cache_reference as R
import prompt_reference as P
from test_gpu_append_rope import case, close
from test_gpu_cache import dev, make, offs

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f16": torch.float16}
I64 = torch.int64


def near_cache(c, layer, q, seqs, off, out, lse):
    want, wlse, tol, ltol = R.Cache(c).attend(layer, q, seqs, off)
    u = R.UNIT[q.dtype]
    # (the join of two parts: 2^-9 of attention's bound, see test_gpu_attend_shared)
    tol = tol * (1 + 2.0 ** -9 + 2.0 ** -9 * wlse.abs()[..., None])
    assert bool(((out.double().cpu() - want).abs() <= u * want.abs() + R.TINY[q.dtype] + (1 + u) * tol).all())
    assert bool(((lse.double().cpu() - wlse).abs() <= ltol + 2.0 ** -20 + 2.0 ** -21 * wlse.abs()).all())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("T,dim,hkv,G,prompts,forks", [(64, 128, 2, 4, [150, 70, 301], 3), (16, 64, 4, 1, [33, 100], 2),
                                                       (32, 128, 1, 8, [900], 20)])
def test_prompts_enter_fork_and_answer(T, dim, hkv, G, prompts, forks, dtype):
    """Prompts in two chunks (the second attends to both), into the cache, forked, a question each, then single tokens by a
    captured step."""
    import paper_2605_29657_gb300 as occ
    layers, hq, n, steps = 2, hkv * G, len(prompts), 3
    branches = n * forks
    questions = [1 + 3 * i % 7 for i in range(branches)]
    most = max(prompts) + max(questions) + steps + 1
    c = make(layers=layers, heads=hkv, dim=dim, T=T, seqs=n + branches, max_pages=-(-most // T),
             pages=sum(-(-p // T) for p in prompts) + branches * (2 + (max(questions) + steps) // T))
    seqs, off = list(range(n)), offs(prompts)
    first = [p // 2 for p in prompts]
    q, k, v, pos, freq, axis = case(off[-1], hq, hkv, dim, dim, 3, dtype, 1)
    ws = occ.alloc_prompt_workspace(off[-1], hq, off[-1], hkv)
    cws = c.alloc_workspace(sum(questions), hq)
    occ.occam_cache_extend(c, dev(seqs), dev(prompts))
    for layer in range(layers):
        tq, tk = occ.occam_rope(q, k, pos, freq, axis)
        # chunk by chunk: the rows of the first half over their own keys, of the second over all
        a = torch.cat([torch.arange(off[i], off[i] + first[i]) for i in range(n)]).cuda()
        b = torch.cat([torch.arange(off[i] + first[i], off[i + 1]) for i in range(n)]).cuda()
        oa, ob = offs(first), offs([p - f for p, f in zip(prompts, first)])
        out1, lse1 = occ.occam_prompt_attend(tq[a], tk[a], v[a], dev(oa, I64), ws)
        out2, lse2 = occ.occam_prompt_attend(tq[b], tk, v, dev(ob, I64), ws, key_off=dev(off, I64))
        want, wlse, tol, ltol = P.attend(tq, tk, v, off)
        for rows, out, lse in ((a, out1, lse1), (b, out2, lse2)):
            P.assert_near(out, want[rows], tol[rows], q.dtype, "out")
            P.assert_near(lse, wlse[rows], ltol[rows], torch.float32, "lse")
        eq = occ.occam_cache_append_rope(c, layer, q, k, v, dev(seqs), dev(off, I64), pos, freq, axis)
        assert torch.equal(eq, tq)
    assert occ.occam_get_status(ws) == 0 and c.status() == 0
    kids = list(range(n, n + branches))
    occ.occam_cache_fork(c, dev([i for i in range(n) for _ in range(forks)]), dev(kids))
    goff = dev([i * forks for i in range(n + 1)])

    def answer(rows, seed):
        """A captured or eager step's tensors."""
        o = offs(rows)
        q, k, v, pos, _, _ = case(o[-1], hq, hkv, dim, dim, 3, dtype, seed)
        return [x.contiguous() for x in (q, k, v, pos)], o

    def run(x, rows, o, out, lse, eq):
        occ.occam_cache_extend(c, ids, dev(rows) if counts is None else counts, ws=cws)
        for layer in range(layers):
            occ.occam_cache_append_rope(c, layer, *x[:3], ids, o, x[3], freq, axis, out_q=eq, ws=cws)
            occ.occam_cache_attend_shared(c, layer, eq, ids, o, max(rows), goff, max(rows) * forks, cws, out=out[layer], lse=lse[layer])

    ids, counts = dev(kids), None
    x, o = answer(questions, 2)
    out, lse, eq = [torch.empty_like(x[0]) for _ in range(layers)], [torch.empty(x[0].shape[:2], device="cuda") for _ in range(layers)], torch.empty_like(x[0])
    run(x, questions, dev(o, I64), out, lse, eq)
    assert c.status(ws=cws) == 0
    for layer in range(layers):
        close(eq, x[0], x[3], freq, axis, "half", False)
        near_cache(c, layer, eq, kids, o, out[layer], lse[layer])
    rows = [1] * branches
    counts = dev(rows)
    x, o = answer(rows, 3)
    out, lse, eq = [torch.empty_like(x[0]) for _ in range(layers)], [torch.empty(x[0].shape[:2], device="cuda") for _ in range(layers)], torch.empty_like(x[0])
    od = dev(o, I64)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(x, rows, od, out, lse, eq)
    for step in range(steps):
        for to, y in zip(x, answer(rows, 10 + step)[0]):
            to.copy_(y)
        graph.replay()
        assert c.status(ws=cws) == 0
        assert c.length[kids].tolist() == [p + questions[i * forks + j] + step + 1 for i, p in enumerate(prompts) for j in range(forks)]
        for layer in range(layers):
            near_cache(c, layer, eq, kids, o, out[layer], lse[layer])
    occ.occam_cache_release(c, dev(kids + seqs))
    assert c.status() == 0 and int(c.refs.sum()) == 0


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_a_layer_s_attention_and_its_gradient(dtype):
    """Rotation, attention, its gradient and the rotation's, eager and captured: the graph's gradients are the eager ones."""
    import paper_2605_29657_gb300 as occ
    rows, H, Hkv, D = [70, 1, 200], 8, 2, 64
    off = offs(rows)
    q, k, v, pos, freq, axis = case(off[-1], H, Hkv, D, D, 3, dtype, 5, 0.5)
    dout = (0.1 * torch.randn(q.shape, generator=torch.Generator().manual_seed(6))).to(q.dtype).cuda()
    ws = occ.alloc_prompt_workspace(off[-1], H, off[-1], Hkv)
    do = dev(off, I64)
    grad_of = torch.empty((off[-1], H + 2 * Hkv, D), dtype=q.dtype, device="cuda")  # of the projection

    def step():
        tq, tk = occ.occam_rope(q, k, pos, freq, axis)
        out, lse = occ.occam_prompt_attend(tq, tk, v, do, ws)
        dq, dk, dv = grad_of.split((H, Hkv, Hkv), 1)
        occ.occam_prompt_attend_grad(tq, tk, v, out, lse, dout, do, ws, dq=dq, dk=dk, dv=dv)
        turned = grad_of.clone()
        occ.occam_rope(dq, dk, pos, freq, axis, inverse=True, out_q=dq, out_k=dk)
        return tq, tk, out, turned

    tq, tk, out, turned = step()
    eager = grad_of.clone()
    assert occ.occam_get_status(ws) == 0
    want = P.grad(tq, tk, v, dout, off)
    for x, w, t in zip(turned.split((H, Hkv, Hkv), 1), want[:3], want[3:]):
        P.assert_near(x, w, t, q.dtype)
    for x, y in zip(eager.split((H, Hkv, Hkv), 1)[:2], turned.split((H, Hkv, Hkv), 1)):
        close(x, y, pos, freq, axis, "half", True)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        kept = step()
    for _ in range(2):
        grad_of.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(grad_of, eager) and torch.equal(kept[2], out)


def test_rows_far_apart():
    """Rows 2^28 bytes apart: elements past 2^31 of q, k, v and of every result of the gradient."""
    import paper_2605_29657_gb300 as occ
    n, H, Hkv, D, stride = 20, 4, 2, 64, 1 << 27
    g = torch.Generator(device="cuda").manual_seed(3)

    def far(heads):
        x = torch.empty(n * stride, dtype=torch.bfloat16, device="cuda")
        return x.as_strided((n, heads, D), (stride, D, 1))

    whole, into = far(H + 2 * Hkv), far(H + 2 * Hkv)
    whole.copy_(torch.randn(whole.shape, generator=g, device="cuda"))
    into.fill_(7.0)
    q, k, v = whole.split((H, Hkv, Hkv), 1)
    dq, dk, dv = into.split((H, Hkv, Hkv), 1)
    off = dev([0, 7, 20], I64)
    dout = 0.1 * torch.randn((n, H, D), generator=g, device="cuda").bfloat16()
    ws = occ.alloc_prompt_workspace(n, H, n, Hkv)
    near = [x.contiguous() for x in (q, k, v)]
    res = []
    for a in ((q, k, v), near):
        out, lse = occ.occam_prompt_attend(*a, off, ws)
        res.append((out, lse))
    assert torch.equal(res[0][0], res[1][0]) and torch.equal(res[0][1], res[1][1])
    occ.occam_prompt_attend_grad(q, k, v, *res[0], dout, off, ws, dq=dq, dk=dk, dv=dv)
    want = occ.occam_prompt_attend_grad(*near, *res[1], dout, off, ws)
    assert occ.occam_get_status(ws) == 0
    for x, y in zip((dq, dk, dv), want):
        assert torch.equal(x, y)


def test_results_past_32_bits():
    """4,200 sequences of 64 rows of 64 heads: 2.2 G elements in q, out and dq; the last sequences by themselves."""
    import paper_2605_29657_gb300 as occ
    n, r, H, Hkv, D = 4200, 64, 64, 8, 128
    g = torch.Generator(device="cuda").manual_seed(4)
    normal = lambda h: torch.randn((n * r, h, D), generator=g, device="cuda", dtype=torch.bfloat16)
    q, k, v, dout = normal(H), normal(Hkv), normal(Hkv), normal(H)
    assert q.numel() > 1 << 31
    ws = occ.alloc_prompt_workspace(n * r, H, n * r, Hkv)
    off = torch.arange(0, n * r + 1, r, device="cuda")
    out, lse = occ.occam_prompt_attend(q, k, v, off, ws)
    got = occ.occam_prompt_attend_grad(q, k, v, out, lse, dout, off, ws)
    assert occ.occam_get_status(ws) == 0
    a, o = slice((n - 2) * r, n * r), [0, r, 2 * r]
    want, wlse, tol, ltol = P.attend(q[a], k[a], v[a], o)
    P.assert_near(out[a], want, tol, q.dtype)
    P.assert_near(lse[a], wlse, ltol, torch.float32)
    want = P.grad(q[a], k[a], v[a], dout[a], o)
    for x, w, t in zip(got, want[:3], want[3:]):
        P.assert_near(x[a], w, t, q.dtype)


def test_pool_past_32_bits():
    """A pool of more than 2^32 codes a tensor: rotated appends to, and shared pages among, the pages at its end."""
    import paper_2605_29657_gb300 as occ
    pages = (1 << 32) // (2 * 128 * 128) + 50
    c = occ.PagedCache(1, pages, 2, 128, 6, 9, page_tokens=128)
    c.refs[:pages - 14] = 1
    small = make(layers=1, pages=14, heads=2, dim=128, T=128, seqs=6, max_pages=9)
    q, k, v, pos, freq, axis = case(900, 4, 2, 128, 128, 3, "bf16", 7)
    got = []
    for cc in (c, small):
        ws = cc.alloc_workspace(900, 4)
        occ.occam_cache_extend(cc, dev([0]), dev([900]))
        res = [occ.occam_cache_append_rope(cc, 0, q, k, v, dev([0]), dev([0, 900], I64), pos, freq, axis)]
        kids = [1, 2, 3, 4]
        occ.occam_cache_fork(cc, dev([0] * 4), dev(kids))
        occ.occam_cache_extend(cc, dev(kids), dev([3] * 4))
        res.append(occ.occam_cache_append_rope(cc, 0, q[:12], k[:12], v[:12], dev(kids), dev([0, 3, 6, 9, 12], I64), pos[:, :12], freq, axis))
        for a in (1, 3):
            off = dev([a * i for i in range(5)], I64)
            res += occ.occam_cache_attend_shared(cc, 0, q[:4 * a], dev(kids), off, a, dev([0, 4]), 4 * a, ws)
        assert cc.status() == 0 and cc.status(ws=ws) == 0
        got.append(res)
    assert int(c.table.max()) >= pages - 14
    for a, b in zip(*got):
        assert torch.equal(a, b)
