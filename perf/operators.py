"""Measured cases of the operators that take a pruned prefix into decoding.

Pruning leaves a ragged prefix of kept rows. What a serving program does with
it next: turn the queries and keys by their (time, height, width) positions
(``rope``), put the keys and values into a paged cache held in 8 bits with one
scale per block of tokens and head (``append``), attend over that cache from
single tokens, questions and long prefixes (``attend``), and manage the
cache's pages: share a prefix between questions, prune a shared prefix, drop it
(``pages``).

``run`` with ``own`` false is the plain form of each operator, in elementary
torch operations and 32 bits; with ``own`` true it makes the calls of the
framework. Sizes are those of this repository's workloads: 576 + 4 rows per
crop, five crops a sample, 1024 + 4 rows per frame, 16 frames a video, 16 to
512 text tokens, 32 query heads, 32 or 8 key heads, 128 dims, vision heads of
72 and 80 dims.
"""

from __future__ import annotations

import math

import torch

own = False

E4M3 = torch.float8_e4m3fn
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
DEV = "cuda"


# ------------------------------------------------------------------ cases

def listed():
    return [
        # one new token of each of 64 conversations: latency of a decode step
        dict(name="rope_step_b64", op="rope", rows=64, hq=32, hk=8, dim=128, rot=128, axes=3, interleaved=True,
             pairing="half", dtype="bf16", inverse=False, max_pos=20000, fused_qkv=True),
        # all rows of a batch of four 16-frame videos, one key head per query head
        dict(name="rope_video_b4", op="rope", rows=65792, hq=32, hk=32, dim=128, rot=128, axes=3, interleaved=False,
             pairing="half", dtype="bf16", inverse=False, max_pos=20000, fused_qkv=False),
        # gradient through the two-axis rotary of a vision tower: 16 heads of 72 dims, ragged images
        dict(name="rope_vision_grad", op="rope", rows=34813, hq=16, hk=16, dim=72, rot=72, axes=2, interleaved=False,
             pairing="half", dtype="f32", inverse=True, max_pos=64, fused_qkv=True),
        # one token a conversation, written into half-filled pages
        dict(name="append_step_b64", op="append", seqs=64, rows_lo=1, rows_hi=1, len_lo=200, len_hi=4096, heads=8,
             dim=128, page=64, dtype="bf16"),
        # the kept rows of a pruned batch of 64 (about 160 visual + 20 registers + 16..256 text tokens each)
        dict(name="append_prompt_b64", op="append", seqs=64, rows_lo=196, rows_hi=436, len_lo=0, len_hi=40, heads=32,
             dim=128, page=64, dtype="bf16"),
        # one image, one conversation, one token: the smallest call
        dict(name="attend_step_b1", op="attend", seqs=1, rows_lo=1, rows_hi=1, len_lo=612, len_hi=612, hq=32, hkv=8,
             dim=128, page=64, dtype="bf16", masked=False),
        # decode step of 64 conversations over ragged, grouped-query caches
        dict(name="attend_step_b64", op="attend", seqs=64, rows_lo=1, rows_hi=1, len_lo=256, len_hi=4608, hq=32, hkv=8,
             dim=128, page=64, dtype="bf16", masked=False),
        # decode step over four unpruned videos, one key head per query head, small pages
        dict(name="attend_video_b4", op="attend", seqs=4, rows_lo=1, rows_hi=1, len_lo=16448, len_hi=16704, hq=32,
             hkv=32, dim=128, page=32, dtype="f16", masked=False),
        # 32 questions of 32..512 tokens against cached images, visual tokens outside S2 masked
        dict(name="attend_questions_b32", op="attend", seqs=32, rows_lo=32, rows_hi=512, len_lo=768, len_hi=4608,
             hq=32, hkv=8, dim=128, page=64, dtype="bf16", masked=True),
        # a long prefix attending to itself
        dict(name="attend_prefill_8k", op="attend", seqs=1, rows_lo=8257, rows_hi=8257, len_lo=8257, len_hi=8257,
             hq=32, hkv=8, dim=128, page=64, dtype="bf16", masked=False),
        # eight continuations of each of four cached prefixes, 1..64 new tokens each: latency of the page bookkeeping
        dict(name="pages_branch_b4", op="pages", kind="branch", parents=4, children=8, len_lo=200, len_hi=1500,
             layers=10, heads=8, dim=128, page=64, keep=0.0),
        # a second question on each of eight cached 5-crop images: fork the prefix, keep its S2 rows in 11 layers
        dict(name="pages_prune_b8", op="pages", kind="prune", parents=8, children=1, len_lo=2916, len_hi=3156,
             layers=11, heads=32, dim=128, page=64, keep=0.085),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "append", "attend", "attend", "pages"])
    if op == "rope":
        axes = rng.choice([1, 2, 3])
        dim = rng.choice([64, 72, 80, 128])
        rot = dim if rng.random() < 0.6 else dim // 2
        hq, hk = rng.choice([(16, 16), (32, 8), (32, 32), (28, 4), (5, 1)])
        return dict(op="rope", rows=_log_int(rng, 1, 30000), hq=hq, hk=hk, dim=dim, rot=rot, axes=axes,
                    interleaved=rng.random() < 0.5, pairing=rng.choice(["half", "adjacent"]),
                    dtype=rng.choice(["bf16", "f16", "f32"]), inverse=rng.random() < 0.4, max_pos=_log_int(rng, 32, 1000),
                    fused_qkv=rng.random() < 0.5)
    if op == "append":
        lo = _log_int(rng, 1, 150)
        return dict(op="append", seqs=_log_int(rng, 1, 64), rows_lo=lo, rows_hi=lo + rng.randint(0, lo), len_lo=0,
                    len_hi=_log_int(rng, 1, 3000), heads=rng.choice([1, 4, 8, 32]), dim=rng.choice([64, 128]),
                    page=rng.choice([16, 32, 64, 128]), dtype=rng.choice(["bf16", "f16"]))
    if op == "attend":
        hq, hkv = rng.choice([(32, 8), (32, 32), (28, 4), (16, 16), (12, 2), (8, 1)])
        form = rng.choice(["step", "step", "question", "prefix"])
        if form == "step":
            rows, seqs, hi = (1, rng.choice([1, 1, 1, 4])), _log_int(rng, 1, 48), _log_int(rng, 64, 6000)
        elif form == "question":
            r = _log_int(rng, 2, 200)
            rows, seqs, hi = (r, 2 * r), _log_int(rng, 1, 16), _log_int(rng, 64, 3500)
        else:
            r = _log_int(rng, 300, 3500)
            rows, seqs, hi = (r, r + rng.randint(0, 500)), rng.randint(1, 2), r
        lo = max(rows[1], hi // rng.choice([1, 2, 8]))
        return dict(op="attend", seqs=seqs, rows_lo=rows[0], rows_hi=rows[1], len_lo=lo, len_hi=max(lo, hi), hq=hq,
                    hkv=hkv, dim=rng.choice([64, 128, 128]), page=rng.choice([16, 32, 64, 128]),
                    dtype=rng.choice(["bf16", "f16"]), masked=rng.random() < 0.4)
    kind = rng.choice(["branch", "prune"])
    lo, keep = _log_int(rng, 20, 1500), rng.choice([0.03, 0.1, 0.3, 0.9])
    return dict(op="pages", kind=kind, parents=rng.randint(1, 8 if keep < 0.2 else 2), children=rng.randint(1, 8) if kind == "branch" else 1,
                len_lo=lo, len_hi=lo + rng.randint(0, lo // 2), layers=rng.randint(1, 11), heads=rng.choice([1, 8, 32]),
                dim=rng.choice([64, 128]), page=rng.choice([16, 32, 64, 128]),
                keep=0.0 if kind == "branch" else keep)


# ------------------------------------------------------------------ quantisation of a block, in elementary operations

def _pow2_scale(amax):
    """The smallest power of two s, 2^-100 at least, with amax <= 448 s."""
    bits = amax.contiguous().view(torch.int32)
    e = (bits >> 23) - 135 + ((bits & 0x7FFFFF) > 0x600000).int()
    return (e.clamp(-100, 120) + 127).bitwise_left_shift(23).view(torch.float32)


def _fill_blocks(shape, g, gain):
    """Random codes and scales of cache blocks [P, H, T, D], quantised from normal values."""
    x = torch.randn(shape, device=DEV, generator=g) * gain
    s = _pow2_scale(x.abs().amax((-1, -2)))
    return (x / s[..., None, None]).to(E4M3), s


# ------------------------------------------------------------------ inputs

def _lengths(lo, hi, n):
    """n ragged lengths in lo..hi, the same for every seed (they are the case's sizes), in no order."""
    g = torch.Generator().manual_seed(1000003 * lo + 101 * hi + n)
    return torch.randint(lo, hi + 1, (n,), generator=g, dtype=torch.int64)


def _cache(case, layers, lens, extra_pages, cpu, g, slots, spare_seqs=0, max_pages=None, gain=None):
    """A cache whose sequences (at table rows `slots`) hold lens tokens in shuffled pages; spare pages come last."""
    T, H, D = case["page"], case.get("heads", case.get("hkv")), case["dim"]
    per = [(int(x) + T - 1) // T for x in lens]
    used = sum(per)
    pages = used + extra_pages
    max_pages = max_pages or max(per + [1])
    S = len(lens) + spare_seqs
    table = torch.full((S, max_pages), -1, dtype=torch.int32)
    length = torch.zeros(S, dtype=torch.int32)
    perm = torch.randperm(used, generator=cpu).int()
    at = 0
    for s, n, x in zip(slots, per, lens):
        table[s, :n] = perm[at:at + n]
        length[s] = int(x)
        at += n
    refs = torch.zeros(pages, dtype=torch.int32)
    refs[:used] = 1
    k = torch.empty((layers, pages, H, T, D), dtype=E4M3, device=DEV)
    v = torch.empty_like(k)
    ks = torch.empty((layers, pages, H), device=DEV)
    vs = torch.empty_like(ks)
    for i in range(layers):
        k[i], ks[i] = _fill_blocks((pages, H, T, D), g, 1.0 if gain is None else gain)
        v[i], vs[i] = _fill_blocks((pages, H, T, D), g, torch.exp(0.5 * torch.randn((pages, H, 1, 1), device=DEV, generator=g)))
    return dict(k=k, v=v, k_scale=ks, v_scale=vs, table=table.to(DEV), length=length.to(DEV), refs=refs.to(DEV)), used


def prepare(case, seed):
    cpu = torch.Generator().manual_seed(seed)
    g = torch.Generator(device=DEV).manual_seed(seed)
    st = dict(case=case)
    if case["op"] == "rope":
        _prepare_rope(case, st, cpu, g)
        return st
    if case["op"] == "append":
        n = case["seqs"]
        rows = _lengths(case["rows_lo"], case["rows_hi"], n)
        had = _lengths(case["len_lo"], case["len_hi"], n)
        slots = torch.randperm(n, generator=cpu)
        st["cache"], _ = _cache(case, 2, (had + rows).tolist(), 3, cpu, g, slots.tolist())
        st["layer"] = 1
        total = int(rows.sum())
        gain = torch.exp(0.7 * torch.randn((1, case["heads"], case["dim"]), device=DEV, generator=g))
        burst = 1 + 7 * (torch.rand((total, 1, 1), device=DEV, generator=g) < 0.1).float()
        for name in ("k_new", "v_new"):
            st[name] = (torch.randn((total, case["heads"], case["dim"]), device=DEV, generator=g) * gain * burst).to(DTYPES[case["dtype"]])
    elif case["op"] == "attend":
        n = case["seqs"]
        rows = _lengths(case["rows_lo"], case["rows_hi"], n)
        lens = torch.maximum(_lengths(case["len_lo"], case["len_hi"], n), rows)
        slots = torch.randperm(n, generator=cpu)
        st["cache"], _ = _cache(case, 1, lens.tolist(), 2, cpu, g, slots.tolist())
        st["layer"] = 0
        total = int(rows.sum())
        st["q"] = (1.5 * torch.randn((total, case["hq"], case["dim"]), device=DEV, generator=g)).to(DTYPES[case["dtype"]])
        st["max_rows"], st["max_len"] = int(rows.max()), int(lens.max())
        st["keep"] = st["keep_off"] = None
        if case["masked"]:
            # the text (the last third, and the rows that ask) is kept, a quarter of the rest is
            off = torch.zeros(n + 1, dtype=torch.int64)
            off[1:] = lens.cumsum(0)
            pos = torch.arange(int(off[-1])) - torch.repeat_interleave(off[:-1], lens)
            text = pos >= torch.repeat_interleave(torch.minimum(lens * 2 // 3, lens - rows), lens)
            st["keep"] = (text | (torch.rand(pos.shape, generator=cpu) < 0.25)).to(torch.uint8).to(DEV)
            st["keep_off"] = off.to(DEV)
    else:
        _prepare_pages(case, st, cpu, g)
        return st
    off = torch.zeros(n + 1, dtype=torch.int64)
    off[1:] = rows.cumsum(0)
    st["seqs"] = slots.int().to(DEV)
    st["row_off"] = off.to(DEV)
    seq_of = torch.repeat_interleave(torch.arange(n), rows)
    st["row_seq"] = seq_of.to(DEV)
    st["row_j"] = (torch.arange(total) - off[seq_of]).to(DEV)
    _handle(st)
    return st


def _handle(st):
    if own:
        import paper_2605_29657_gb300 as occ

        st["handle"] = occ.PagedCache.wrap(**st["cache"])


def _prepare_rope(case, st, cpu, g):
    rows, hq, hk, D = case["rows"], case["hq"], case["hk"], case["dim"]
    dt = DTYPES[case["dtype"]]
    if case["fused_qkv"]:  # views of one projection's output [rows, hq + 2 hk, D]
        qkv = torch.randn((rows, hq + 2 * hk, D), device=DEV, generator=g).to(dt)
        st["q"], st["k"] = qkv[:, :hq], qkv[:, hq:hq + hk]
    else:
        st["q"] = torch.randn((rows, hq, D), device=DEV, generator=g).to(dt)
        st["k"] = torch.randn((rows, hk, D), device=DEV, generator=g).to(dt)
    half = case["rot"] // 2
    st["positions"] = torch.randint(0, case["max_pos"], (case["axes"], rows), generator=cpu, dtype=torch.int32).to(DEV)
    i = torch.arange(half)
    if case["interleaved"]:
        axis = i % case["axes"]
    else:
        axis = i * case["axes"] // half
    st["axis"] = axis.int().to(DEV)
    st["inv_freq"] = (10000.0 ** (-(2.0 * i.double()) / case["rot"])).float().to(DEV)


def _prepare_pages(case, st, cpu, g):
    n, c, T = case["parents"], case["children"], case["page"]
    lens = _lengths(case["len_lo"], case["len_hi"], n)
    nc = n * c
    per = max((int(x) + T - 1) // T for x in lens) + 64 // T + 1
    src = torch.arange(n).repeat_interleave(c)
    if case["kind"] == "branch":
        add = _lengths(1, 64, nc).int()
        # a partial last page of its own, and the pages of the new tokens
        new = sum(1 + (int(lens[s]) % T + int(a)) // T + 1 for s, a in zip(src, add))
        st["add"] = add.to(DEV)
    else:
        # the rows that pruning leaves: the first 35 (prompt), the last 64 (question), scattered ones between
        ln = lens[src].tolist()
        off = torch.zeros(nc + 1, dtype=torch.int64)
        off[1:] = lens[src].cumsum(0)
        keep = torch.zeros(int(off[-1]), dtype=torch.bool)
        for a, x in zip(off.tolist(), ln):
            keep[a:a + 35] = True
            keep[max(a, a + x - 64):a + x] = True
            mid = max(0, x - 99)
            keep[a + 35 + torch.randperm(mid, generator=cpu)[:round(case["keep"] * mid)]] = True
        new = sum(int(k.sum()) // T + 3 for k in keep.split(ln))
        st["keep"], st["keep_off"] = keep.to(torch.uint8).to(DEV), off.to(DEV)
    st["cache"], st["first_spare"] = _cache(case, case["layers"], lens.tolist(), new, cpu, g, list(range(n)),
                                            spare_seqs=nc, max_pages=per)
    st["src"] = src.int().to(DEV)
    st["dst"] = (n + torch.arange(nc)).int().to(DEV)
    st["max_len"] = int(lens.max())
    _handle(st)


# ------------------------------------------------------------------ run

def run(st):
    op = st["case"]["op"]
    if own:
        return {"rope": _own_rope, "append": _own_append, "attend": _own_attend, "pages": _own_pages}[op](st)
    return {"rope": _plain_rope, "append": _plain_append, "attend": _plain_attend, "pages": _plain_pages}[op](st)


def _own_rope(st):
    import paper_2605_29657_gb300 as occ

    q, k = occ.occam_rope(st["q"], st["k"], st["positions"], st["inv_freq"], st["axis"],
                          pairing=st["case"]["pairing"], inverse=st["case"]["inverse"])
    return {"q": q, "k": k}


def _own_append(st):
    import paper_2605_29657_gb300 as occ

    c = st["handle"]
    occ.occam_cache_append(c, st["layer"], st["k_new"], st["v_new"], st["seqs"], st["row_off"])
    i = st["layer"]
    return {"k": c.k[i], "v": c.v[i], "k_scale": c.k_scale[i], "v_scale": c.v_scale[i]}


def _own_attend(st):
    import paper_2605_29657_gb300 as occ

    out, lse = occ.occam_cache_attend(st["handle"], st["layer"], st["q"], st["seqs"], st["row_off"], st["max_rows"],
                                      keep=st["keep"], keep_off=st["keep_off"])
    return {"out": out, "lse": lse}


def _own_pages(st):
    import paper_2605_29657_gb300 as occ

    c = st["handle"]
    occ.occam_cache_release(c, st["dst"])
    occ.occam_cache_fork(c, st["src"], st["dst"])
    if st["case"]["kind"] == "branch":
        occ.occam_cache_extend(c, st["dst"], st["add"])
    else:
        occ.occam_cache_compact(c, st["dst"], st["keep"], st["keep_off"])
    return _pages_out(st)


def _pages_out(st):
    c, f = st["cache"], st["first_spare"]
    return {"table": c["table"], "length": c["length"], "refs": c["refs"], "k": c["k"][:, f:], "v": c["v"][:, f:],
            "k_scale": c["k_scale"][:, f:], "v_scale": c["v_scale"][:, f:]}


def _plain_rope(st):
    case = st["case"]
    half = case["rot"] // 2
    ang = st["positions"][st["axis"].long()].float().T * st["inv_freq"]
    cos, sin = ang.cos()[:, None], ang.sin()[:, None]
    if case["inverse"]:
        sin = -sin

    def turn(x):
        y = x.float()
        r, rest = y[..., :case["rot"]], y[..., case["rot"]:]
        if case["pairing"] == "half":
            a, b = r[..., :half], r[..., half:]
            r = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
        else:
            a, b = r[..., 0::2], r[..., 1::2]
            r = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
        return torch.cat([r, rest], -1).to(x.dtype)

    return {"q": turn(st["q"]), "k": turn(st["k"])}


def _plain_append(st):
    c, i, T = st["cache"], st["layer"], st["case"]["page"]
    seqs, rows = st["seqs"].long(), st["row_off"][1:] - st["row_off"][:-1]
    length = c["length"][seqs].long()
    start = length - rows
    pos = start[st["row_seq"]] + st["row_j"]
    page = c["table"][seqs[st["row_seq"]], pos // T].long()
    # a sequence's first page may hold tokens already: their block keeps at least its scale
    first = c["table"][seqs, (start // T).clamp(max=c["table"].shape[1] - 1)].long()
    held = start % T
    has = (held > 0) & (rows > 0)
    first = torch.where(has, first, torch.zeros_like(first))
    old_slot = (torch.arange(T, device=DEV) < held[:, None]) & has[:, None]
    for codes, scale, new in ((c["k"][i], c["k_scale"][i], st["k_new"]), (c["v"][i], c["v_scale"][i], st["v_new"])):
        x = new.float()
        amax = torch.zeros_like(scale)
        amax.scatter_reduce_(0, page[:, None].expand(-1, amax.shape[1]), x.abs().amax(-1), "amax")
        need = _pow2_scale(amax)
        touched = torch.zeros(scale.shape[0], 1, dtype=torch.bool, device=DEV)
        touched[page] = True
        base = torch.zeros_like(scale)
        base.scatter_reduce_(0, first[:, None].expand(-1, scale.shape[1]),
                             scale[first] * has[:, None].float(), "amax")
        now = torch.where(touched, torch.maximum(need, base), scale)
        block = _at(codes, first)
        again = (block.float() * (scale[first] / now[first])[..., None, None]).to(E4M3)
        # blocks whose scale stays, and slots that are not held tokens, keep their codes
        move = old_slot[:, None, :, None] & (now[first] > scale[first])[..., None, None]
        s, t = torch.nonzero(old_slot, as_tuple=True)
        raw = codes.view(torch.uint8)
        raw[first[s], :, t] = torch.where(move, again.view(torch.uint8), block.view(torch.uint8))[s, :, t]
        raw[page, :, pos % T] = (x / now[page][..., None]).to(E4M3).view(torch.uint8)
        scale.copy_(now)
    return {"k": c["k"][i], "v": c["v"][i], "k_scale": c["k_scale"][i], "v_scale": c["v_scale"][i]}


def _plain_attend(st):
    case, c, i = st["case"], st["cache"], st["layer"]
    T, D, Hkv = case["page"], case["dim"], case["hkv"]
    G, n, R = case["hq"] // Hkv, case["seqs"], st["max_rows"]
    seqs = st["seqs"].long()
    length = c["length"][seqs].long()
    rows = st["row_off"][1:] - st["row_off"][:-1]
    npg = (st["max_len"] + T - 1) // T
    pages = c["table"][seqs, :npg].clamp(min=0).long()
    L = npg * T

    def values(codes, scale):
        x = _at(codes[i], pages).float() * scale[i][pages][..., None, None]
        return x.transpose(1, 2).reshape(n, Hkv, L, D)

    K, V = values(c["k"], c["k_scale"]), values(c["v"], c["v_scale"])
    q = torch.zeros((n, R, case["hq"], D), device=DEV)
    q[st["row_seq"], st["row_j"]] = st["q"].float()
    q = q.reshape(n, R, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(n, Hkv, R * G, D)
    key = torch.arange(L, device=DEV)
    seen = key < length[:, None]
    if st["keep"] is not None:
        off = st["keep_off"]
        at = (off[:-1, None] + key).clamp(max=st["keep"].shape[0] - 1)
        seen = seen & (st["keep"][at] != 0)
    last = (length - rows)[:, None] + torch.arange(R, device=DEV)
    mask = (seen[:, None] & (key <= last[..., None])).repeat_interleave(G, 1)[:, None]
    s = (q @ K.transpose(-1, -2)) * (1.0 / math.sqrt(D))
    s = torch.where(mask, s, s.new_full((), -math.inf))
    m = s.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = torch.exp(s - m)
    l = p.sum(-1, keepdim=True)
    V = torch.where(seen[:, None, :, None], V, V.new_zeros(()))
    o = (p @ V) / torch.where(l == 0, torch.ones_like(l), l)
    lse = m + torch.log(l)
    back = lambda x: x.reshape(n, Hkv, R, G, -1).permute(0, 2, 1, 3, 4).reshape(n, R, case["hq"], -1)[st["row_seq"], st["row_j"]]  # noqa: E731
    return {"out": back(o).to(st["q"].dtype), "lse": back(lse)[..., 0].contiguous()}


def _at(codes, index):
    return codes.view(torch.uint8)[index].view(E4M3)


def _free_pages(refs):
    return torch.nonzero(refs == 0)[:, 0].int()


def _plain_pages(st):
    case, c, T = st["case"], st["cache"], st["case"]["page"]
    table, length, refs = c["table"], c["length"], c["refs"]
    src, dst = st["src"].long(), st["dst"].long()
    slot = torch.arange(table.shape[1], device=DEV)

    def drop(rows):
        held = table[rows]
        refs.index_add_(0, held.clamp(min=0).reshape(-1).long(), -(held >= 0).int().reshape(-1))

    drop(dst)
    table[dst] = -1
    length[dst] = 0
    # fork: full pages are shared, a last page that is not full is copied (lowest free pages first, in order)
    ln = length[src]
    full, part = ln // T, (ln % T > 0)
    shared = torch.where(slot < full[:, None], table[src], torch.full_like(table[src], -1))
    refs.index_add_(0, shared.clamp(min=0).reshape(-1).long(), (shared >= 0).int().reshape(-1))
    new = _free_pages(refs)
    rank = part.cumsum(0) - part.int()
    own_page = torch.where(part, new[rank.clamp(max=new.shape[0] - 1)], torch.full_like(ln, -1))
    table[dst] = torch.where((slot == full[:, None]) & part[:, None], own_page[:, None], shared)
    length[dst] = ln
    refs.index_add_(0, own_page.clamp(min=0).long(), part.int())
    a = torch.nonzero(part)[:, 0]
    frm = table[src[a], full[a].long()].long()
    for name in ("k", "v", "k_scale", "v_scale"):
        x = c[name].view(torch.uint8) if name in ("k", "v") else c[name]
        x[:, own_page[a].long()] = x[:, frm]
    if case["kind"] == "branch":
        have, want = (length[dst] + T - 1) // T, (length[dst] + st["add"] + T - 1) // T
        more = (slot >= have[:, None]) & (slot < want[:, None])
        rank = more.reshape(-1).cumsum(0) - more.reshape(-1).int()
        new = _free_pages(refs)
        got = torch.where(more.reshape(-1), new[rank.clamp(max=new.shape[0] - 1)], torch.full_like(rank, -1).int()).view_as(more)
        table[dst] = torch.where(more, got, table[dst])
        refs.index_add_(0, got.clamp(min=0).reshape(-1).long(), more.reshape(-1).int())
        length[dst] += st["add"]
        return _pages_out(st)
    # compact: leading full pages that keep every token stay, the other kept tokens move to new pages
    off, n, P = st["keep_off"], dst.shape[0], table.shape[1]
    ln = length[dst].long()
    pos = torch.arange(P * T, device=DEV)
    keep = (st["keep"][(off[:-1, None] + pos).clamp(max=st["keep"].shape[0] - 1)] != 0) & (pos < ln[:, None])
    lead = keep.view(n, P, T).all(-1).int().cumprod(-1).sum(-1)
    to = keep.int().cumsum(-1) - 1
    count = keep.sum(-1)
    want = (count + T - 1) // T
    more = (slot >= lead[:, None]) & (slot < want[:, None])
    rank = more.reshape(-1).cumsum(0) - more.reshape(-1).int()
    new = _free_pages(refs)
    got = torch.where(more.reshape(-1), new[rank.clamp(max=new.shape[0] - 1)], torch.full_like(rank, -1).int()).view_as(more)
    old = table[dst]
    s, p = torch.nonzero(keep & (to >= lead[:, None] * T), as_tuple=True)
    sp, ss = old[s, p // T].long(), p % T
    dp, ds = got[s, to[s, p] // T].long(), to[s, p] % T
    gone = (slot >= lead[:, None]) & (old >= 0)
    for name in ("k", "v"):
        codes, scale = c[name], c[name + "_scale"]
        raw = codes.view(torch.uint8)
        x = raw[:, sp, :, ss].view(E4M3).transpose(0, 1).float() * scale[:, sp][..., None]  # [layers, tokens, H, D]
        amax = torch.zeros_like(scale)
        amax.scatter_reduce_(1, dp[None, :, None].expand(x.shape[:3]), x.abs().amax(-1), "amax")
        now = _pow2_scale(amax)
        raw[:, dp, :, ds] = (x / now[:, dp][..., None]).to(E4M3).view(torch.uint8).transpose(0, 1)
        g = got[more].long()
        scale[:, g] = now[:, g]
    table[dst] = torch.where(slot < lead[:, None], old, got)
    refs.index_add_(0, got.clamp(min=0).reshape(-1).long(), more.reshape(-1).int())
    refs.index_add_(0, old.clamp(min=0).reshape(-1).long(), -gone.reshape(-1).int())
    length[dst] = count.int()
    return _pages_out(st)


# ------------------------------------------------------------------ work

def work(case):
    b = 4 if case.get("dtype") == "f32" else 2
    if case["op"] == "rope":
        vals = case["rows"] * (case["hq"] + case["hk"]) * case["dim"]
        pairs = case["rows"] * (case["hq"] + case["hk"]) * case["rot"] // 2
        return {"bytes": 2 * vals * b + case["rows"] * case["axes"] * 4, "flops": 6 * pairs}
    if case["op"] == "append":
        rows = case["seqs"] * (case["rows_lo"] + case["rows_hi"]) / 2
        vals = 2 * rows * case["heads"] * case["dim"]
        return {"bytes": vals * (b + 1) + 2 * 4 * case["heads"] * (rows / case["page"] + case["seqs"]), "flops": 2 * vals}
    if case["op"] == "attend":
        rows = (case["rows_lo"] + case["rows_hi"]) / 2
        ln = max((case["len_lo"] + case["len_hi"]) / 2, rows)
        pairs = case["seqs"] * rows * (ln - (rows - 1) / 2)
        q = case["seqs"] * rows * case["hq"]
        kv = 2 * case["seqs"] * ln * case["hkv"] * (case["dim"] + 4 / case["page"])
        return {"bytes": 2 * q * case["dim"] * b + 4 * q + kv + (case["seqs"] * ln if case["masked"] else 0),
                "flops": 4 * pairs * case["hq"] * case["dim"]}
    ln, nc, T = (case["len_lo"] + case["len_hi"]) / 2, case["parents"] * case["children"], case["page"]
    token = 2 * case["layers"] * case["heads"] * case["dim"]
    copied = 2 * nc * (T / 2) * token  # partial pages of the forks, read and written
    if case["kind"] == "prune":
        copied += 2 * nc * (99 + case["keep"] * max(0, ln - 99)) * token + nc * ln
    return {"bytes": copied + 8 * nc * ln / T, "flops": 0.0}


# ------------------------------------------------------------------ the operators' definitions, in 64 bits

def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    return {"rope": _exact_rope, "append": _exact_append, "attend": _exact_attend, "pages": _exact_pages}[case["op"]](st)


def _exact_rope(st):
    case = st["case"]
    f, half = st["inv_freq"].double(), case["rot"] // 2
    z = torch.polar(torch.ones((), dtype=torch.float64, device=DEV),
                    (-1.0 if case["inverse"] else 1.0) * st["positions"].double()[st["axis"].long()].T * f)
    out = {}
    for name in ("q", "k"):
        x = st[name].double().contiguous()
        y = x.clone()
        lo, hi = (slice(0, half), slice(half, 2 * half)) if case["pairing"] == "half" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
        for h in range(x.shape[1]):
            w = torch.complex(x[:, h, lo].contiguous(), x[:, h, hi].contiguous()) * z
            y[:, h, lo], y[:, h, hi] = w.real, w.imag
        out[name] = y
    return out


def _round_code(x):
    """x (64 bits, |x| <= 448) to the nearest 8-bit value (1 sign, 4 exponent, 3 mantissa bits), ties to even."""
    _, e = torch.frexp(x)
    ulp = ((e.clamp(min=-5) - 4 + 1023).long() << 52).view(torch.float64)  # a power of two, exactly
    return torch.round(x / ulp) * ulp


def _need(amax):
    """The smallest power of two s, 2^-100 at least, with amax <= 448 s, as a float."""
    if amax <= 0:
        return 2.0 ** -100
    e = math.ceil(math.log2(amax / 448.0)) - 1
    while amax > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** min(max(e, -100), 120)


def _need_each(amax):
    return torch.tensor([_need(a) for a in amax.reshape(-1).tolist()], dtype=torch.float64, device=DEV).view(amax.shape)


def _exact_append(st):
    c, i, T = st["cache"], st["layer"], st["case"]["page"]
    if st["k_new"].numel() > 2e8:
        return None
    out = {n: c[n][i].double() for n in ("k", "v", "k_scale", "v_scale")}
    table, length, off = c["table"].cpu(), c["length"].cpu(), st["row_off"].tolist()
    for n, s in enumerate(st["seqs"].tolist()):
        end = int(length[s])
        p = end - (off[n + 1] - off[n])
        r = off[n]
        while p < end:
            o, pg = p % T, int(table[s, p // T])
            m = min(T - o, end - p)
            for name in ("k", "v"):
                x = st[name + "_new"][r:r + m].double()  # [m, H, D]
                was = out[name + "_scale"][pg].clone()
                now = _need_each(x.abs().amax((0, 2)))
                if o:
                    now = torch.maximum(now, was)
                    grown = now > was
                    out[name][pg, grown, :o] = _round_code(out[name][pg, grown, :o] * (was / now)[grown, None, None])
                out[name][pg, :, o:o + m] = _round_code(x / now[:, None]).transpose(0, 1)
                out[name + "_scale"][pg] = now
            p, r = p + m, r + m
    return out


def _exact_attend(st):
    case, c, i = st["case"], st["cache"], st["layer"]
    w = work(case)
    if w["flops"] > 8e11:
        return None
    T, D, G = case["page"], case["dim"], case["hq"] // case["hkv"]
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(st["q"].shape[:2], dtype=torch.float64, device=DEV)
    off = st["row_off"].tolist()
    koff = st["keep_off"].tolist() if st["keep"] is not None else None
    for n, s in enumerate(st["seqs"].tolist()):
        ln, r = int(c["length"][s]), off[n + 1] - off[n]
        pages = c["table"][s, :(ln + T - 1) // T].long()
        allow = torch.arange(ln, device=DEV) <= (ln - r + torch.arange(r, device=DEV))[:, None]
        if koff is not None:
            allow &= st["keep"][koff[n]:koff[n] + ln].bool()
        for h in range(case["hkv"]):
            K = (c["k"][i, pages, h].double() * c["k_scale"][i, pages, h].double()[:, None, None]).reshape(-1, D)[:ln]
            V = (c["v"][i, pages, h].double() * c["v_scale"][i, pages, h].double()[:, None, None]).reshape(-1, D)[:ln]
            for a in range(0, r, 2048):
                q = st["q"][off[n] + a:off[n] + min(a + 2048, r), h * G:(h + 1) * G].double()
                x = torch.einsum("rgd,kd->rgk", q, K) / math.sqrt(D)
                x.masked_fill_(~allow[a:a + 2048, None], -math.inf)
                z = torch.logsumexp(x, -1)
                rows = slice(off[n] + a, off[n] + a + q.shape[0])
                lse[rows, h * G:(h + 1) * G] = z
                out[rows, h * G:(h + 1) * G] = torch.einsum("rgk,kd->rgd", torch.exp(x - z[..., None]).nan_to_num(0.0), V)
    return {"out": out, "lse": lse}


def _exact_pages(st):
    case, c, T, f = st["case"], st["cache"], st["case"]["page"], st["first_spare"]
    table, length, refs = c["table"].cpu().clone(), c["length"].cpu().clone(), c["refs"].cpu().clone()
    out = {n: c[n][:, f:].double() for n in ("k", "v", "k_scale", "v_scale")}

    def take():
        p = int((refs == 0).int().argmax())
        refs[p] = 1
        return p

    src, dst = st["src"].tolist(), st["dst"].tolist()
    for a, b in zip(src, dst):
        for p in range(int(length[a]) // T):
            table[b, p] = table[a, p]
            refs[table[a, p]] += 1
        length[b] = length[a]
    for a, b in zip(src, dst):
        if int(length[a]) % T:
            p, at = take(), int(length[a]) // T
            table[b, at] = p
            for n in out:
                out[n][:, p - f] = c[n][:, int(table[a, at])].double()
    if case["kind"] == "branch":
        for b, add in zip(dst, st["add"].tolist()):
            for at in range(-(-int(length[b]) // T), -(-(int(length[b]) + add) // T)):
                table[b, at] = take()
            length[b] += add
        return {**out, "table": table, "length": length, "refs": refs}
    koff, gone = st["keep_off"].tolist(), []
    for n, b in enumerate(dst):
        flags = st["keep"][koff[n]:koff[n] + int(length[b])].cpu().bool()
        at, lead = torch.nonzero(flags)[:, 0].tolist(), 0
        while (lead + 1) * T <= len(at) and at[(lead + 1) * T - 1] == (lead + 1) * T - 1:
            lead += 1
        old = table[b].tolist()
        gone += [p for p in old[lead:] if p >= 0]
        table[b, lead:] = -1
        for j in range(lead, -(-len(at) // T)):
            mine = at[j * T:(j + 1) * T]
            p = take()
            table[b, j] = p
            pg = torch.tensor([old[x // T] for x in mine], device=DEV)
            sl = torch.tensor([x % T for x in mine], device=DEV)
            for name in ("k", "v"):
                # a copied last page holds what its origin holds
                own_pg = pg >= f
                sc = torch.where(own_pg[:, None], out[name + "_scale"][:, (pg - f).clamp(min=0)], c[name + "_scale"][:, pg].double())
                cd = torch.where(own_pg[:, None, None, None], out[name][:, (pg - f).clamp(min=0), :, sl], c[name].view(torch.uint8)[:, pg, :, sl].view(E4M3).double())
                x = cd.transpose(0, 1) * sc[..., None]
                now = _need_each(x.abs().amax((1, 3)))
                out[name][:, p - f, :, :len(mine)] = _round_code(x / now[:, None, :, None]).transpose(1, 2)
                out[name + "_scale"][:, p - f] = now
        length[b] = len(at)
    for p in gone:
        refs[p] -= 1
    return {**out, "table": table, "length": length, "refs": refs}
