"""Measured cases of the operators that fill a shared prefix and answer over it.

``perf/operators.py`` measures what takes a pruned prefix into decoding. This
file measures what stands before and beside it: a whole prompt's attention to
itself while its keys are still 16-bit rows (``prompt``), the same with its
gradient (``train``), keys turned by their positions on their way into the paged
8-bit cache, with the queries (``enter``), and attention of many questions over one
cached prefix that is read once for all of them (``shared``).

``run`` with ``own`` false is the plain form of each operator, in elementary
torch operations and 32 bits; with ``own`` true it makes the calls of the
framework. Sizes are those of this repository's workloads: 576 + 4 rows per
crop, five crops a sample, 1024 + 4 rows per frame, 16 frames a video, 16 to
512 text tokens, 32 query heads, 32 or 8 key heads of 128 dims, vision towers of 16
heads of 64 or 72 dims.
"""

from __future__ import annotations

import math

import torch

own = False

E4M3 = torch.float8_e4m3fn
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
DEV = "cuda"


# ------------------------------------------------------------------ cases

def listed():
    return [
        # one short question by itself: the smallest prompt, where latency counts
        dict(name="prompt_question_b1", op="prompt", seqs=1, rows_lo=37, rows_hi=37, more_lo=0, more_hi=0, hq=32, hkv=8,
             dim=128, causal=True, dtype="bf16", fused=True),
        # the kept rows of a pruned batch of 64 (about 160 visual + 20 registers + 16..256 text tokens each)
        dict(name="prompt_pruned_b64", op="prompt", seqs=64, rows_lo=196, rows_hi=436, more_lo=0, more_hi=0, hq=32, hkv=32,
             dim=128, causal=True, dtype="bf16", fused=True),
        # half a video's tokens and a question as one prompt
        dict(name="prompt_video_8k", op="prompt", seqs=1, rows_lo=8257, rows_hi=8257, more_lo=0, more_hi=0, hq=32, hkv=8,
             dim=128, causal=True, dtype="bf16", fused=True),
        # a vision tower over ragged images: every patch sees its whole image
        dict(name="prompt_vision_b12", op="prompt", seqs=12, rows_lo=260, rows_hi=4100, more_lo=0, more_hi=0, hq=16, hkv=16,
             dim=72, causal=False, dtype="f16", fused=True),
        # fine-tuning on pruned prompts: ragged, odd lengths
        dict(name="train_pruned_b16", op="train", seqs=16, rows_lo=196, rows_hi=1219, more_lo=0, more_hi=0, hq=32, hkv=8,
             dim=128, causal=True, dtype="bf16", fused=True),
        # fine-tuning on a long prompt (four frames and text)
        dict(name="train_video_4k", op="train", seqs=1, rows_lo=4177, rows_hi=4177, more_lo=0, more_hi=0, hq=32, hkv=8,
             dim=128, causal=True, dtype="bf16", fused=False),
        # a vision tower's crops, 576 patches, a class token and 4 registers each
        dict(name="train_crops_b40", op="train", seqs=40, rows_lo=581, rows_hi=581, more_lo=0, more_hi=0, hq=16, hkv=16,
             dim=64, causal=False, dtype="f16", fused=True),
        # one new token of each of 64 conversations enters the cache
        dict(name="enter_step_b64", op="enter", seqs=64, rows_lo=1, rows_hi=1, len_lo=200, len_hi=4096, hq=32, hkv=8, dim=128,
             rot=128, axes=3, interleaved=True, pairing="half", page=64, dtype="bf16"),
        # the kept rows of a pruned batch of 64 enter the cache
        dict(name="enter_prompt_b64", op="enter", seqs=64, rows_lo=196, rows_hi=436, len_lo=0, len_hi=40, hq=32, hkv=32,
             dim=128, rot=128, axes=3, interleaved=False, pairing="half", page=64, dtype="bf16"),
        # three questions on one image, a token each: the smallest call
        dict(name="shared_step_b3", op="shared", groups=1, each=3, rows_lo=1, rows_hi=1, pre_lo=612, pre_hi=612, own_lo=9,
             own_hi=70, hq=32, hkv=8, dim=128, page=64, dtype="bf16"),
        # decode step of 64 questions on one video
        dict(name="shared_video_b64", op="shared", groups=1, each=64, rows_lo=1, rows_hi=1, pre_lo=16448, pre_hi=16448,
             own_lo=20, own_hi=300, hq=32, hkv=8, dim=128, page=64, dtype="bf16"),
        # eight questions of 16..128 tokens on each of eight 5-crop images
        dict(name="shared_questions_b8", op="shared", groups=8, each=8, rows_lo=16, rows_hi=128, pre_lo=2900, pre_hi=2935,
             own_lo=16, own_hi=160, hq=32, hkv=8, dim=128, page=64, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["prompt", "prompt", "train", "train", "enter", "shared", "shared"])
    if op in ("prompt", "train"):
        form = rng.choice(["one", "few", "many"])
        if form == "one":
            n, lo = 1, _log_int(rng, 1, 7000 if op == "prompt" else 3500)
            hi = lo
        elif form == "few":
            n, lo = rng.randint(2, 8), _log_int(rng, 1, 900)
            hi = lo + rng.randint(0, lo)
        else:
            n, lo = _log_int(rng, 9, 64), _log_int(rng, 1, 250)
            hi = lo + rng.randint(0, lo)
        # a chunk of a longer prompt, now and then: keys before the rows
        more = _log_int(rng, 1, 1000) if rng.random() < 0.25 else 0
        hq, hkv = rng.choice([(32, 8), (32, 32), (16, 16), (28, 4), (12, 2), (8, 1), (5, 1)])
        return dict(op=op, seqs=n, rows_lo=lo, rows_hi=hi, more_lo=more // 2, more_hi=more, hq=hq, hkv=hkv,
                    dim=rng.choice([64, 72, 80, 128, 128]), causal=rng.random() < 0.7, dtype=rng.choice(["bf16", "f16"]),
                    fused=more == 0 and rng.random() < 0.6)
    hq, hkv = rng.choice([(32, 8), (32, 32), (28, 4), (16, 16), (12, 2), (8, 1)])
    if op == "enter":
        lo, dim = _log_int(rng, 1, 150), rng.choice([64, 128])
        rot = dim if rng.random() < 0.6 else rng.choice([dim // 2, 24, 10])
        return dict(op="enter", seqs=_log_int(rng, 1, 64), rows_lo=lo, rows_hi=lo + rng.randint(0, lo), len_lo=0,
                    len_hi=_log_int(rng, 1, 3000), hq=hq, hkv=hkv, dim=dim, rot=rot, axes=rng.choice([1, 2, 3]),
                    interleaved=rng.random() < 0.5, pairing=rng.choice(["half", "adjacent"]),
                    page=rng.choice([16, 32, 64, 128]), dtype=rng.choice(["bf16", "f16"]))
    groups = rng.choice([1, 1, 2, 5])
    each = _log_int(rng, 1, 48) if groups == 1 else _log_int(rng, 1, 10)
    r = 1 if rng.random() < 0.6 else _log_int(rng, 2, 60)
    own_lo, pre = _log_int(rng, r, r + 200), _log_int(rng, 20, 9000 // groups)
    return dict(op="shared", groups=groups, each=each, rows_lo=r, rows_hi=r if r == 1 else r + rng.randint(0, r),
                pre_lo=max(1, pre // rng.choice([1, 2])), pre_hi=pre, own_lo=own_lo, own_hi=own_lo + rng.randint(0, 300),
                hq=hq, hkv=hkv, dim=rng.choice([64, 128, 128]), page=rng.choice([16, 32, 64, 128]),
                dtype=rng.choice(["bf16", "f16"]))


# ------------------------------------------------------------------ inputs

def _lengths(lo, hi, n):
    """n ragged lengths in lo..hi, the same for every seed (they are the case's sizes), in no order."""
    g = torch.Generator().manual_seed(1000003 * lo + 101 * hi + n)
    return torch.randint(lo, hi + 1, (n,), generator=g, dtype=torch.int64)


def _offsets(counts):
    off = torch.zeros(counts.numel() + 1, dtype=torch.int64)
    off[1:] = counts.cumsum(0)
    return off


def _place(off):
    """Of each row of ragged runs: its run and its place in the run, on the GPU."""
    run = torch.repeat_interleave(torch.arange(off.numel() - 1), off.diff())
    return run.to(DEV), (torch.arange(int(off[-1])) - off[run]).to(DEV)


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


def _blocks(layers, pages, H, T, D, g):
    k = torch.empty((layers, pages, H, T, D), dtype=E4M3, device=DEV)
    v = torch.empty_like(k)
    ks = torch.empty((layers, pages, H), device=DEV)
    vs = torch.empty_like(ks)
    for i in range(layers):
        k[i], ks[i] = _fill_blocks((pages, H, T, D), g, 1.0)
        v[i], vs[i] = _fill_blocks((pages, H, T, D), g, torch.exp(0.5 * torch.randn((pages, H, 1, 1), device=DEV, generator=g)))
    return dict(k=k, v=v, k_scale=ks, v_scale=vs)


def prepare(case, seed):
    cpu = torch.Generator().manual_seed(seed)
    g = torch.Generator(device=DEV).manual_seed(seed)
    st = dict(case=case)
    {"prompt": _prepare_prompt, "train": _prepare_prompt, "enter": _prepare_enter, "shared": _prepare_shared}[case["op"]](case, st, cpu, g)
    return st


def _prompt_lengths(case):
    rows = _lengths(case["rows_lo"], case["rows_hi"], case["seqs"])
    return rows, rows + _lengths(case["more_lo"], case["more_hi"], case["seqs"])


def _prepare_prompt(case, st, cpu, g):
    hq, hkv, D, dt = case["hq"], case["hkv"], case["dim"], DTYPES[case["dtype"]]
    rows, keys = _prompt_lengths(case)
    off, koff = _offsets(rows), _offsets(keys)
    total, ktotal = int(off[-1]), int(koff[-1])

    def normal(n, h, gain):
        return (torch.randn((n, h, D), device=DEV, generator=g) * gain).to(dt)

    if case["fused"]:  # views of one projection's output
        qkv = normal(total, hq + 2 * hkv, 1.2)
        st["q"], st["k"], st["v"] = qkv.split((hq, hkv, hkv), 1)
    else:
        st["q"], st["k"], st["v"] = normal(total, hq, 1.4), normal(ktotal, hkv, 1.2), normal(ktotal, hkv, 1.0)
    if case["op"] == "train":
        # a loss's gradient: small, and of different size from row to row
        size = 0.02 * torch.exp(torch.randn((total, 1, 1), device=DEV, generator=g))
        st["dout"] = (torch.randn((total, hq, D), device=DEV, generator=g) * size).to(dt)
    st["max_rows"], st["max_keys"] = int(rows.max()), int(keys.max())
    st["row_off"], st["key_off"] = off.to(DEV), koff.to(DEV)
    st["row_seq"], st["row_j"] = _place(off)
    st["key_seq"], st["key_j"] = _place(koff)
    if own:
        import paper_2605_29657_gb300 as occ

        st["ws"] = occ.alloc_prompt_workspace(total, hq, ktotal, hkv)


def _handle(st, **more):
    if own:
        import paper_2605_29657_gb300 as occ

        st["handle"] = occ.PagedCache.wrap(**st["cache"])
        st["ws"] = st["handle"].alloc_workspace(**more)


def _prepare_enter(case, st, cpu, g):
    n, T, H, D, dt = case["seqs"], case["page"], case["hkv"], case["dim"], DTYPES[case["dtype"]]
    rows = _lengths(case["rows_lo"], case["rows_hi"], n)
    lens = rows + _lengths(case["len_lo"], case["len_hi"], n)
    slots = torch.randperm(n, generator=cpu)
    per = (lens + T - 1) // T
    first = _offsets(per)
    perm = torch.randperm(int(first[-1]), generator=cpu).int()
    table = torch.full((n, int(per.max())), -1, dtype=torch.int32)
    length = torch.zeros(n, dtype=torch.int32)
    for i, s in enumerate(slots.tolist()):
        table[s, :int(per[i])] = perm[int(first[i]):int(first[i + 1])]
        length[s] = int(lens[i])
    pages = int(first[-1]) + 3
    refs = torch.zeros(pages, dtype=torch.int32)
    refs[:int(first[-1])] = 1
    st["cache"] = dict(**_blocks(2, pages, H, T, D, g), table=table.to(DEV), length=length.to(DEV), refs=refs.to(DEV))
    st["layer"] = 1
    off = _offsets(rows)
    total = int(off[-1])
    gain = torch.exp(0.7 * torch.randn((1, case["hq"] + 2 * H, D), device=DEV, generator=g))
    burst = 1 + 7 * (torch.rand((total, 1, 1), device=DEV, generator=g) < 0.1).float()
    qkv = (torch.randn((total, case["hq"] + 2 * H, D), device=DEV, generator=g) * gain * burst).to(dt)
    st["q"], st["k_new"], st["v_new"] = qkv.split((case["hq"], H, H), 1)
    half = case["rot"] // 2
    i = torch.arange(half)
    axis = i % case["axes"] if case["interleaved"] else i * case["axes"] // half
    st["axis"] = axis.int().to(DEV)
    st["inv_freq"] = (10000.0 ** (-(2.0 * i.double()) / case["rot"])).float().to(DEV)
    st["positions"] = torch.randint(0, 20000, (case["axes"], total), generator=cpu, dtype=torch.int32).to(DEV)
    st["seqs"], st["row_off"] = slots.int().to(DEV), off.to(DEV)
    st["row_seq"], st["row_j"] = _place(off)
    _handle(st)


def _shared_lengths(case):
    """Prefix tokens of each group, rows and own tokens (the rows among them) of each sequence."""
    n = case["groups"] * case["each"]
    rows = _lengths(case["rows_lo"], case["rows_hi"], n)
    return _lengths(case["pre_lo"], case["pre_hi"], case["groups"]), rows, torch.maximum(_lengths(case["own_lo"], case["own_hi"], n), rows)


def _prepare_shared(case, st, cpu, g):
    T, H, D, each, n = case["page"], case["hkv"], case["dim"], case["each"], case["groups"] * case["each"]
    pre, rows, mine = _shared_lengths(case)
    lens = pre.repeat_interleave(each) + mine
    full = pre // T  # pages of a group's prefix that its sequences hold together
    rest = (lens + T - 1) // T - full.repeat_interleave(each)
    used = int(full.sum() + rest.sum())
    perm = torch.randperm(used, generator=cpu).int()
    slots = torch.randperm(n, generator=cpu)
    table = torch.full((n, int(((lens + T - 1) // T).max())), -1, dtype=torch.int32)
    length = torch.zeros(n, dtype=torch.int32)
    refs = torch.zeros(used + 2, dtype=torch.int32)
    at = 0
    for grp in range(case["groups"]):
        f = int(full[grp])
        together = perm[at:at + f]
        at += f
        refs[together.long()] = each
        for i in range(grp * each, (grp + 1) * each):
            s, r = int(slots[i]), int(rest[i])
            table[s, :f] = together
            table[s, f:f + r] = perm[at:at + r]
            refs[perm[at:at + r].long()] = 1
            at += r
            length[s] = int(lens[i])
    st["cache"] = dict(**_blocks(1, used + 2, H, T, D, g), table=table.to(DEV), length=length.to(DEV), refs=refs.to(DEV))
    st["layer"] = 0
    off = _offsets(rows)
    total = int(off[-1])
    st["q"] = (1.5 * torch.randn((total, case["hq"], D), device=DEV, generator=g)).to(DTYPES[case["dtype"]])
    st["max_rows"], st["max_len"] = int(rows.max()), int(lens.max())
    st["max_group_rows"] = int(rows.view(case["groups"], each).sum(1).max())
    st["seqs"], st["row_off"] = slots.int().to(DEV), off.to(DEV)
    st["group_off"] = torch.arange(0, n + 1, each, dtype=torch.int32).to(DEV)
    st["row_seq"], st["row_j"] = _place(off)
    _handle(st, rows=total, heads=case["hq"])


# ------------------------------------------------------------------ run

def run(st):
    op = st["case"]["op"]
    if own:
        return {"prompt": _own_prompt, "train": _own_train, "enter": _own_enter, "shared": _own_shared}[op](st)
    return {"prompt": _plain_prompt, "train": _plain_train, "enter": _plain_enter, "shared": _plain_shared}[op](st)


def _own_prompt(st):
    import paper_2605_29657_gb300 as occ

    out, lse = occ.occam_prompt_attend(st["q"], st["k"], st["v"], st["row_off"], st["ws"], key_off=st["key_off"],
                                       causal=st["case"]["causal"])
    return {"out": out, "lse": lse}


def _own_train(st):
    import paper_2605_29657_gb300 as occ

    keys = dict(key_off=st["key_off"], causal=st["case"]["causal"])
    out, lse = occ.occam_prompt_attend(st["q"], st["k"], st["v"], st["row_off"], st["ws"], **keys)
    dq, dk, dv = occ.occam_prompt_attend_grad(st["q"], st["k"], st["v"], out, lse, st["dout"], st["row_off"], st["ws"], **keys)
    return {"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv}


def _own_enter(st):
    import paper_2605_29657_gb300 as occ

    c, i = st["handle"], st["layer"]
    q = occ.occam_cache_append_rope(c, i, st["q"], st["k_new"], st["v_new"], st["seqs"], st["row_off"], st["positions"],
                                    st["inv_freq"], st["axis"], pairing=st["case"]["pairing"], ws=st["ws"])
    return {"q": q, "k": c.k[i], "v": c.v[i], "k_scale": c.k_scale[i], "v_scale": c.v_scale[i]}


def _own_shared(st):
    import paper_2605_29657_gb300 as occ

    out, lse = occ.occam_cache_attend_shared(st["handle"], st["layer"], st["q"], st["seqs"], st["row_off"], st["max_rows"],
                                             st["group_off"], st["max_group_rows"], st["ws"])
    return {"out": out, "lse": lse}


def _padded(x, run, j, n, R):
    out = torch.zeros((n, R, *x.shape[1:]), device=DEV)
    out[run, j] = x.float()
    return out


def _prompt_parts(st):
    """Queries, keys and values of a padded batch, scores (hidden ones -inf) and their softmax."""
    case = st["case"]
    n, R, L, Hkv, D = case["seqs"], st["max_rows"], st["max_keys"], case["hkv"], case["dim"]
    G = case["hq"] // Hkv
    q = _grouped(_padded(st["q"], st["row_seq"], st["row_j"], n, R), Hkv, G)
    k = _padded(st["k"], st["key_seq"], st["key_j"], n, L).transpose(1, 2)
    v = _padded(st["v"], st["key_seq"], st["key_j"], n, L).transpose(1, 2)
    rows, keys = st["row_off"].diff(), st["key_off"].diff()
    key = torch.arange(L, device=DEV)
    seen = (key < keys[:, None])[:, None]
    if case["causal"]:
        seen = seen & (key <= (keys - rows)[:, None, None] + torch.arange(R, device=DEV)[:, None])
    mask = seen.expand(n, R, L).repeat_interleave(G, 1)[:, None]
    s = (q @ k.transpose(-1, -2)) * (1.0 / math.sqrt(D))
    s = torch.where(mask, s, s.new_full((), -math.inf))
    m = s.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = torch.exp(s - m)
    del s
    l = p.sum(-1, keepdim=True)
    p /= torch.where(l == 0, torch.ones_like(l), l)
    return q, k, v, p, m + torch.log(l)


def _grouped(x, Hkv, G):
    """[n, R, heads, D] to [n, key heads, R G, D]."""
    n, R, _, D = x.shape
    return x.reshape(n, R, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(n, Hkv, R * G, D)


def _rows_of(x, st, G):
    """[n, key heads, R G, D] back to the ragged rows [rows, heads, D]."""
    n, Hkv, RG, D = x.shape
    x = x.reshape(n, Hkv, RG // G, G, D).permute(0, 2, 1, 3, 4).reshape(n, RG // G, Hkv * G, D)
    return x[st["row_seq"], st["row_j"]]


def _plain_prompt(st):
    G = st["case"]["hq"] // st["case"]["hkv"]
    _, _, v, p, lse = _prompt_parts(st)
    return {"out": _rows_of(p @ v, st, G).to(st["q"].dtype), "lse": _rows_of(lse, st, G)[..., 0].contiguous()}


def _plain_train(st):
    case, dt = st["case"], st["q"].dtype
    Hkv, scale = case["hkv"], 1.0 / math.sqrt(case["dim"])
    G = case["hq"] // Hkv
    q, k, v, p, lse = _prompt_parts(st)
    o = p @ v
    do = _grouped(_padded(st["dout"], st["row_seq"], st["row_j"], case["seqs"], st["max_rows"]), Hkv, G)
    dv = p.transpose(-1, -2) @ do
    ds = do @ v.transpose(-1, -2)
    ds -= (do * o).sum(-1, keepdim=True)
    ds *= p
    dq = (ds @ k) * scale
    dk = (ds.transpose(-1, -2) @ q) * scale

    def keys(x):
        return x.transpose(1, 2)[st["key_seq"], st["key_j"]].to(dt)

    return {"out": _rows_of(o, st, G).to(dt), "lse": _rows_of(lse, st, G)[..., 0].contiguous(),
            "dq": _rows_of(dq, st, G).to(dt), "dk": keys(dk), "dv": keys(dv)}


def _at(codes, index):
    return codes.view(torch.uint8)[index].view(E4M3)


def _plain_enter(st):
    case, c, i = st["case"], st["cache"], st["layer"]
    T, rot, half = case["page"], case["rot"], case["rot"] // 2
    # angles of far positions in 64 bits, the turn itself in 32
    ang = st["positions"][st["axis"].long()].double().T * st["inv_freq"].double()
    cos, sin = ang.cos().float()[:, None], ang.sin().float()[:, None]

    def turn(x):
        y = x.float()
        r, rest = y[..., :rot], y[..., rot:]
        if case["pairing"] == "half":
            a, b = r[..., :half], r[..., half:]
            r = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
        else:
            a, b = r[..., 0::2], r[..., 1::2]
            r = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
        return torch.cat([r, rest], -1)

    seqs, rows = st["seqs"].long(), st["row_off"].diff()
    start = c["length"][seqs].long() - rows
    pos = start[st["row_seq"]] + st["row_j"]
    page = c["table"][seqs[st["row_seq"]], pos // T].long()
    # a sequence's first page may hold tokens already: their block keeps at least its scale
    first = c["table"][seqs, (start // T).clamp(max=c["table"].shape[1] - 1)].long()
    held = start % T
    has = (held > 0) & (rows > 0)
    first = torch.where(has, first, torch.zeros_like(first))
    old_slot = (torch.arange(T, device=DEV) < held[:, None]) & has[:, None]
    s, t = torch.nonzero(old_slot, as_tuple=True)

    def put(codes, scale, x):
        amax = torch.zeros_like(scale)
        amax.scatter_reduce_(0, page[:, None].expand(-1, amax.shape[1]), x.abs().amax(-1), "amax")
        need = _pow2_scale(amax)
        touched = torch.zeros(scale.shape[0], 1, dtype=torch.bool, device=DEV)
        touched[page] = True
        base = torch.zeros_like(scale)
        base.scatter_reduce_(0, first[:, None].expand(-1, scale.shape[1]), scale[first] * has[:, None].float(), "amax")
        now = torch.where(touched, torch.maximum(need, base), scale)
        block = _at(codes, first)
        again = (block.float() * (scale[first] / now[first])[..., None, None]).to(E4M3)
        # blocks whose scale stays, and slots that are not held tokens, keep their codes
        move = old_slot[:, None, :, None] & (now[first] > scale[first])[..., None, None]
        raw = codes.view(torch.uint8)
        raw[first[s], :, t] = torch.where(move, again.view(torch.uint8), block.view(torch.uint8))[s, :, t]
        raw[page, :, pos % T] = (x / now[page][..., None]).to(E4M3).view(torch.uint8)
        scale.copy_(now)

    put(c["k"][i], c["k_scale"][i], turn(st["k_new"]))
    put(c["v"][i], c["v_scale"][i], st["v_new"].float())
    return {"q": turn(st["q"]).to(st["q"].dtype), "k": c["k"][i], "v": c["v"][i], "k_scale": c["k_scale"][i],
            "v_scale": c["v_scale"][i]}


def _plain_shared(st):
    case, c, i = st["case"], st["cache"], st["layer"]
    T, D, Hkv = case["page"], case["dim"], case["hkv"]
    G, n, R = case["hq"] // Hkv, case["groups"] * case["each"], st["max_rows"]
    seqs = st["seqs"].long()
    length = c["length"][seqs].long()
    rows = st["row_off"].diff()
    npg = (st["max_len"] + T - 1) // T
    pages = c["table"][seqs, :npg].clamp(min=0).long()
    L = npg * T

    def values(codes, scale):
        x = _at(codes[i], pages).float() * scale[i][pages][..., None, None]
        return x.transpose(1, 2).reshape(n, Hkv, L, D)

    K = values(c["k"], c["k_scale"])
    q = _grouped(_padded(st["q"], st["row_seq"], st["row_j"], n, R), Hkv, G)
    key = torch.arange(L, device=DEV)
    last = (length - rows)[:, None] + torch.arange(R, device=DEV)
    mask = ((key < length[:, None])[:, None] & (key <= last[..., None])).repeat_interleave(G, 1)[:, None]
    s = (q @ K.transpose(-1, -2)) * (1.0 / math.sqrt(D))
    s = torch.where(mask, s, s.new_full((), -math.inf))
    m = s.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = torch.exp(s - m)
    l = p.sum(-1, keepdim=True)
    V = values(c["v"], c["v_scale"])
    V = torch.where((key < length[:, None])[:, None, :, None], V, V.new_zeros(()))
    o = (p @ V) / torch.where(l == 0, torch.ones_like(l), l)
    lse = m + torch.log(l)
    return {"out": _rows_of(o, st, G).to(st["q"].dtype), "lse": _rows_of(lse, st, G)[..., 0].contiguous()}


# ------------------------------------------------------------------ work

def _seen_pairs(rows, keys, causal):
    """(row, key) pairs that are seen; the rows are the last of their keys."""
    return float((rows * keys - rows * (rows - 1) // 2).sum() if causal else (rows * keys).sum())


def work(case):
    if case["op"] in ("prompt", "train"):
        rows, keys = _prompt_lengths(case)
        pairs = _seen_pairs(rows, keys, case["causal"]) * case["hq"] * case["dim"]
        q, kv = float(rows.sum()) * case["hq"] * case["dim"] * 2, 2 * float(keys.sum()) * case["hkv"] * case["dim"] * 2
        lse = float(rows.sum()) * case["hq"] * 4
        if case["op"] == "prompt":
            return {"bytes": 2 * q + kv + lse, "flops": 4 * pairs}
        # q, k, v and the output's gradient read; out, lse and the three gradients written
        return {"bytes": 4 * q + 2 * kv + lse, "flops": 14 * pairs}
    if case["op"] == "enter":
        rows = float(_lengths(case["rows_lo"], case["rows_hi"], case["seqs"]).sum())
        q, vals = rows * case["hq"] * case["dim"], 2 * rows * case["hkv"] * case["dim"]
        return {"bytes": 4 * q + 3 * vals + 2 * 4 * case["hkv"] * (rows / case["page"] + case["seqs"]) + 4 * rows * case["axes"],
                "flops": 3 * rows * (case["hq"] + case["hkv"]) * case["rot"] + 2 * vals}
    pre, rows, mine = _shared_lengths(case)
    held = float(pre.sum() + mine.sum())
    q = float(rows.sum()) * case["hq"]
    pairs = _seen_pairs(rows, pre.repeat_interleave(case["each"]) + mine, True)
    return {"bytes": 4 * q * case["dim"] + 4 * q + 2 * held * case["hkv"] * (case["dim"] + 4 / case["page"]),
            "flops": 4 * pairs * case["hq"] * case["dim"]}


# ------------------------------------------------------------------ the operators' definitions, in 64 bits

def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    return {"prompt": _exact_prompt, "train": _exact_prompt, "enter": _exact_enter, "shared": _exact_shared}[case["op"]](st)


def _exact_prompt(st):
    """Sequence by sequence and head by head, the sums over rows in blocks."""
    case = st["case"]
    if work(case)["flops"] > 4e12:
        return None
    train, G, scale = case["op"] == "train", case["hq"] // case["hkv"], case["dim"] ** -0.5
    f64 = dict(dtype=torch.float64, device=DEV)
    out, lse = torch.zeros(st["q"].shape, **f64), torch.zeros(st["q"].shape[:2], **f64)
    dq, dk, dv = torch.zeros_like(out), torch.zeros(st["k"].shape, **f64), torch.zeros(st["v"].shape, **f64)
    off, koff = st["row_off"].tolist(), st["key_off"].tolist()
    for n in range(case["seqs"]):
        r, m = off[n + 1] - off[n], koff[n + 1] - koff[n]
        ks = slice(koff[n], koff[n + 1])
        for h in range(case["hq"]):
            K, V = st["k"][ks, h // G].double(), st["v"][ks, h // G].double()
            for a in range(0, r, 4096):
                b = min(a + 4096, r)
                rs = slice(off[n] + a, off[n] + b)
                Q = st["q"][rs, h].double()
                x = torch.mul(Q @ K.T, scale)
                if case["causal"]:
                    x.masked_fill_(torch.ones((b - a, m), dtype=torch.bool, device=DEV).triu(m - r + a + 1), -math.inf)
                z = torch.logsumexp(x, 1)
                x = torch.exp(x - z[:, None])
                out[rs, h], lse[rs, h] = x @ V, z
                if train:
                    dO = st["dout"][rs, h].double()
                    dv[ks, h // G] += x.T @ dO
                    x = x * (dO @ V.T - torch.linalg.vecdot(dO, out[rs, h])[:, None])
                    dq[rs, h] = scale * (x @ K)
                    dk[ks, h // G] += scale * (x.T @ Q)
    return {"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv} if train else {"out": out, "lse": lse}


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


def _exact_enter(st):
    case, c, i, T = st["case"], st["cache"], st["layer"], st["case"]["page"]
    half = case["rot"] // 2
    lo, hi = (slice(0, half), slice(half, 2 * half)) if case["pairing"] == "half" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
    z = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), st["positions"].double()[st["axis"].long()].T * st["inv_freq"].double())

    def turned(x):
        y = x.double().contiguous()
        w = torch.complex(y[..., lo].contiguous(), y[..., hi].contiguous()) * z[:, None]
        y[..., lo], y[..., hi] = w.real, w.imag
        return y

    new = {"k": turned(st["k_new"]), "v": st["v_new"].double()}
    out = {n: c[n][i].double() for n in ("k", "v", "k_scale", "v_scale")}
    table, length, off = c["table"].cpu(), c["length"].cpu(), st["row_off"].tolist()
    for n, s in enumerate(st["seqs"].tolist()):
        end = int(length[s])
        r, p = off[n], end - (off[n + 1] - off[n])
        while p < end:
            o, pg = p % T, int(table[s, p // T])
            m = min(T - o, end - p)
            for name in ("k", "v"):
                x = new[name][r:r + m]  # [m, H, D]
                was = out[name + "_scale"][pg].clone()
                now = torch.tensor([_need(a) for a in x.abs().amax((0, 2)).tolist()], dtype=torch.float64, device=DEV)
                if o:
                    now = torch.maximum(now, was)
                    grown = now > was
                    out[name][pg, grown, :o] = _round_code(out[name][pg, grown, :o] * (was / now)[grown, None, None])
                out[name][pg, :, o:o + m] = _round_code(x / now[:, None]).transpose(0, 1)
                out[name + "_scale"][pg] = now
            p, r = p + m, r + m
    return {"q": turned(st["q"]), **out}


def _exact_shared(st):
    case, c, i = st["case"], st["cache"], st["layer"]
    if work(case)["flops"] > 4e12:
        return None
    T, D, G = case["page"], case["dim"], case["hq"] // case["hkv"]
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(st["q"].shape[:2], dtype=torch.float64, device=DEV)
    off = st["row_off"].tolist()
    for n, s in enumerate(st["seqs"].tolist()):
        ln, rs = int(c["length"][s]), slice(off[n], off[n + 1])
        pages = c["table"][s, :(ln + T - 1) // T].long()
        r = off[n + 1] - off[n]
        hidden = torch.ones((r, ln), dtype=torch.bool, device=DEV).triu(ln - r + 1)
        for h in range(case["hkv"]):
            K = (c["k"][i, pages, h].double() * c["k_scale"][i, pages, h].double()[:, None, None]).reshape(-1, D)[:ln]
            V = (c["v"][i, pages, h].double() * c["v_scale"][i, pages, h].double()[:, None, None]).reshape(-1, D)[:ln]
            x = torch.einsum("rgd,kd->rgk", st["q"][rs, h * G:(h + 1) * G].double(), K) / math.sqrt(D)
            x.masked_fill_(hidden[:, None], -math.inf)
            z = torch.logsumexp(x, -1)
            lse[rs, h * G:(h + 1) * G] = z
            out[rs, h * G:(h + 1) * G] = torch.einsum("rgk,kd->rgd", torch.exp(x - z[..., None]), V)
    return {"out": out, "lse": lse}
