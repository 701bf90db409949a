"""Pruned images as the prefix of a small decoder: prune, fill the cache,
answer two questions about every image, give the pages back.

    python examples/prune_and_answer.py

1. occam_prune keeps the visual rows that pass both tests and gathers them.
2. The kept rows go through the decoder as its prefix: rotary positions (time,
   height, width) from where each row stood before pruning, keys and values
   into the paged 8-bit cache.
3. The prefixes are forked for a second question; there the same scores are
   tested against a higher threshold and the branch is pruned again in place.
4. Both branches read their question and generate greedily, a token at a time.
5. All sequences are released.

Nothing between the prune call and the answers waits for the GPU: offsets and
counts stay on the device. Weights, images and questions are random and seeded.
"""

from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2605_29657_gb300 as occ  # noqa: E402
from synth import tiny_batch  # noqa: E402

HIDDEN, LAYERS, HEADS, KV_HEADS, DIM, VOCAB = 256, 2, 8, 2, 64, 512
GRID = 8  # patches in a row of an image
SECTIONS = (8, 12, 12)  # pairs that turn with time, height, width


def norm(x):
    return torch.nn.functional.rms_norm(x, x.shape[-1:])


class Decoder:
    """Attention layers over the paged cache (bf16, random weights)."""

    def __init__(self, cache: occ.PagedCache, seed: int = 0):
        g = torch.Generator().manual_seed(seed)

        def weight(n_in, n_out):
            return (torch.randn((n_in, n_out), generator=g) * n_in ** -0.5).to(torch.bfloat16).cuda()

        self.cache = cache
        self.qkv = [weight(HIDDEN, (HEADS + 2 * KV_HEADS) * DIM) for _ in range(LAYERS)]
        self.proj = [weight(HEADS * DIM, HIDDEN) for _ in range(LAYERS)]
        self.embed = weight(HIDDEN, VOCAB).T.contiguous()
        pairs = sum(SECTIONS)
        self.inv_freq = (10000.0 ** (-torch.arange(pairs, dtype=torch.float32) / pairs)).cuda()
        self.axis = occ.rope_axes(SECTIONS)

    def attend(self, layer, q, seqs, row_off, max_rows):
        return occ.occam_cache_attend(self.cache, layer, q, seqs, row_off, max_rows)[0]

    def __call__(self, x, positions, seqs, row_off, max_rows):
        """Rows x [rows, HIDDEN] as the newest tokens of the sequences: the cache grows by
        them, and their new hidden states come back."""
        occ.occam_cache_extend(self.cache, seqs, row_off.diff().to(torch.int32))
        for layer in range(LAYERS):
            rows = (norm(x) @ self.qkv[layer]).view(-1, HEADS + 2 * KV_HEADS, DIM)
            q, k, v = rows.split((HEADS, KV_HEADS, KV_HEADS), 1)  # views: every call takes them as they lie
            q, k = occ.occam_rope(q, k, positions, self.inv_freq, self.axis)
            occ.occam_cache_append(self.cache, layer, k, v, seqs, row_off)
            x = x + self.attend(layer, q, seqs, row_off, max_rows).view(-1, HEADS * DIM) @ self.proj[layer]
        return norm(x)


def answer(decoder, seqs, tokens, start: int, steps: int):
    """Reads the question `tokens` [n, length] at text positions start, start + 1, ..
    and generates `steps` tokens greedily. Returns (tokens [n, steps], logits of the last)."""
    n, out = tokens.shape[0], []
    for _ in range(steps):
        rows = tokens.shape[1]
        at = torch.arange(start, start + rows, dtype=torch.int32, device="cuda").repeat(n)
        row_off = torch.arange(0, (n + 1) * rows, rows, dtype=torch.int64, device="cuda")
        x = decoder(decoder.embed[tokens.reshape(-1)], at.expand(len(SECTIONS), -1).contiguous(), seqs, row_off, rows)
        logits = x.view(n, rows, HIDDEN)[:, -1].float() @ decoder.embed.T.float()
        tokens = logits.argmax(-1, keepdim=True)
        out.append(tokens)
        start += rows
    return torch.cat(out, 1), logits


def run(images: int = 4, steps: int = 4, stricter: float = 1.5, seed: int = 7, decoder_type=Decoder) -> dict:
    """stricter: the factor on the second question's threshold (0: its branch keeps all)."""
    lambda1, lambda2 = 0.3, 1.0
    b = tiny_batch(B=images, segs=1, P=tuple(GRID * (GRID - i % 3) for i in range(images)), R=4,
                   M=tuple(9 + 3 * i for i in range(images)), H1=16, d1=64, H2=32, d2=128, hidden=HIDDEN, seed=seed)
    layout = occ.BatchLayout.from_batch(b, "cuda")
    d = {k: b[k].cuda() for k in ("q_cls", "k_cls", "K1", "Q_text", "K_text", "K2", "hidden")}
    pruned = occ.occam_prune(layout, dict(mode="cls", q=d["q_cls"], k_cls=d["k_cls"], K1=d["K1"]),
                             dict(Q_text=d["Q_text"], K_text=d["K_text"], K2=d["K2"]), lambda1, lambda2,
                             gather=(d["hidden"],))
    row_off, (hidden,) = pruned["out_off"], pruned["gathered"]

    # Where every row stands in its image, and from that the kept rows' positions.
    # (Rows past the kept ones are not used; their indices are brought into range.)
    ends = b["meta"]["row_off_host"]
    place = torch.cat([torch.arange(int(n)) for n in ends[1:] - ends[:-1]])
    grid = torch.stack((torch.zeros_like(place), place // GRID, place % GRID)).to(torch.int32).cuda()
    kept = pruned["out_index"].long().clamp(0, layout.total_rows - 1)
    max_rows = int((ends[1:] - ends[:-1]).max())

    cache = occ.PagedCache(layers=LAYERS, pages=24 * images, heads=KV_HEADS, dim=DIM, max_seqs=2 * images, max_pages=16,
                           page_tokens=16)
    decoder = decoder_type(cache)
    first = torch.arange(images, dtype=torch.int32, device="cuda")
    second = first + images
    decoder(hidden, grid[:, kept].contiguous(), first, row_off, max_rows)

    occ.occam_cache_fork(cache, first, second)
    if stricter:
        flags, _ = occ.occam_threshold(layout, pruned["s2"], pruned["ref2"], occ.OCCAM_REF_SAMPLE, stricter * lambda2,
                                       prev_keep=pruned["keep2"])
        occ.occam_cache_compact(cache, second, flags[kept].contiguous(), row_off)
    prefix = cache.length.clone()

    g = torch.Generator().manual_seed(seed)
    question = torch.randint(0, VOCAB, (2, images, 6), generator=g).cuda()
    answers = [answer(decoder, s, q, GRID, steps) for s, q in ((first, question[0]), (second, question[1 if stricter else 0]))]

    occ.occam_cache_release(cache, torch.cat((first, second)))
    return dict(status=cache.status(), prefix=prefix.view(2, -1).tolist(), rows=(ends[1:] - ends[:-1]).tolist(),
                answers=[a.tolist() for a, _ in answers], logits=[x for _, x in answers], cache=cache)


if __name__ == "__main__":
    r = run()
    print("rows of each image:", r["rows"])
    print("kept, first question:", r["prefix"][0], " second:", r["prefix"][1])
    print("answers:", r["answers"][0], r["answers"][1])
    print("status", r["status"], " pages still held:", int(r["cache"].refs.sum()))
