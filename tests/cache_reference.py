"""Plain 64-bit implementations of the rotary and cache operators (CPU, from
their definitions), and the bounds their results are held to."""

from __future__ import annotations

import math

import torch

E4M3 = torch.float8_e4m3fn
UNIT = {t: torch.finfo(t).eps / 2 for t in (torch.bfloat16, torch.float16, torch.float32)}  # half an ulp, relative
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}  # half the least subnormal


def rope(x, positions, inv_freq, axis, pairing, inverse):
    """(result, |a| + |b| of each value's pair) in float64."""
    x = x.double().cpu()
    half = inv_freq.numel()
    t = positions.cpu().double()[axis.cpu().long()].T * inv_freq.cpu().double()  # [rows, pairs]
    c, s = torch.cos(t)[:, None], torch.sin(t)[:, None] * (-1.0 if inverse else 1.0)
    lo, hi = ((slice(0, half), slice(half, 2 * half)) if pairing == "half"
              else (slice(0, 2 * half, 2), slice(1, 2 * half, 2)))
    y, mag = x.clone(), torch.zeros_like(x)
    a, b = x[..., lo], x[..., hi]
    y[..., lo], y[..., hi] = a * c - b * s, b * c + a * s
    mag[..., lo] = mag[..., hi] = a.abs() + b.abs()
    return y, mag


def need_scale(amax: float) -> float:
    """The smallest power of two s >= 2^-100 with amax <= 448 s."""
    e = -100
    while e < 120 and amax > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def code(x):
    """float64 to the value of the nearest e4m3 code (ties to even), |x| > 448 and infinities to 448; NaN stays."""
    x = x.clamp(-448.0, 448.0)
    _, e = torch.frexp(torch.where(torch.isfinite(x), x, torch.zeros_like(x)))
    ulp = torch.pow(torch.tensor(2.0, dtype=torch.float64), (e.clamp(min=-5) - 4).double())
    return torch.round(x / ulp) * ulp


def finite_amax(x):
    a = torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x))
    return float(a.max()) if a.numel() else 0.0


class Cache:
    """The cache's state as float64 / lists on the CPU, changed by the operators' definitions."""

    def __init__(self, c):
        self.T = c.page_tokens
        self.k, self.v = c.k.cpu().double(), c.v.cpu().double()
        self.ks, self.vs = c.k_scale.cpu().double(), c.v_scale.cpu().double()
        self.table, self.length, self.refs = c.table.cpu().clone(), c.length.cpu().tolist(), c.refs.cpu().tolist()

    def take(self):
        p = self.refs.index(0)
        self.refs[p] = 1
        return p

    def extend(self, seqs, counts):
        for s, n in zip(seqs, counts):
            for j in range(-(-self.length[s] // self.T), -(-(self.length[s] + n) // self.T)):
                self.table[s, j] = self.take()
            self.length[s] += n

    def fork(self, src, dst):
        T = self.T
        for a, b in zip(src, dst):
            for j in range(self.length[a] // T):
                self.table[b, j] = self.table[a, j]
                self.refs[int(self.table[a, j])] += 1
            self.length[b] = self.length[a]
        for a, b in zip(src, dst):
            if self.length[a] % T:
                j, p = self.length[a] // T, self.take()
                f = int(self.table[a, j])
                self.table[b, j] = p
                for x in (self.k, self.v, self.ks, self.vs):
                    x[:, p] = x[:, f]

    def release(self, seqs):
        for s in seqs:
            for j, p in enumerate(self.table[s].tolist()):
                if p >= 0:
                    self.refs[p] -= 1
                    self.table[s, j] = -1
            self.length[s] = 0

    def append(self, layer, k, v, seqs, row_off):
        T = self.T
        for i, s in enumerate(seqs):
            r, end = row_off[i], self.length[s]
            p = end - (row_off[i + 1] - row_off[i])
            while p < end:
                o, page = p % T, int(self.table[s, p // T])
                m = min(T - o, end - p)
                for codes, scales, x in ((self.k, self.ks, k), (self.v, self.vs, v)):
                    new = x[r:r + m].double().cpu()  # [m, H, D]
                    for h in range(new.shape[1]):
                        was = float(scales[layer, page, h])
                        now = need_scale(finite_amax(new[:, h]))
                        if o:
                            now = max(now, was)
                            if now > was:
                                codes[layer, page, h, :o] = code(codes[layer, page, h, :o] * (was / now))
                        codes[layer, page, h, o:o + m] = code(new[:, h] / now)
                        scales[layer, page, h] = now
                p, r = p + m, r + m

    def kept(self, i, s, keep, keep_off):
        n = min(keep_off[i + 1] - keep_off[i], self.length[s])
        return [p for p in range(self.length[s]) if p >= n or keep[keep_off[i] + p]]

    def compact(self, seqs, keep, keep_off, layers):
        T, gone = self.T, []
        for i, s in enumerate(seqs):
            at = self.kept(i, s, keep, keep_off)
            lead = 0
            while at[lead * T:(lead + 1) * T] == list(range(lead * T, (lead + 1) * T)):
                lead += 1
            old = self.table[s].tolist()
            gone += old[lead:-(-self.length[s] // T)]
            self.table[s, lead:] = -1
            for j in range(lead, -(-len(at) // T)):
                page, mine = self.take(), at[j * T:(j + 1) * T]
                self.table[s, j] = page
                pg = torch.tensor([old[p // T] for p in mine])
                sl = torch.tensor([p % T for p in mine])
                for layer in range(*layers):
                    for codes, scales in ((self.k, self.ks), (self.v, self.vs)):
                        x = codes[layer, pg, :, sl] * scales[layer, pg][..., None]  # [m, H, D]
                        for h in range(x.shape[1]):
                            now = need_scale(finite_amax(x[:, h]))
                            codes[layer, page, h, :len(mine)] = code(x[:, h] / now)
                            scales[layer, page, h] = now
            self.length[s] = len(at)
        for p in gone:
            self.refs[p] -= 1

    def attend(self, layer, q, seqs, row_off, scale=0.0, causal=True, keep=None, keep_off=None):
        """(out, lse, bound of out without its rounding, bound of lse) in float64.

        The bounds. A score's error is at most (dim + 8) fp32 roundings of the
        sum of its terms' magnitudes, and the exponential's 2^-20: d. A
        probability is rounded to f16: 2^-11 relative, or 2^-25 of the running
        maximum's, where v's scale may be 2^6 under the reference it is held in.
        """
        q = q.double().cpu()
        rows, H, D = q.shape
        G = H // self.k.shape[2]
        scale = scale or 1.0 / math.sqrt(D)
        out = torch.zeros((rows, H, D), dtype=torch.float64)
        lse = torch.full((rows, H), -math.inf, dtype=torch.float64)
        out_tol, lse_tol = torch.zeros_like(out), torch.zeros_like(lse)
        for i, s in enumerate(seqs):
            n, ln = row_off[i + 1] - row_off[i], self.length[s]
            if n == 0:
                continue
            pg = self.table[s, :-(-ln // self.T)].long()
            seen = torch.zeros(ln, dtype=torch.bool)
            seen[self.kept(i, s, keep, keep_off) if keep is not None else slice(None)] = True
            limit = (ln - n + torch.arange(n) + 1) if causal else torch.full((n,), ln)
            see = seen & (torch.arange(ln) < limit[:, None])
            for h in range(H):
                K = (self.k[layer, pg, h // G] * self.ks[layer, pg, h // G][:, None, None]).reshape(-1, D)[:ln]
                V = (self.v[layer, pg, h // G] * self.vs[layer, pg, h // G][:, None, None]).reshape(-1, D)[:ln]
                a = slice(row_off[i], row_off[i + 1])
                x = (q[a, h] @ torch.where(seen[:, None], K, torch.zeros_like(K)).T) * scale
                x = torch.where(see, x, torch.full_like(x, -math.inf))
                m = x.amax(-1, keepdim=True)
                m = torch.where(m == -math.inf, torch.zeros_like(m), m)
                p = torch.exp(x - m)
                l = p.sum(-1, keepdim=True)
                Vz = torch.where(torch.isnan(V), torch.zeros_like(V), V)
                o = torch.where(l > 0, p / l, p) @ torch.where(seen[:, None], Vz, torch.zeros_like(V))
                bad = (see.double() @ torch.isnan(V).double()) > 0
                out[a, h] = torch.where(bad, torch.full_like(o, math.nan), o)
                lse[a, h] = (m + torch.log(l))[:, 0]
                Ka = torch.where(seen[:, None], K, torch.zeros_like(K)).nan_to_num().abs()
                mass = (q[a, h].abs() @ Ka.T * scale).amax(-1, keepdim=True)
                d = (D + 8) * 2.0 ** -23 * mass + 2.0 ** -20
                Va = torch.where(seen[:, None], Vz.abs(), torch.zeros_like(V))
                pn = torch.where(l > 0, p / l, p)
                out_tol[a, h] = (2.0 ** -11 + 2 * d) * (pn.nan_to_num() @ Va) + 2.0 ** -19 * (see.double() @ Va) / l.clamp(min=1.0)
                lse_tol[a, h] = d[:, 0] + 2.0 ** -20 + 2.0 ** -22 * lse[a, h].nan_to_num(0, 0, 0).abs()
        return out, lse, out_tol, lse_tol


def assert_codes(c, ref):
    """A PagedCache equals the reference state exactly."""
    assert torch.equal(c.table.cpu(), ref.table)
    assert c.length.cpu().tolist() == ref.length
    assert c.refs.cpu().tolist() == ref.refs
    for got, want in ((c.k, ref.k), (c.v, ref.v), (c.k_scale, ref.ks), (c.v_scale, ref.vs)):
        torch.testing.assert_close(got.cpu().double(), want, rtol=0, atol=0, equal_nan=True)
