"""Plain forms of what stands beside the paged cache: rows in 8 bits, head norms, capped scores, tokens read back.  On the CPU, apart from the library."""
import math

import numpy as np
import torch

from tests import paged

F64 = torch.float64


def _values():
    """The 127 e4m3 values that are not negative, by their bits."""
    out = []
    for u in range(127):
        e, m = u >> 3, u & 7
        out.append(m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))
    return np.array(out)


VALUES = _values()


def to8(x):
    """x [..., d] (fp32 values) -> (bytes uint8 [..., d], codes uint8 [...]), in 64 bits: the smallest power of two from 2^-126 on that leaves nothing
    finite above 448; elements to the nearest value, ties to even bits; NaN (0x7f) where x is not finite."""
    x = np.asarray(x, np.float64)
    fine = np.isfinite(x)
    m = np.max(np.where(fine, np.abs(x), 0.0), axis=-1)
    c = np.ones(m.shape, np.int64)
    some = m > 448 * 2.0 ** -126
    e = np.frexp(m[some] / 448.0)                         # m / 448 = f 2^e with f in [0.5, 1): 2^e >= m / 448; 2^(e - 1) only where f = 0.5
    c[some] = e[1] + 127 - (m[some] <= np.ldexp(448.0, e[1] - 1))
    y = np.where(fine, np.abs(x), 0.0) * np.ldexp(1.0, 127 - c)[..., None]
    hi = np.searchsorted(VALUES, y, side="left").clip(max=126)
    lo = np.maximum(hi - 1, 0)
    up, down = VALUES[hi] - y, y - VALUES[lo]
    bits = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    bits = bits | np.where(np.signbit(x), 128, 0)
    return np.where(fine, bits, 0x7f).astype(np.uint8), c.astype(np.uint8)


def of8(bits, codes):
    """What they stand for, in 64 bits."""
    v = np.where((bits & 127) == 127, np.nan, VALUES[np.minimum(bits & 127, 126)]) * np.where(bits & 128, -1.0, 1.0)
    return v * np.ldexp(1.0, codes.astype(np.int64) - 127)[..., None]


class Problem8(paged.Problem):
    """A problem whose rows are what an 8-bit cache stands for: rows_k and rows_v hold the dequantised values (exact in bf16), bytes and codes beside them."""

    def __init__(self, seed, d, P, hq, hkv, new, kv, spare=3, scale=1.0, spread=1.0):
        super().__init__(seed, "bf16", d, P, hq, hkv, new, kv, spare=spare, scale=scale)
        self.quantise(spread)

    def quantise(self, spread=0.0):
        self.bytes = {"k": [], "v": []}
        self.codes = {"k": [], "v": []}
        for name, rows in (("k", self.rows_k), ("v", self.rows_v)):
            for s, x in enumerate(rows):
                size = torch.exp(spread * torch.randn(x.shape[0], x.shape[1], 1, generator=self.g)) if spread else 1.0
                b, c = to8((x.to(F64) * size).numpy())
                self.bytes[name].append(b)
                self.codes[name].append(c)
                rows[s] = torch.from_numpy(of8(b, c)).to(torch.bfloat16).reshape(x.shape)

    def pack8(self, garbage=True):
        """k, v, scale as a cache holds them; slots that no sequence has reached hold NaN and the code 255."""
        d, P, hkv = self.d, self.P, self.hkv
        k = np.full((self.n_pages, hkv, d // 16, P, 16), 0x7f if garbage else 0, np.uint8)
        v = np.full((self.n_pages, hkv, P // 16, d, 16), 0xff if garbage else 0, np.uint8)
        scale = np.full((self.n_pages, hkv, 2, P), 255 if garbage else 1, np.uint8)
        for s in range(self.n_seq):
            for p in range(self.kv[s]):
                if not self.mapped(s, p):
                    continue
                page, slot = int(self.table[s, p // P]), p % P
                k[page, :, :, slot] = self.bytes["k"][s][p].reshape(hkv, d // 16, 16)
                v[page, :, slot // 16, :, slot % 16] = self.bytes["v"][s][p]
                scale[page, :, 0, slot] = self.codes["k"][s][p]
                scale[page, :, 1, slot] = self.codes["v"][s][p]
        return k, v, scale

    def cache(self, signatures=False, sig=None, garbage=True):
        import paper_2601_17702_amd as s3
        k, v, scale = (torch.from_numpy(x).cuda() for x in self.pack8(garbage))
        f8 = torch.float8_e4m3fn
        return s3.KVCache8(self.n_pages, self.P, self.hkv, self.d, signatures=signatures, k=k.view(f8), v=v.view(f8), scale=scale,
                           sig=None if sig is None else sig.cuda())


def problem(dtype, seed, d, P, hq, hkv, new, kv, garbage=float("nan"), **more):
    return Problem8(seed, d, P, hq, hkv, new, kv, **more) if dtype == "e4m3" else paged.Problem(seed, dtype, d, P, hq, hkv, new, kv, garbage=garbage, **more)


def attend(pr, cap, window=0, scale=None, sel=None, qb=None):
    """As paged.attend, with scores cap * tanh(score / cap).  The score's own error shrinks with tanh's slope, at most 1; tanh is good to 2^-20 of the
    capped score, which the bounds take for its largest.  Over rows of bf16 and with caps up to 2048 a score comes as 2 cap r - cap, r = 1 / (1 + exp(-2 z)) in
    (0, 1): r is off by half a unit of its reciprocal (2^-24) and by r (1 - r) <= 1/4 of its exponential's relative error (2^-22 with its argument's rounding, 2^-24
    |2 z| log2(e) r (1 - r) being less), so by less than 2^-23, and the score by 2^-22 of the cap."""
    scale = pr.d ** -0.5 if scale is None else scale
    G, T = pr.hq // pr.hkv, pr.T
    out = torch.zeros(T, pr.hq, pr.d, dtype=F64)
    lse = torch.full((T, pr.hq), -math.inf, dtype=F64)
    tol, ltol = torch.zeros(T, pr.hq, pr.d, dtype=F64), torch.zeros(T, pr.hq, dtype=F64)
    row = tile = 0
    bf = pr.dtype == torch.bfloat16
    for s in range(pr.n_seq):
        n, m = pr.new[s], pr.kv[s]
        ok = torch.tensor([pr.mapped(s, p) for p in range(m)], dtype=torch.bool)
        at = torch.arange(m)
        K, V = pr.rows_k[s].to(F64), pr.rows_v[s].to(F64)
        for i in range(n):
            pos = m - n + i
            see = ok & (at <= pos)
            if window:
                see &= at > pos - window
            for h in range(pr.hkv):
                times = torch.ones(m, dtype=torch.long)
                if sel is not None:
                    ids = [int(b) for b in sel[tile + i // qb, h] if b >= 0]
                    times = torch.tensor([ids.count(p // pr.P) for p in range(m)])
                idx = torch.repeat_interleave(at, times * see)
                if len(idx) == 0:
                    continue
                k, v = K[idx, h], V[idx, h]
                q = pr.q[row + i, h * G:(h + 1) * G].to(F64)
                z = cap * torch.tanh(q @ k.t() * scale / cap)
                p = torch.softmax(z, 1)
                o = p @ v
                out[row + i, h * G:(h + 1) * G] = o
                lse[row + i, h * G:(h + 1) * G] = torch.logsumexp(z, 1)
                e = (pr.d * 2.0 ** -24 * scale * (q.abs() @ k.abs().t()) + 2.0 ** -20 * z.abs() + 2.0 ** -23 * z.abs()).amax(1) + 2.0 ** -21
                if bf and cap <= 2048:
                    e = e + 2.0 ** -22 * cap
                rel = 2 * e + len(idx) * 2.0 ** -24 + (2.0 ** -8 if bf else 0.0)
                tol[row + i, h * G:(h + 1) * G] = rel[:, None] * (p @ v.abs()) + (2.0 ** -8 if bf else 2.0 ** -24) * o.abs() * 1.01
                ltol[row + i, h * G:(h + 1) * G] = e + len(idx) * 2.0 ** -24 + 2.0 ** -22 * lse[row + i, h * G:(h + 1) * G].abs()
        row += n
        if qb:
            tile += -(-n // qb)
    return out, lse, tol, ltol


def norm(x, w, eps):
    """x [..., d] fp32 over the root of its mean square plus eps (64 bits, its inverse rounded to fp32), times w: every product rounded to fp32."""
    with np.errstate(all="ignore"):
        ms = np.sum(x.astype(np.float64) ** 2, axis=-1, keepdims=True) / x.shape[-1] + np.float64(np.float32(eps))
        r = (1.0 / np.sqrt(ms)).astype(np.float32)
        return (x * r) * w


def rotate(x, table, rot, inter):
    """x [heads, d] fp32 by one row of the rotation's table, every product and sum rounded to fp32."""
    x = x.copy()
    if rot:
        c, s = table[:rot // 2], table[rot // 2:]
        a, b = (slice(0, rot, 2), slice(1, rot, 2)) if inter else (slice(0, rot // 2), slice(rot // 2, rot))
        u, v = x[:, a].copy(), x[:, b].copy()
        with np.errstate(all="ignore"):
            x[:, a], x[:, b] = u * c - v * s, v * c + u * s
    return x


def round_to(x, dtype):
    return torch.from_numpy(np.ascontiguousarray(x)).to(dtype)
