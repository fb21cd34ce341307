"""Plain 64-bit forms of the paged-cache operators, on the CPU, token by token and head by head, and the problems that the tests
draw.  Nothing here is shared with the library."""
import math

import numpy as np
import torch

F64 = torch.float64
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


class Problem:
    """A ragged batch over a paged cache: tensors on the CPU in the storage type, `.cuda()` copies on demand."""

    def __init__(self, seed, dtype, d, P, hq, hkv, new, kv, spare=3, scale=1.0, garbage=None):
        g = torch.Generator().manual_seed(seed)
        self.g, self.dtype, self.d, self.P, self.hq, self.hkv, self.new, self.kv = g, DTYPES[dtype], d, P, hq, hkv, list(new), list(kv)
        self.E = 16 // self.dtype.itemsize
        self.T, self.n_seq = sum(new), len(new)
        blocks = [-(-n // P) for n in kv]
        self.n_pages = sum(blocks) + spare
        self.table = torch.full((self.n_seq, max(blocks + [1]) + 1), -1, dtype=torch.int32)
        perm = torch.randperm(self.n_pages, generator=g).to(torch.int32)
        at = 0
        for s, n in enumerate(blocks):
            self.table[s, :n] = perm[at:at + n]
            at += n
        self.kv_len = torch.tensor(kv, dtype=torch.int32)
        self.q_start = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32)
        self.q = (torch.randn(self.T, hq, d, generator=g) * scale).to(self.dtype)
        # tokens' keys and values as rows; slots that no sequence has reached hold `garbage`
        self.rows_k = [(torch.randn(n, hkv, d, generator=g) * scale).to(self.dtype) for n in kv]
        self.rows_v = [torch.randn(n, hkv, d, generator=g).to(self.dtype) for n in kv]
        self.garbage = garbage

    def pack(self):
        """(k, v) cache arrays that hold rows_k and rows_v."""
        fill = 0.0 if self.garbage is None else self.garbage
        k = torch.full((self.n_pages, self.hkv, self.d // self.E, self.P, self.E), fill, dtype=self.dtype)
        v = torch.full((self.n_pages, self.hkv, self.P // self.E, self.d, self.E), fill, dtype=self.dtype)
        for s in range(self.n_seq):
            for p in range(self.kv[s]):
                if not self.mapped(s, p):
                    continue
                page = int(self.table[s, p // self.P])
                slot = p % self.P
                k[page, :, :, slot] = self.rows_k[s][p].view(self.hkv, self.d // self.E, self.E)
                v[page, :, slot // self.E, :, slot % self.E] = self.rows_v[s][p]
        return k, v

    def cache(self, signatures=False, sig=None):
        import paper_2601_17702_amd as s3
        k, v = self.pack()
        return s3.KVCache(self.n_pages, self.P, self.hkv, self.d, self.dtype, signatures=signatures, k=k.cuda(), v=v.cuda(),
                          sig=None if sig is None else sig.cuda())

    def args(self):
        return self.kv_len.cuda(), self.table.cuda()

    def mapped(self, s, p):
        b = p // self.P
        return b < self.table.shape[1] and 0 <= int(self.table[s, b]) < self.n_pages

    def tiles(self, qb):
        return (self.T + self.n_seq * (qb - 1)) // qb


def attend(pr, window=0, scale=None, sel=None, qb=None):
    """(out, lse, bound of |error| of out, bound of lse's) in 64 bits, from the rows.  A row's masked tokens do not enter at all.

    Bounds, first order: a score is a sum of d products in 32 bits, off by at most d 2^-24 sum|q k| scale =: e, one more
    rounding of its scaled value, up to 2^-24 (|s| + |m|), and exp2 is good to 2^-22; weights and their sum are off by the relative
    sum of these, the sum of n weights by n 2^-24 more.  With bf16 a weight is rounded once more (2^-8, half a unit of 8 significant bits) and so is the result (2^-8 |o|)."""
    scale = pr.d ** -0.5 if scale is None else scale
    G, T = pr.hq // pr.hkv, pr.T
    out = torch.zeros(T, pr.hq, pr.d, dtype=F64)
    lse = torch.full((T, pr.hq), -math.inf, dtype=F64)
    tol = torch.zeros(T, pr.hq, pr.d, dtype=F64)
    ltol = torch.zeros(T, pr.hq, dtype=F64)
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
                for g in range(G):
                    qr = pr.q[row + i, h * G + g].to(F64)
                    z = (k @ qr) * scale
                    p = torch.softmax(z, 0)
                    o = (p[:, None] * v).sum(0)
                    out[row + i, h * G + g] = o
                    lse[row + i, h * G + g] = torch.logsumexp(z, 0)
                    e = float((pr.d * 2.0 ** -24 * scale * (k.abs() @ qr.abs()) + 2.0 ** -23 * z.abs()).max()) + 2.0 ** -21
                    rel = 2 * e + len(idx) * 2.0 ** -24 + (2.0 ** -8 if bf else 0.0)
                    tol[row + i, h * G + g] = rel * (p[:, None] * v.abs()).sum(0) + (2.0 ** -8 if bf else 2.0 ** -24) * o.abs() * 1.01
                    ltol[row + i, h * G + g] = e + len(idx) * 2.0 ** -24 + 2.0 ** -22 * abs(float(lse[row + i, h * G + g]))
        row += n
        if qb:
            tile += -(-n // qb)
    return out, lse, tol, ltol


def check(pr, got, lse, want):
    out, l64, tol, ltol = want
    got, lse = got.cpu().to(F64), lse.cpu().to(F64)
    empty = torch.isinf(l64) & (l64 < 0)
    assert torch.equal(torch.isinf(lse) & (lse < 0), empty)
    assert torch.all(got[empty] == 0)
    odd = ~torch.isfinite(out)
    assert torch.equal(torch.isnan(got), torch.isnan(out)) and torch.equal(got[odd & ~torch.isnan(out)], out[odd & ~torch.isnan(out)])
    err = (got - out).abs()
    bad = ~odd & (err > tol)
    assert not bad.any(), (int(bad.sum()), float((err / tol.clamp(min=1e-300))[bad].max()), bad.nonzero()[0].tolist())
    lerr = (lse - l64).abs()[~empty]
    assert torch.all(lerr <= ltol[~empty]), float((lerr / ltol[~empty]).max())


def grid8(x):
    """Rounding to whole multiples of 2^(floor(log2 max|x|) - 6), a vector at a time, in 64 bits."""
    x = np.asarray(x, dtype=np.float64)
    out = np.zeros_like(x)
    for i in np.ndindex(x.shape[:-1]):
        m = np.max(np.abs(x[i]))
        if np.isfinite(m) and 2.0 ** -40 <= m < 2.0 ** 50:
            unit = 2.0 ** (np.floor(np.log2(m)) - 6)
            out[i] = np.rint(x[i] / unit) * unit
    return out


def signature(rows):
    """The signature of a page that holds these keys [n, d]: fp32 partial sums in the documented order, then the 8 bit grid."""
    rows = rows.to(torch.float32).numpy()
    part = [np.zeros(rows.shape[1], np.float32) for _ in range(8)]
    for t in range(rows.shape[0]):
        part[t % 8] = part[t % 8] + rows[t]
    m = (((part[0] + part[1]) + (part[2] + part[3])) + ((part[4] + part[5]) + (part[6] + part[7]))) / np.float32(rows.shape[0])
    return grid8(m.astype(np.float32))


def select(pr, sig, top, qb, lead, tail):
    """sel [tiles, hkv, top] from signatures [n_pages, hkv, d], in 64 bits."""
    G = pr.hq // pr.hkv
    sel = np.full((pr.tiles(qb), pr.hkv, top), -1, np.int32)
    row = t = 0
    for s in range(pr.n_seq):
        n, m = pr.new[s], pr.kv[s]
        for i in range(0, n, qb):
            c = min(qb, n - i)
            p0, p1 = m - n + i, m - n + i + c - 1
            cand = [b for b in range(p1 // pr.P + 1) if pr.mapped(s, b * pr.P)] if p1 >= 0 else []
            for h in range(pr.hkv):
                q = grid8(pr.q[row + i:row + i + c, h * G:(h + 1) * G].to(F64).numpy().reshape(c * G, pr.d))
                keyed = []
                for b in cand:
                    forced = b < lead or (tail > 0 and b >= max(p0, 0) // pr.P - tail + 1)
                    score = np.max(q @ sig[int(pr.table[s, b]), h].to(F64).numpy())
                    keyed.append((0 if forced else 1, -score, b))
                pick = sorted(b for _, _, b in sorted(keyed)[:top])
                sel[t, h, :len(pick)] = pick
            t += 1
        row += n
    return sel
