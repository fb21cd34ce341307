"""The operators around a paged key/value cache, as cases that can be timed and compared.

Four kinds, all through s3.KVCache:
  append   keys and values of new tokens into their pages, rotated on the way; the queries of the same tokens rotated; the
           signatures of the pages that were written
  attend   attention of the new tokens over everything in their pages (a decoding step, or a chunk of a prompt)
  select   the blocks (pages) that each tile of queries will read, chosen by the signatures
  blocks   attention over the listed blocks only

Shapes are those of this repository's configurations: 32 query heads over 8 key/value heads and 28 over 4, d_head 128,
chunks of 2048 and contexts of 32768 to 131072 tokens, and the tests' d_head 64 and 256 and fp32; the rest is generic serving.

Cache layout (E elements are 16 bytes): keys [n_pages, n_kv, d/E, P, E], values [n_pages, n_kv, P/E, d, E].
"""
from __future__ import annotations

import math
import random

import torch

own = False
DEV = "cuda"
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


# ------------------------------------------------------------------------------------------------ the cases
def _case(name, kind, new, kv, hq=32, hkv=8, d=128, P=64, dtype="bf16", **more):
    """new, kv: "n" for one sequence, "lo:hi:n" for n sequences spread over a range (evenly in the logarithm)."""
    return {"name": name, "kind": kind, "new": new, "kv": kv, "hq": hq, "hkv": hkv, "d": d, "P": P, "dtype": dtype, **more}


def listed():
    return [
        # one decoding step of a serving batch: 64 sequences, a token each, queries rotated in the same call
        _case("append_decode", "append", "1:1:64", "100:2000:64", rot=128, inter=False),
        # prefill: eight prompts bring a chunk of 2048 tokens each
        _case("append_chunk", "append", "2048:2048:8", "2048:4000:8", rot=128, inter=False),
        # fp32, small heads, small pages, ragged chunks, half of the channels rotated, pairs side by side
        _case("append_fp32_ragged", "append", "3:777:5", "800:1500:5", hq=8, hkv=8, d=64, P=16, dtype="fp32", rot=32, inter=True),
        # one user, one token, a short context: latency
        _case("attend_one_short", "attend", "1", "1000"),
        # a serving batch with contexts from a few hundred tokens to 32768
        _case("attend_decode_ragged", "attend", "1:1:64", "300:32768:64"),
        # the last chunk of a prompt of 131072 tokens: the largest
        _case("attend_chunk_131k", "attend", "2048", "131072"),
        # three prompts of the 28:4 configuration in one call, chunks of odd lengths, one of them nearly finished
        _case("attend_chunk_ragged", "attend", "37:2048:3", "5001:32768:3", hq=28, hkv=4),
        # fp32, wide heads, small pages, a chunk that is the whole prompt
        _case("attend_fp32_d256", "attend", "333", "333", hq=8, hkv=2, d=256, P=16, dtype="fp32"),
        # choice of 32 blocks of 64 tokens for a batch of decoding steps at long contexts
        _case("select_decode", "select", "1:1:64", "8000:32768:64", qb=1, top=32),
        # choice for each 16 queries of a chunk at the end of 131072 tokens
        _case("select_chunk", "select", "2048", "131072", qb=16, top=64),
        # the decoding steps that read those 32 blocks
        _case("blocks_decode", "blocks", "1:1:64", "8000:32768:64", qb=1, top=32),
        # a chunk whose tiles of 64 queries read 64 blocks each
        _case("blocks_chunk", "blocks", "2048", "131072", qb=64, top=64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "attend", "attend", "attend", "select", "blocks", "blocks"])
    hq, hkv = rng.choice([(32, 8), (32, 8), (28, 4), (8, 8), (16, 1), (16, 2)])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    d = rng.choice([64, 128, 128, 128, 256])
    P = rng.choice([16, 32, 64, 64, 128, 256])
    decode = rng.random() < 0.5
    if decode:
        n = _log(rng, 1, 96)
        new = "1:1:%d" % n if rng.random() < 0.7 else "1:%d:%d" % (rng.randint(2, 8), n)
        top = max(64, min(131072, 2_000_000 * 4 * 128 // (n * hkv * d)))
    else:
        n = rng.choice([1, 1, 2, 4])
        hi = _log(rng, 20, 2048)
        new = "%d:%d:%d" % (rng.randint(1, hi), hi, n)
        top = min(131072, 4_000_000 * 32 * 128 // (n * hq * d)) // (8 if dtype == "fp32" else 1)
    kv_hi = _log(rng, 64, top)
    kv = "%d:%d:%d" % (max(1, kv_hi // rng.randint(1, 30)), kv_hi, n)
    c = {"kind": kind, "new": new, "kv": kv, "hq": hq, "hkv": hkv, "d": d, "P": P, "dtype": dtype}
    if kind == "append":
        c.update(rot=rng.choice([d, d, d // 2, 0]), inter=rng.random() < 0.3)
    if kind in ("select", "blocks"):
        qb = 1 if decode else rng.choice([1, 16, 16, 32, 64, 128])
        c.update(qb=qb, top=3 + qb // P + _log(rng, 4, 96))
    if kind == "attend" and rng.random() < 0.2:
        c["window"] = _log(rng, 1, 4096)
    return c


def _spread(text):
    """Whole numbers spread over lo..hi evenly in the logarithm, in an order that mixes short and long."""
    p = [int(x) for x in text.split(":")]
    if len(p) == 1:
        return p
    lo, hi, n = p
    out = [hi if i == n - 1 else int(round(lo * (hi / lo) ** (i / max(n - 1, 1)))) for i in range(n)]
    random.Random(n).shuffle(out)
    return out


def _lens(case):
    new, kv = _spread(case["new"]), _spread(case["kv"])
    return new, [max(a, b) for a, b in zip(new, kv)]


def _tiles(case):
    return sum(-(-n // case["qb"]) for n in _lens(case)[0])


# ------------------------------------------------------------------------------------------------ inputs
def _grid8(x):
    """A vector on its 8 bit grid: whole multiples (at most 128) of a power of two, zero where it is too small or too large."""
    m = x.abs().amax(-1, keepdim=True)
    e = torch.frexp(m)[1] - 7
    ok = (m >= 2.0 ** -40) & (m < 2.0 ** 50)
    e = torch.where(ok, e, torch.zeros_like(e))
    return torch.where(ok, torch.ldexp(torch.round(torch.ldexp(x, -e)), e), torch.zeros_like(x))


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    new, kv = _lens(case)
    hq, hkv, d, P, dt = case["hq"], case["hkv"], case["d"], case["P"], DT[case["dtype"]]
    E = 16 // dt.itemsize
    n_seq, T = len(new), sum(new)
    blocks = [-(-n // P) for n in kv]
    n_pages, width = sum(blocks) + 3, max(blocks) + 1
    perm = torch.randperm(n_pages, generator=g, device=DEV, dtype=torch.int64).to(torch.int32)     # pages in no order
    table = torch.full((n_seq, width), -1, dtype=torch.int32, device=DEV)
    at = 0
    for s, n in enumerate(blocks):
        table[s, :n] = perm[at:at + n]
        at += n
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    st = {"case": case, "table": table, "kv_len": torch.tensor(kv, dtype=torch.int32, device=DEV),
          "q_start": torch.tensor(starts, dtype=torch.int32, device=DEV), "T": T, "new": new, "kv": kv}

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32)

    # channels of unequal size with two outliers, as keys have them
    chan = torch.exp(0.25 * normal(hkv, d))
    chan[:, :2] *= 4.0
    if T and case["kind"] == "append":
        # one projection's output: queries, keys and values of a token side by side
        w = (hq + 2 * hkv) * d
        qkv = normal(T, hq + 2 * hkv, d)
        qkv[:, hq:hq + hkv] *= chan
        qkv = qkv.to(dt).view(T, w)
        st["qkv"] = qkv
    if case["kind"] != "select":
        kc = torch.empty(n_pages, hkv, d // E, P, E, dtype=dt, device=DEV)
        vc = torch.empty(n_pages, hkv, P // E, d, E, dtype=dt, device=DEV)
        for p in range(0, n_pages, 1024):
            m = min(1024, n_pages - p)
            kc[p:p + m] = normal(m, hkv, d // E, P, E) * chan.view(1, hkv, d // E, 1, E)
            vc[p:p + m] = normal(m, hkv, P // E, d, E)
        st["k"], st["v"] = kc, vc
    if case["kind"] in ("append", "select"):
        st["sig"] = _grid8(normal(n_pages, hkv, d) * chan * 0.2).to(torch.bfloat16)
    if case["kind"] != "append":
        st["q"] = normal(T, hq, d).to(dt)
    if case["kind"] == "append" and case["rot"]:
        r = case["rot"]
        ang = torch.arange(max(kv), device=DEV, dtype=torch.float64)[:, None] * \
            10000.0 ** (-torch.arange(0, r, 2, device=DEV, dtype=torch.float64) / r)
        st["rope"] = torch.cat([ang.cos(), ang.sin()], 1).to(torch.float32)
    if case["kind"] == "blocks":
        # first block, the tile's own blocks, and others anywhere before them, in ascending order
        qb, top = case["qb"], case["top"]
        sel = torch.full((max(1, (T + n_seq * (qb - 1)) // qb), hkv, top), -1, dtype=torch.int32, device=DEV)
        t = 0
        for s in range(n_seq):
            for i in range(0, new[s], qb):
                p0 = kv[s] - new[s] + i
                lo, hi = p0 // P, (min(p0 + qb, kv[s]) - 1) // P
                own_blocks = hi - lo + 1
                n = min(top, hi + 1)
                key = torch.rand(hkv, hi + 1, generator=g, device=DEV)
                key[:, lo:] = 3.0
                key[:, 0] = 2.0 if lo else 3.0
                assert own_blocks <= top
                sel[t, :, :n] = key.topk(n, dim=1).indices.sort(dim=1).values.to(torch.int32)
                t += 1
        st["sel"] = sel
    if own:
        import paper_2601_17702_amd as s3
        st["cache"] = s3.KVCache(n_pages, P, hkv, d, dt, signatures="sig" in st, k=st.get("k"), v=st.get("v"),
                                 sig=st.get("sig"))
    return st


# ------------------------------------------------------------------------------------------------ one pass
def run(st):
    case = st["case"]
    return (_own if own else _plain)[case["kind"]](st, case)


def _split(st, case):
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    x = st["qkv"].view(st["T"], hq + 2 * hkv, d)
    return x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]


def _own_append(st, case):
    c = st["cache"]
    q, k, v = _split(st, case)
    qr = c.append(k, v, st["kv_len"], st["table"], q_start=st["q_start"], rope=st.get("rope"), interleaved=case["inter"], q=q)
    return {"k": c.k, "v": c.v, "sig": c.sig, "q": qr}


def _own_attend(st, case):
    o, lse = st["cache"].attention(st["q"], st["kv_len"], st["table"], q_start=st["q_start"], max_new=max(st["new"]),
                                   max_kv=max(st["kv"]), window=case.get("window", 0), want_lse=True)
    return {"o": o, "lse": lse}


def _own_select(st, case):
    return st["cache"].select(st["q"], st["kv_len"], st["table"], case["top"], q_start=st["q_start"], q_block=case["qb"],
                              lead=1, tail=1, max_kv=max(st["kv"]))


def _own_blocks(st, case):
    o, lse = st["cache"].block_attention(st["q"], st["kv_len"], st["table"], st["sel"], q_start=st["q_start"],
                                         q_block=case["qb"], want_lse=True)
    return {"o": o, "lse": lse}


_own = {"append": _own_append, "attend": _own_attend, "select": _own_select, "blocks": _own_blocks}


def _rotate(x, st, case, pos):
    """x [T, heads, d] in the storage type -> fp32 rotated and rounded to it."""
    r = case["rot"]
    if not r:
        return x
    cs = st["rope"][pos]
    c, s = cs[:, None, :r // 2], cs[:, None, r // 2:]
    y = x.to(torch.float32)
    if case["inter"]:
        a, b = y[..., 0:r:2], y[..., 1:r:2]
    else:
        a, b = y[..., :r // 2], y[..., r // 2:r]
    a2, b2 = a * c - b * s, b * c + a * s
    if case["inter"]:
        y = torch.cat([torch.stack([a2, b2], -1).flatten(-2), y[..., r:]], -1)
    else:
        y = torch.cat([a2, b2, y[..., r:]], -1)
    return y.to(x.dtype)


def _plain_append(st, case):
    hkv, d, P = case["hkv"], case["d"], case["P"]
    kc, vc, sig = st["k"], st["v"], st["sig"]
    E = kc.shape[-1]
    q, k, v = _split(st, case)
    T = st["T"]
    tok = torch.arange(T, device=DEV, dtype=torch.int32)
    seq = torch.searchsorted(st["q_start"][1:], tok, right=True)
    pos = (st["kv_len"][seq] - (st["q_start"][seq + 1] - tok)).long()
    page, slot = st["table"][seq, pos // P].long(), pos % P
    kc[page, :, :, slot] = _rotate(k, st, case, pos).reshape(T, hkv, d // E, E)
    vc[page, :, slot // E, :, slot % E] = v
    # the last new token of every page written: its page's keys, summed by slot % 8 and joined in pairs
    last = torch.ones(T, dtype=torch.bool, device=DEV)
    last[:-1] = page[1:] != page[:-1]
    at = last.nonzero().flatten()
    for part in at.split(4096):
        n = slot[part] + 1
        x = kc[page[part]].transpose(2, 3).reshape(len(part), hkv, P, d).to(torch.float32)
        x = torch.where((torch.arange(P, device=DEV)[None, :] < n[:, None])[:, None, :, None], x, torch.zeros_like(x))
        x = x.view(len(part), hkv, P // 8, 8, d)
        m = x[:, :, 0]
        for i in range(1, P // 8):
            m = m + x[:, :, i]
        m = m[:, :, 0::2] + m[:, :, 1::2]
        m = m[:, :, 0::2] + m[:, :, 1::2]
        m = (m[:, :, 0] + m[:, :, 1]) / n.to(torch.float32)[:, None, None]
        sig[page[part]] = _grid8(m).to(torch.bfloat16)
    return {"k": kc, "v": vc, "sig": sig, "q": _rotate(q, st, case, pos).contiguous()}


def _tokens(cache, pages, keys):
    """[hkv, n, d] fp32 of whole pages, in order."""
    x = cache[pages.long()]
    x = x.permute(1, 0, 3, 2, 4) if keys else x.permute(1, 0, 2, 4, 3)
    hkv, n = x.shape[0], x.shape[1]
    return x.reshape(hkv, n * cache.shape[3] if keys else n * cache.shape[2] * cache.shape[4], -1).to(torch.float32)


def _softmax_v(q, k, v, rowpos, keypos, scale, window):
    """q [R, d], k, v [n, d] fp32; rowpos [R], keypos [n].  Returns o [R, d], lse [R]; slabs of rows bound the memory."""
    o, lse = torch.empty_like(q), torch.empty(q.shape[0], device=DEV, dtype=torch.float32)
    step = max(1, (1 << 28) // max(1, k.shape[0]))
    for r in range(0, q.shape[0], step):
        x = (q[r:r + step] @ k.t()) * scale
        hide = keypos[None, :] > rowpos[r:r + step, None]
        if window:
            hide = hide | (keypos[None, :] <= rowpos[r:r + step, None] - window)
        x.masked_fill_(hide, -math.inf)
        m = x.amax(1, keepdim=True)
        x = torch.exp(x.sub_(m))
        z = x.sum(1, keepdim=True)
        o[r:r + step] = (x @ v) / z
        lse[r:r + step] = (m + torch.log(z)).flatten()
    return o, lse


def _plain_attend(st, case):
    hq, hkv, d, P = case["hq"], case["hkv"], case["d"], case["P"]
    G = hq // hkv
    q = st["q"]
    out, lse = torch.empty_like(q), torch.empty(st["T"], hq, device=DEV, dtype=torch.float32)
    at = 0
    for s, (n, kv) in enumerate(zip(st["new"], st["kv"])):
        if n == 0:
            continue
        pages = st["table"][s, :-(-kv // P)]
        k, v = _tokens(st["k"], pages, True)[:, :kv], _tokens(st["v"], pages, False)[:, :kv]
        x = q[at:at + n].to(torch.float32).view(n, hkv, G, d)
        keypos = torch.arange(kv, device=DEV)
        rowpos = torch.arange(kv - n, kv, device=DEV).repeat_interleave(G)
        for h in range(hkv):
            o, l = _softmax_v(x[:, h].reshape(n * G, d), k[h], v[h], rowpos, keypos, d ** -0.5, case.get("window", 0))
            out[at:at + n, h * G:(h + 1) * G] = o.view(n, G, d).to(q.dtype)
            lse[at:at + n, h * G:(h + 1) * G] = l.view(n, G)
        at += n
    return {"o": out, "lse": lse}


def _rows(st, first, m, hkv, G, d):
    """Rows of a tile per key/value head: [hkv, m * G, d] fp32."""
    return st["q"][first:first + m].to(torch.float32).view(m, hkv, G, d).transpose(0, 1).reshape(hkv, m * G, d)


def _plain_select(st, case):
    hq, hkv, d, P, qb, top = (case[x] for x in ("hq", "hkv", "d", "P", "qb", "top"))
    G = hq // hkv
    n_seq = len(st["new"])
    sel = torch.full((max(1, (st["T"] + n_seq * (qb - 1)) // qb), hkv, top), -1, dtype=torch.int32, device=DEV)
    at = t = 0
    for s, (n, kv) in enumerate(zip(st["new"], st["kv"])):
        sig = st["sig"][st["table"][s, :-(-kv // P)].long()].to(torch.float32)          # [blocks, hkv, d]
        for i in range(0, n, qb):
            m = min(qb, n - i)
            p0, p1 = kv - n + i, kv - n + i + m - 1
            nb = p1 // P + 1
            rows = _grid8(_rows(st, at + i, m, hkv, G, d))
            score = torch.stack([(rows[h] @ sig[:nb, h].t()).amax(0) for h in range(hkv)])
            score[:, :1] = math.inf                                                       # the first block, and the tile's own
            score[:, p0 // P:] = math.inf
            keep = min(top, nb)
            pick = torch.sort(score, dim=1, descending=True, stable=True).indices[:, :keep]
            sel[t, :, :keep] = torch.sort(pick, dim=1).values.to(torch.int32)
            t += 1
        at += n
    return sel


def _plain_blocks(st, case):
    hq, hkv, d, P, qb = (case[x] for x in ("hq", "hkv", "d", "P", "qb"))
    G = hq // hkv
    out, lse = torch.empty_like(st["q"]), torch.empty(st["T"], hq, device=DEV, dtype=torch.float32)
    at = t = 0
    for s, (n, kv) in enumerate(zip(st["new"], st["kv"])):
        for i in range(0, n, qb):
            m = min(qb, n - i)
            rows = _rows(st, at + i, m, hkv, G, d)
            rowpos = torch.arange(kv - n + i, kv - n + i + m, device=DEV).repeat_interleave(G)
            count = min(case["top"], (kv - n + i + m - 1) // P + 1)
            for h in range(hkv):
                ids = st["sel"][t, h, :count].long()
                keypos = (ids[:, None] * P + torch.arange(P, device=DEV)).flatten()
                pages = st["table"][s, ids].long()
                k = st["k"][pages, h].transpose(1, 2).reshape(-1, d).to(torch.float32)
                v = st["v"][pages, h].transpose(2, 3).reshape(-1, d).to(torch.float32)
                o, l = _softmax_v(rows[h], k, v, rowpos, keypos, d ** -0.5, 0)
                out[at + i:at + i + m, h * G:(h + 1) * G] = o.view(m, G, d).to(out.dtype)
                lse[at + i:at + i + m, h * G:(h + 1) * G] = l.view(m, G)
            t += 1
        at += n
    return {"o": out, "lse": lse}


_plain = {"append": _plain_append, "attend": _plain_attend, "select": _plain_select, "blocks": _plain_blocks}


# ------------------------------------------------------------------------------------------------ what a pass needs
def work(case):
    new, kv = _lens(case)
    hq, hkv, d, P = case["hq"], case["hkv"], case["d"], case["P"]
    es = DT[case["dtype"]].itemsize
    T = sum(new)
    if case["kind"] == "append":
        old = sum((b - a) % P for a, b in zip(new, kv) if a)             # keys of the first page that were there before
        pages = sum(-(-b // P) - (b - a) // P for a, b in zip(new, kv) if a)
        rot = case["rot"]
        return {"bytes": T * 2 * (hq + 2 * hkv) * d * es + T * rot * 4 + old * hkv * d * es + pages * hkv * d * 2,
                "flops": T * (hq + hkv) * rot * 3 + (T + old) * hkv * d}
    if case["kind"] == "select":
        qb, top = case["qb"], case["top"]
        flops = 0
        for a, b in zip(new, kv):
            for i in range(0, a, qb):
                m = min(qb, a - i)
                flops += 2 * d * m * hq * ((b - a + i + m - 1) // P + 1)
        blocks = sum(-(-b // P) for a, b in zip(new, kv) if a)
        return {"bytes": T * hq * d * es + blocks * hkv * d * 2 + _tiles(case) * hkv * top * 4, "flops": flops}
    io = T * hq * (2 * d * es + 4)
    if case["kind"] == "attend":
        w = case.get("window", 0)
        pairs = tokens = 0
        for a, b in zip(new, kv):
            if not a:
                continue
            first = b - a + 1                                             # keys that the first new token sees
            if w and first >= w:
                pairs += a * w
            elif w and b > w:
                pairs += (first + w) * (w - first + 1) // 2 + (b - w) * w
            else:
                pairs += (first + b) * a // 2
            tokens += min(b, a + w - 1) if w else b
        return {"bytes": io + tokens * hkv * 2 * d * es, "flops": 4 * d * hq * pairs}
    qb, top = case["qb"], case["top"]
    pairs = union = 0
    for a, b in zip(new, kv):
        lists = 0
        for i in range(0, a, qb):
            m = min(qb, a - i)
            n = min(top, (b - a + i + m - 1) // P + 1)
            lists += n
            pairs += m * n * P
        union += min(lists, -(-b // P)) * P if a else 0
    return {"bytes": io + union * hkv * 2 * d * es + _tiles(case) * hkv * top * 4, "flops": 4 * d * hq * pairs}


# ------------------------------------------------------------------------------------------------ the definition, in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    new, kv = st["new"], st["kv"]
    hq, hkv, d, P = case["hq"], case["hkv"], case["d"], case["P"]
    G = hq // hkv
    D = torch.float64
    where = []                                                            # (sequence, position) of every new token
    for s in range(len(new)):
        where += [(s, p) for p in range(kv[s] - new[s], kv[s])]
    if case["kind"] == "append":
        E, r = st["k"].shape[-1], case["rot"]
        seq = torch.tensor([w[0] for w in where], device=DEV)
        pos = torch.tensor([w[1] for w in where], device=DEV)
        x = st["qkv"].to(D).view(len(where), hq + 2 * hkv, d)
        if r:
            i = torch.arange(r // 2, device=DEV)
            ia, ib = (2 * i, 2 * i + 1) if case["inter"] else (i, i + r // 2)
            z = torch.complex(st["rope"][pos, :r // 2].to(D), st["rope"][pos, r // 2:].to(D))
            y = torch.complex(x[:, :hq + hkv, ia], x[:, :hq + hkv, ib]) * z[:, None]
            x[:, :hq + hkv, ia], x[:, :hq + hkv, ib] = y.real, y.imag
        k64, v64 = st["k"].to(D), st["v"].to(D)
        flat = (st["table"][seq, pos.div(P, rounding_mode="floor")].long() * hkv)[:, None, None] + \
            torch.arange(hkv, device=DEV)[None, :, None]                  # page and head
        ch = torch.arange(d, device=DEV)[None, None, :]
        sl = pos.remainder(P)[:, None, None]
        k64.view(-1)[(flat * (d // E) + ch // E) * (P * E) + sl * E + ch % E] = x[:, hq:hq + hkv]
        v64.view(-1)[(flat * (P // E) + sl // E) * (d * E) + ch * E + sl % E] = x[:, hq + hkv:]
        return {"k": k64, "v": v64, "sig": None, "q": x[:, :hq].contiguous()}

    if case["kind"] == "select":
        qb, top = case["qb"], case["top"]
        sel = torch.full((max(1, (st["T"] + len(new) * (qb - 1)) // qb), hkv, top), -1, dtype=torch.int32)
        row = t = 0
        for s in range(len(new)):
            sig = st["sig"].to(D)[st["table"][s].long().clamp(min=0)].transpose(0, 1)     # [hkv, blocks, d]
            for i in range(0, new[s], qb):
                m = min(qb, new[s] - i)
                p0 = kv[s] - new[s] + i
                nb = (p0 + m - 1) // P + 1
                x = st["q"][row + i:row + i + m].to(D)
                big = x.abs().amax(-1, keepdim=True)
                unit = torch.exp2(torch.floor(torch.log2(big.clamp(min=2.0 ** -60))) - 6)
                x = torch.where((big >= 2.0 ** -40) & (big < 2.0 ** 50), torch.round(x / unit) * unit, 0.0 * x)
                for h in range(hkv):
                    a = (x[:, h * G:(h + 1) * G].reshape(-1, d) @ sig[h, :nb].t()).amax(0)
                    must = {0} | set(range(p0 // P, nb))
                    order = torch.argsort(a, descending=True, stable=True).tolist()
                    pick = sorted(must) + [b for b in order if b not in must]
                    pick = sorted(pick[:top])
                    sel[t, h, :len(pick)] = torch.tensor(pick, dtype=torch.int32)
                t += 1
            row += new[s]
        return sel.to(DEV)

    o = torch.zeros(st["T"], hq, d, dtype=D, device=DEV)
    lse = torch.full((st["T"], hq), -math.inf, dtype=D, device=DEV)
    row = t = 0
    for s in range(len(new)):
        n, m = new[s], kv[s]
        step = n if case["kind"] == "attend" else case["qb"]
        for i in range(0, n, max(1, step)):
            c = min(step, n - i)
            for h in range(hkv):
                at = torch.arange(m, device=DEV)
                if case["kind"] == "blocks":
                    ids = st["sel"][t, h]
                    at = at[torch.isin(at // P, ids[ids >= 0].long())]
                page, slot = st["table"][s, at // P].long(), at % P
                k = st["k"][page, h, :, slot].reshape(len(at), d).to(D)
                E = st["v"].shape[-1]
                v = st["v"][page, h, slot // E, :, slot % E].to(D)
                per = max(1, (1 << 27) // max(1, len(at)))
                for g in range(G):
                    for a in range(0, c, per):
                        b = min(c, a + per)
                        tok = torch.arange(i + a, i + b, device=DEV)
                        z = st["q"][row + i + a:row + i + b, h * G + g].to(D) @ k.t() / math.sqrt(d)
                        gap = (m - n + tok)[:, None] - at[None, :]
                        see = gap >= 0
                        if case.get("window"):
                            see &= gap < case["window"]
                        z = torch.where(see, z, -math.inf)
                        lse[row + i + a:row + i + b, h * G + g] = torch.logsumexp(z, 1)
                        o[row + i + a:row + i + b, h * G + g] = torch.softmax(z, 1) @ v
            t += 1
        row += n
    return {"o": o, "lse": lse}
