"""Operators of a paged key/value cache held in 8 bits, and what stands beside them, as cases that can be timed and compared.

Five kinds:
  norm     keys and values of new tokens into a bf16 or fp32 cache, keys and queries normed for each head and rotated on the way
  append8  the same into an 8-bit cache: e4m3 values, one power of two for each token and head
  attend8  attention of the new tokens over an 8-bit cache, over all of it or (with `top`) over listed blocks
  cap      attention whose scores are capped by a tanh, over caches of any type
  read     tokens of a cache back as rows: all of a sequence's, or those at given positions

Shapes are those of this repository's configurations: 32 query heads over 8 key/value heads and 28 over 4, d_head 128,
chunks of 2048 and contexts of 32768 to 131072 tokens, and the tests' d_head 64 and 256 and fp32; the rest is generic serving.

Cache layout (E elements are 16 bytes): keys [n_pages, n_kv, d/E, P, E], values [n_pages, n_kv, P/E, d, E]; an 8-bit cache's
scales [n_pages, n_kv, 2, P]: the code c of a token's key, and of its value, whose elements stand for themselves times 2^(c - 127).
"""
from __future__ import annotations

import math
import random
import struct

import torch

own = False
DEV = "cuda"
F8 = torch.float8_e4m3fn
DT = {"bf16": torch.bfloat16, "fp32": torch.float32, "e4m3": F8}
EPS = struct.unpack("f", struct.pack("f", 1e-6))[0]                 # as 32 bits hold it


# ------------------------------------------------------------------------------------------------ the cases
def _case(name, kind, new, kv, hq=32, hkv=8, d=128, P=64, dtype="bf16", **more):
    """new, kv: "n" for one sequence, "lo:hi:n" for n sequences spread over a range (evenly in the logarithm)."""
    return {"name": name, "kind": kind, "new": new, "kv": kv, "hq": hq, "hkv": hkv, "d": d, "P": P, "dtype": dtype, **more}


def listed():
    return [
        # one decoding step of a serving batch of a model with head norms: latency
        _case("norm_decode", "norm", "1:1:64", "100:2000:64", rot=128, inter=False, sig=True),
        # its prefill: four prompts of the 28:4 configuration bring odd chunks, half of the channels rotated in neighbouring pairs
        _case("norm_chunk_ragged", "norm", "517:2048:4", "2048:9000:4", hq=28, hkv=4, rot=64, inter=True, sig=True),
        # the decoding step into an 8-bit cache, with norms
        _case("append8_decode", "append8", "1:1:64", "100:2000:64", dtype="e4m3", rot=128, inter=False, norm=True, sig=True),
        # prefill into it: eight prompts bring a chunk of 2048 tokens each, no norms
        _case("append8_chunk", "append8", "2048:2048:8", "2048:4000:8", dtype="e4m3", rot=128, inter=False, norm=False, sig=True),
        # one user, one token, a short context: latency
        _case("attend8_one_short", "attend8", "1", "1000", dtype="e4m3"),
        # a serving batch with contexts from a few hundred tokens to 32768
        _case("attend8_decode_ragged", "attend8", "1:1:64", "300:32768:64", dtype="e4m3"),
        # the last chunk of a prompt of 131072 tokens: the largest
        _case("attend8_chunk_131k", "attend8", "2048", "131072", dtype="e4m3"),
        # decoding steps that read 32 chosen blocks of 64 tokens each
        _case("blocks8_decode", "attend8", "1:1:64", "8000:32768:64", dtype="e4m3", qb=1, top=32),
        # decoding with capped scores, a batch in bf16
        _case("cap_decode", "cap", "1:1:32", "500:16384:32", cap=50.0),
        # three chunks of odd lengths with capped scores, in layers that see a window of 4096
        _case("cap_chunk_window", "cap", "333:2048:3", "4001:20000:3", cap=30.0, window=4096),
        # evidence: 64 spans of 64 tokens anywhere in a context of 131072 come back as rows
        _case("read_evidence", "read", "4096", "131072", dtype="e4m3", span=64),
        # a batch's whole sequences come back, as for a copy to another cache
        _case("read_all", "read", "4096:32768:4", "4096:32768:4", dtype="e4m3", span=0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "append8", "append8", "attend8", "attend8", "attend8", "cap", "cap", "read"])
    hq, hkv = rng.choice([(32, 8), (32, 8), (28, 4), (8, 8), (16, 1), (16, 2)])
    d = rng.choice([64, 128, 128, 128, 256])
    P = rng.choice([16, 32, 64, 64, 128, 256])
    dtype = "e4m3"
    if kind == "norm":
        dtype = rng.choice(["bf16", "bf16", "fp32"])
    if kind in ("cap", "read"):
        dtype = rng.choice(["bf16", "e4m3", "fp32"])
    decode = kind != "read" and rng.random() < 0.5
    if decode:
        n = _log(rng, 1, 96)
        new = "1:1:%d" % n if rng.random() < 0.7 else "1:%d:%d" % (rng.randint(2, 8), n)
        top = max(64, min(131072, 2_000_000 * 4 * 128 // (n * hkv * d)))
    else:
        n = rng.choice([1, 1, 2, 4])
        hi = _log(rng, 20, 32768 if kind == "read" else 2048)
        new = "%d:%d:%d" % (rng.randint(1, hi), hi, n)
        top = min(131072, 4_000_000 * 32 * 128 // (n * hq * d)) // (8 if dtype == "fp32" else 1)
    kv_hi = _log(rng, 64, max(64, top))
    kv = "%d:%d:%d" % (max(1, kv_hi // rng.randint(1, 30)), kv_hi, n)
    c = {"kind": kind, "new": new, "kv": kv, "hq": hq, "hkv": hkv, "d": d, "P": P, "dtype": dtype}
    if kind in ("norm", "append8"):
        c.update(rot=rng.choice([d, d, d // 2, 0]), inter=rng.random() < 0.3, sig=rng.random() < 0.7)
    if kind == "append8":
        c.update(norm=rng.random() < 0.5)
    if kind == "cap":
        c.update(cap=rng.choice([15.0, 30.0, 50.0]))
        if rng.random() < 0.3:
            c.update(window=_log(rng, 16, 4096))
    if kind == "attend8" and rng.random() < 0.35:
        qb = 1 if decode else rng.choice([16, 32, 64, 128])
        c.update(qb=qb, top=3 + qb // P + _log(rng, 4, 96))
    elif kind == "attend8" and rng.random() < 0.2:
        c.update(window=_log(rng, 16, 4096))
    if kind == "read":
        c.update(span=rng.choice([0, 1, rng.randint(2, 100), 64]))
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


# ------------------------------------------------------------------------------------------------ inputs
def _codes(x):
    """The scale's code of every row of x [..., d] fp32: the smallest c >= 1 that leaves no finite |x| 2^(127 - c) above 448."""
    m = torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x)).amax(-1)
    u = m.view(torch.int32)
    return ((u >> 23) - 8 + ((u & 0x7fffff) > 0x600000).to(torch.int32)).clamp(min=1)


def _to8(x, codes):
    """Rows in 8 bits, as e4m3 values."""
    return (x * ((254 - codes) << 23).view(torch.float32)[..., None]).to(F8)


def _of8(x, codes):
    """The values that e4m3 elements stand for, fp32; codes [...] uint8 broadcast against x."""
    return x.to(torch.float32) * (codes.to(torch.int32) << 23).view(torch.float32)


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
    eight = dt == F8
    rows = torch.bfloat16 if eight else dt                                      # type of queries and of what comes back
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
    st = {"case": case, "table": table, "kv_len": torch.tensor(kv, dtype=torch.int32, device=DEV), "T": T, "new": new, "kv": kv,
          "q_start": torch.tensor(starts, dtype=torch.int32, device=DEV), "rows": rows,
          "starts": None if max(new) == 1 else torch.tensor(starts, dtype=torch.int32, device=DEV)}      # a step of single tokens has none

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32)

    # channels of unequal size with two outliers, as keys have them; tokens of unequal size
    chan = torch.exp(0.25 * normal(hkv, d))
    chan[:, :2] *= 4.0
    kc = torch.empty(n_pages, hkv, d // E, P, E, dtype=dt, device=DEV)
    vc = torch.empty(n_pages, hkv, P // E, d, E, dtype=dt, device=DEV)
    scale = torch.empty(n_pages, hkv, 2, P, dtype=torch.uint8, device=DEV) if eight else None
    for p in range(0, n_pages, 1024):
        m = min(1024, n_pages - p)
        for x, keys in ((normal(m, hkv, P, d) * chan[None, :, None], True), (normal(m, hkv, P, d), False)):
            x = x * torch.exp(0.4 * normal(m, hkv, P, 1))
            if eight:
                c = _codes(x)
                scale[p:p + m, :, 0 if keys else 1] = c.to(torch.uint8)
                x = _to8(x, c).view(torch.uint8)
            if keys:
                kc[p:p + m].view(torch.uint8 if eight else dt).copy_(x.view(m, hkv, P, d // E, E).transpose(2, 3))
            else:
                vc[p:p + m].view(torch.uint8 if eight else dt).copy_(x.view(m, hkv, P // E, E, d).transpose(3, 4))
    st.update(k=kc, v=vc, scale=scale)
    if case["kind"] in ("norm", "append8"):
        # one projection's output: queries, keys and values of a token side by side
        w = (hq + 2 * hkv) * d
        qkv = normal(T, hq + 2 * hkv, d) * torch.exp(0.4 * normal(T, hq + 2 * hkv, 1))
        qkv[:, hq:hq + hkv] *= chan
        st["qkv"] = qkv.to(rows).view(T, w)
        if case.get("norm", True):
            st["q_norm"], st["k_norm"] = 1.0 + 0.2 * normal(d), 1.0 + 0.2 * normal(d)
        if case["sig"]:
            st["sig"] = _grid8(normal(n_pages, hkv, d) * chan * 0.2).to(torch.bfloat16)
        if case["rot"]:
            r = case["rot"]
            ang = torch.arange(max(kv), device=DEV, dtype=torch.float64)[:, None] * \
                10000.0 ** (-torch.arange(0, r, 2, device=DEV, dtype=torch.float64) / r)
            st["rope"] = torch.cat([ang.cos(), ang.sin()], 1).to(torch.float32)
    if case["kind"] in ("attend8", "cap"):
        # where a cap is, scores reach it
        st["q"] = (normal(T, hq, d) * (8.0 if case["kind"] == "cap" else 1.0)).to(rows)
    if case.get("span"):
        # spans of tokens anywhere in their sequence, in ascending order, as the choice of evidence gives them
        span = case["span"]
        pos = []
        for n, m in zip(new, kv):
            count = -(-n // span)
            begin = (torch.rand(count, generator=g, device=DEV) * max(1, m - span + 1)).to(torch.int64).sort().values
            pos.append((begin[:, None] + torch.arange(span, device=DEV)).flatten()[:n].clamp(max=m - 1))
        st["pos"] = torch.cat(pos).to(torch.int32)
    if "top" in case:
        # first block, the tile's own blocks, and others anywhere before them, in ascending order
        qb, top = case["qb"], case["top"]
        sel = torch.full((max(1, (T + n_seq * (qb - 1)) // qb), hkv, top), -1, dtype=torch.int32, device=DEV)
        t = 0
        for s in range(n_seq):
            for i in range(0, new[s], qb):
                p0 = kv[s] - new[s] + i
                lo, hi = p0 // P, (min(p0 + qb, kv[s]) - 1) // P
                assert hi - lo + 1 <= top
                n = min(top, hi + 1)
                key = torch.rand(hkv, hi + 1, generator=g, device=DEV)
                key[:, lo:] = 3.0
                key[:, 0] = 2.0 if lo else 3.0
                sel[t, :, :n] = key.topk(n, dim=1).indices.sort(dim=1).values.to(torch.int32)
                t += 1
        st["sel"] = sel
    if own:
        import paper_2601_17702_amd as s3
        more = {"k": kc, "v": vc, "sig": st.get("sig"), "signatures": "sig" in st}
        st["cache"] = s3.KVCache8(n_pages, P, hkv, d, scale=scale, **more) if eight else s3.KVCache(n_pages, P, hkv, d, dt, **more)
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
    qr = c.append(k, v, st["kv_len"], st["table"], q_start=st["starts"], rope=st.get("rope"), interleaved=case["inter"], q=q,
                  q_norm=st.get("q_norm"), k_norm=st.get("k_norm"), eps=EPS, max_new=max(st["new"]))
    return {"k": c.k, "v": c.v, "scale": st["scale"], "sig": c.sig, "q": qr}


def _own_attend(st, case):
    same = {"q_start": st["starts"], "max_new": max(st["new"]), "max_kv": max(st["kv"]), "want_lse": True}
    if "cap" in case:
        same["softcap"] = case["cap"]
    if "top" in case:
        o, lse = st["cache"].block_attention(st["q"], st["kv_len"], st["table"], st["sel"], q_block=case["qb"], **same)
    else:
        o, lse = st["cache"].attention(st["q"], st["kv_len"], st["table"], window=case.get("window", 0), **same)
    return {"o": o, "lse": lse}


def _own_read(st, case):
    k, v = st["cache"].read(st["kv_len"], st["table"], st["T"], q_start=st["starts"], positions=st.get("pos"))
    return {"k": k, "v": v}


_own = {"norm": _own_append, "append8": _own_append, "attend8": _own_attend, "cap": _own_attend, "read": _own_read}


def _place(st, pos=None):
    """Of every row: its sequence's page and the slot in it, and its position."""
    tok = torch.arange(st["T"], device=DEV, dtype=torch.int32)
    seq = torch.searchsorted(st["q_start"][1:], tok, right=True)
    if pos is None:
        pos = st["kv_len"][seq] - (st["q_start"][seq + 1] - tok)
    pos = pos.long()
    P = st["case"]["P"]
    return st["table"][seq, pos // P].long(), pos % P, pos


def _normed(x, w):
    """x [T, heads, d] fp32 over the root of its mean square (that in 64 bits), times w, every product rounded to 32 bits."""
    if w is None:
        return x
    inv = (1.0 / torch.sqrt(x.to(torch.float64).square().mean(-1, keepdim=True) + EPS)).to(torch.float32)
    return (x * inv) * w


def _rotated(y, st, case, pos):
    """y [T, heads, d] fp32 -> rotated, every product and sum rounded to 32 bits."""
    r = case["rot"]
    if not r:
        return y
    cs = st["rope"][pos]
    c, s = cs[:, None, :r // 2], cs[:, None, r // 2:]
    a, b = (y[..., 0:r:2], y[..., 1:r:2]) if case["inter"] else (y[..., :r // 2], y[..., r // 2:r])
    a2, b2 = a * c - b * s, b * c + a * s
    turned = torch.stack([a2, b2], -1).flatten(-2) if case["inter"] else torch.cat([a2, b2], -1)
    return torch.cat([turned, y[..., r:]], -1)


def _plain_append(st, case):
    hkv, d, P = case["hkv"], case["d"], case["P"]
    kc, vc, scale, sig = st["k"], st["v"], st["scale"], st.get("sig")
    E = kc.shape[-1]
    q, k, v = _split(st, case)
    page, slot, pos = _place(st)
    T = st["T"]
    q = _rotated(_normed(q.to(torch.float32), st.get("q_norm")), st, case, pos).to(st["rows"])
    k = _rotated(_normed(k.to(torch.float32), st.get("k_norm")), st, case, pos)
    kb, vb = kc, vc
    if scale is not None:
        v = v.to(torch.float32)
        ck, cv = _codes(k), _codes(v)
        k, v = _to8(k, ck).view(torch.uint8), _to8(v, cv).view(torch.uint8)
        kb, vb = kc.view(torch.uint8), vc.view(torch.uint8)
        scale[page, :, 0, slot] = ck.to(torch.uint8)
        scale[page, :, 1, slot] = cv.to(torch.uint8)
    kb[page, :, :, slot] = k.to(kb.dtype).reshape(T, hkv, d // E, E)
    vb[page, :, slot // E, :, slot % E] = v.to(vb.dtype)
    if sig is not None:
        # the last new token of every page written: its page's keys, summed by slot % 8 and joined in pairs
        last = torch.ones(T, dtype=torch.bool, device=DEV)
        last[:-1] = page[1:] != page[:-1]
        at = last.nonzero().flatten()
        n, pg = slot[at] + 1, page[at]
        x = kb[pg].transpose(2, 3).reshape(len(at), hkv, P, d)
        x = x.to(torch.float32) if scale is None else _of8(x.view(F8), scale[pg, :, 0][..., None])
        x = torch.where((torch.arange(P, device=DEV)[None, :] < n[:, None])[:, None, :, None], x, torch.zeros_like(x))
        x = x.view(len(at), hkv, P // 8, 8, d)
        m = x[:, :, 0]
        for i in range(1, P // 8):
            m = m + x[:, :, i]
        m = m[:, :, 0::2] + m[:, :, 1::2]
        m = m[:, :, 0::2] + m[:, :, 1::2]
        m = (m[:, :, 0] + m[:, :, 1]) / n.to(torch.float32)[:, None, None]
        sig[pg] = _grid8(m).to(torch.bfloat16)
    return {"k": kc, "v": vc, "scale": scale, "sig": sig, "q": q.contiguous()}


def _tokens(st, pages):
    """Keys and values of whole pages in order, [hkv, n, d] fp32; pages [hkv or 1, blocks]."""
    eight = st["scale"] is not None
    byte = torch.uint8 if eight else st["k"].dtype
    head = torch.arange(st["k"].shape[1], device=DEV)[:, None]
    k = st["k"].view(byte)[pages, head].transpose(2, 3).flatten(3).flatten(1, 2)
    v = st["v"].view(byte)[pages, head].transpose(3, 4).flatten(1, 3)
    if eight:
        c = st["scale"][pages, head].transpose(1, 2).flatten(2)[:, :, :, None]
        return _of8(k.view(F8), c[:, 0]), _of8(v.view(F8), c[:, 1])
    return k.to(torch.float32), v.to(torch.float32)


def _softmax_v(q, k, v, rowpos, keypos, case):
    """q [hkv, R, d], k, v [hkv, n, d] fp32; rowpos [R], keypos [hkv or 1, n].  Returns o [hkv, R, d], lse [hkv, R]; slabs of rows bound the memory."""
    o, lse = torch.empty_like(q), torch.empty(q.shape[:2], device=DEV, dtype=torch.float32)
    step = max(1, (1 << 30) // max(1, k.shape[0] * k.shape[1]))
    kt = k.transpose(1, 2)
    keypos = keypos.view(-1, 1, k.shape[1])
    for r in range(0, q.shape[1], step):
        x = torch.matmul(q[:, r:r + step], kt) * case["d"] ** -0.5
        if "cap" in case:
            x = case["cap"] * torch.tanh(x / case["cap"])
        at = rowpos[None, r:r + step, None]
        hide = keypos > at
        if case.get("window"):
            hide = hide | (keypos <= at - case["window"])
        x.masked_fill_(hide, -math.inf)
        m = x.amax(2, keepdim=True)
        x = torch.exp(x.sub_(m))
        z = x.sum(2, keepdim=True)
        o[:, r:r + step] = torch.matmul(x, v) / z
        lse[:, r:r + step] = (m + torch.log(z)).squeeze(2)
    return o, lse


def _plain_attend(st, case):
    hq, hkv, d, P = case["hq"], case["hkv"], case["d"], case["P"]
    G, q = hq // hkv, st["q"]
    out, lse = torch.empty_like(q), torch.empty(st["T"], hq, device=DEV, dtype=torch.float32)
    row = t = 0
    for n, kv, table in zip(st["new"], st["kv"], st["table"]):
        step = case.get("qb", n)
        for i in range(0, n, step):
            m = min(step, n - i)
            blocks = torch.arange(-(-kv // P), device=DEV)[None]
            if "top" in case:
                blocks = st["sel"][t, :, :min(case["top"], (kv - n + i + m - 1) // P + 1)].long()
            k, v = _tokens(st, table[blocks].long())
            keypos = (blocks[:, :, None] * P + torch.arange(P, device=DEV)).flatten(1)      # those past the end are beyond every row
            x = q[row + i:row + i + m].to(torch.float32).view(m, hkv, G, d).transpose(0, 1).reshape(hkv, m * G, d)
            rowpos = torch.arange(kv - n + i, kv - n + i + m, device=DEV).repeat_interleave(G)
            o, z = _softmax_v(x, k, v, rowpos, keypos, case)
            out[row + i:row + i + m] = o.view(hkv, m, G, d).transpose(0, 1).reshape(m, hq, d).to(q.dtype)
            lse[row + i:row + i + m] = z.view(hkv, m, G).transpose(0, 1).reshape(m, hq)
            t += 1
        row += n
    return {"o": out, "lse": lse}


def _plain_read(st, case):
    page, slot, _ = _place(st, st.get("pos"))
    T, hkv, d = st["T"], case["hkv"], case["d"]
    E = st["k"].shape[-1]
    eight = st["scale"] is not None
    byte = torch.uint8 if eight else st["k"].dtype
    k = st["k"].view(byte)[page, :, :, slot].reshape(T, hkv, d)
    v = st["v"].view(byte)[page, :, slot // E, :, slot % E].reshape(T, hkv, d)
    if eight:
        k = _of8(k.view(F8), st["scale"][page, :, 0, slot][..., None]).to(torch.bfloat16)
        v = _of8(v.view(F8), st["scale"][page, :, 1, slot][..., None]).to(torch.bfloat16)
    return {"k": k, "v": v}


_plain = {"norm": _plain_append, "append8": _plain_append, "attend8": _plain_attend, "cap": _plain_attend, "read": _plain_read}


# ------------------------------------------------------------------------------------------------ what a pass needs
def work(case):
    new, kv = _lens(case)
    hq, hkv, d, P = case["hq"], case["hkv"], case["d"], case["P"]
    es = DT[case["dtype"]].itemsize
    rs = 2 if es == 1 else es                                             # of a row's element outside the cache
    per = hkv * 2 * (d * es + (es == 1))                                  # a token in the cache
    T = sum(new)
    if case["kind"] in ("norm", "append8"):
        old = sum((b - a) % P for a, b in zip(new, kv)) if case["sig"] else 0      # keys of the first page that were there before
        pages = sum(-(-b // P) - (b - a) // P for a, b in zip(new, kv)) if case["sig"] else 0
        rot, norm = case["rot"], case.get("norm", True)
        return {"bytes": T * ((2 * hq + 2 * hkv) * d * rs + per) + T * rot * 4 + old * hkv * d * es + pages * hkv * d * 2,
                "flops": T * (hq + hkv) * (rot * 3 + norm * d * 4) + (T + old) * hkv * d + (es == 1) * T * hkv * d * 4}
    if case["kind"] == "read":
        if case["span"]:
            return {"bytes": T * (per + 4 + 2 * hkv * d * rs), "flops": T * hkv * 2 * d * (es == 1)}
        return {"bytes": T * (per + 2 * hkv * d * rs), "flops": T * hkv * 2 * d * (es == 1)}
    io = T * hq * (2 * d * rs + 4)
    pairs = tokens = lists = 0
    for a, b in zip(new, kv):
        first = b - a + 1                                                 # keys that the first new token sees
        if "top" in case:
            mine = 0
            for i in range(0, a, case["qb"]):
                m, p0 = min(case["qb"], a - i), b - a + i
                n = min(case["top"], (p0 + m - 1) // P + 1)
                behind = n * P - min(n * P, max(0, n * P - (-(p0 + m) % P)))         # slots of the last block that the tile's last row does not see
                pairs += m * (n * P - behind) - m * (m - 1) // 2
                mine += n
            lists += mine * hkv
            tokens += min(mine * P, b)
            continue
        w = case.get("window", 0)
        if w and first >= w:
            pairs += a * w
        elif w and b > w:
            pairs += (first + w) * (w - first + 1) // 2 + (b - w) * w
        else:
            pairs += (first + b) * a // 2
        tokens += min(b, a + w - 1) if w else b
    return {"bytes": io + tokens * per + lists * 4, "flops": 4 * d * hq * pairs}


# ------------------------------------------------------------------------------------------------ the definition, in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    new, kv = st["new"], st["kv"]
    hq, hkv, d, P = case["hq"], case["hkv"], case["d"], case["P"]
    G = hq // hkv
    D = torch.float64
    E = st["k"].shape[-1]
    eight = case["dtype"] == "e4m3"

    def fetch(s, at):
        """Keys and values [n, hkv, d] of positions `at` of sequence s, in 64 bits."""
        page, slot = st["table"][s, at // P].long(), at % P
        raw = st["k"].view(torch.uint8) if eight else st["k"]
        k = raw[page, :, :, slot].reshape(len(at), hkv, d).contiguous().view(st["k"].dtype).to(D)
        raw = st["v"].view(torch.uint8) if eight else st["v"]
        v = raw[page, :, slot // E, :, slot % E].contiguous().view(st["v"].dtype).to(D)
        if eight:
            two = torch.exp2(st["scale"][page, :, :, slot].to(D) - 127.0)
            k, v = k * two[:, :, 0, None], v * two[:, :, 1, None]
        return k, v

    if case["kind"] == "read":
        ks, vs, row = [], [], 0
        for s in range(len(new)):
            at = st["pos"][row:row + new[s]].long() if "pos" in st else torch.arange(kv[s] - new[s], kv[s], device=DEV)
            k, v = fetch(s, at)
            ks.append(k)
            vs.append(v)
            row += new[s]
        return {"k": torch.cat(ks), "v": torch.cat(vs)}

    if case["kind"] in ("norm", "append8"):
        where = [(s, p) for s in range(len(new)) for p in range(kv[s] - new[s], kv[s])]
        r = case["rot"]
        seq = torch.tensor([w[0] for w in where], device=DEV)
        pos = torch.tensor([w[1] for w in where], device=DEV)
        x = st["qkv"].to(D).view(len(where), hq + 2 * hkv, d)
        if "q_norm" in st:
            w = torch.cat([st["q_norm"].to(D).expand(hq, d), st["k_norm"].to(D).expand(hkv, d)])
            y = x[:, :hq + hkv]
            x = torch.cat([y / torch.sqrt((y * y).sum(-1, keepdim=True) / d + EPS) * w, x[:, hq + hkv:]], 1)
        if r:
            i = torch.arange(r // 2, device=DEV)
            ia, ib = (2 * i, 2 * i + 1) if case["inter"] else (i, i + r // 2)
            z = torch.complex(st["rope"][pos, :r // 2].to(D), st["rope"][pos, r // 2:].to(D))
            y = torch.complex(x[:, :hq + hkv, ia], x[:, :hq + hkv, ib]) * z[:, None]
            x = x.clone()
            x[:, :hq + hkv, ia], x[:, :hq + hkv, ib] = y.real, y.imag
        k, v = x[:, hq:hq + hkv], x[:, hq + hkv:]
        if eight:                                                         # what 8 bits hold: a power of two puts the largest into (224, 448]
            k, v = (y / torch.exp2(torch.ceil(torch.log2(y.abs().amax(-1, keepdim=True) / 448.0))) for y in (k, v))
        k64, v64 = st["k"].to(D), st["v"].to(D)
        flat = (st["table"][seq, pos.div(P, rounding_mode="floor")].long() * hkv)[:, None, None] + \
            torch.arange(hkv, device=DEV)[None, :, None]                  # page and head
        ch = torch.arange(d, device=DEV)[None, None, :]
        sl = pos.remainder(P)[:, None, None]
        k64.view(-1)[(flat * (d // E) + ch // E) * (P * E) + sl * E + ch % E] = k
        v64.view(-1)[(flat * (P // E) + sl // E) * (d * E) + ch * E + sl % E] = v
        return {"k": k64, "v": v64, "scale": None, "sig": None, "q": x[:, :hq].contiguous()}

    o = torch.zeros(st["T"], hq, d, dtype=D, device=DEV)
    lse = torch.full((st["T"], hq), -math.inf, dtype=D, device=DEV)
    row = t = 0
    for s in range(len(new)):
        n, m = new[s], kv[s]
        step = case.get("qb", n)
        K, V = fetch(s, torch.arange(m, device=DEV))
        for i in range(0, n, step):
            c = min(step, n - i)
            for h in range(hkv):
                at = torch.arange(m, device=DEV)
                if "sel" in st:
                    ids = st["sel"][t, h]
                    at = at[torch.isin(at // P, ids[ids >= 0].long())]
                k, v = K[at, h], V[at, h]
                per = max(1, (1 << 27) // max(1, len(at)))
                for g in range(G):
                    for a in range(0, c, per):
                        b = min(c, a + per)
                        tok = torch.arange(i + a, i + b, device=DEV)
                        z = st["q"][row + i + a:row + i + b, h * G + g].to(D) @ k.t() / math.sqrt(d)
                        if "cap" in case:
                            z = case["cap"] * torch.tanh(z / case["cap"])
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
