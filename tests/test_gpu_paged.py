"""GPU checks of the paged key/value cache against plain 64-bit forms (tests/paged.py): append with rotation and signatures,
attention over all blocks, block selection, attention over listed blocks."""
import numpy as np
import pytest
import torch

from tests import paged

pytestmark = pytest.mark.gpu

SHAPES = [   # dtype, d, P, hq, hkv, new, kv
    ("bf16", 128, 64, 32, 8, [1], [1]),                               # the first token of all
    ("bf16", 128, 64, 32, 8, [1, 1, 1], [63, 64, 65]),                # around a page's end
    ("bf16", 128, 16, 28, 4, [5, 0, 33, 1], [5, 0, 40, 17]),          # seven query heads a head, a sequence without tokens
    ("bf16", 64, 32, 8, 8, [70], [300]),                              # one query head a head
    ("bf16", 256, 128, 16, 1, [3, 9], [129, 9]),                      # sixteen, wide heads
    ("bf16", 128, 256, 32, 1, [2], [513]),                            # thirty-two
    ("bf16", 64, 16, 4, 2, [130], [1000]),
    ("bf16", 128, 64, 8, 2, [100, 1, 1, 7], [350, 1, 700, 7]),         # chunks beside single tokens
    ("fp32", 64, 16, 8, 4, [1, 20], [31, 33]),
    ("fp32", 128, 64, 6, 2, [67], [200]),
    ("fp32", 256, 32, 4, 2, [1, 40], [100, 65]),
    ("bf16", 256, 64, 4, 2, [150], [150]),                            # a whole prompt
    ("bf16", 128, 32, 4, 1, [300], [301]),
    ("bf16", 128, 64, 4, 1, [70], [9000]),                            # the tokens of a row tile in parts
    ("fp32", 64, 64, 4, 2, [200, 3], [700, 2000]),
    ("fp32", 128, 32, 4, 2, [90], [1500]),
    ("bf16", 64, 64, 32, 1, [3, 1], [900, 40]),                       # 96 rows of three tokens
]


@pytest.mark.parametrize("dtype,d,P,hq,hkv,new,kv", SHAPES)
def test_attention(dtype, d, P, hq, hkv, new, kv):
    pr = paged.Problem(len(kv) + d + P, dtype, d, P, hq, hkv, new, kv, garbage=float("nan"))
    kv_len, table = pr.args()
    want = paged.attend(pr)
    c = pr.cache()
    o, lse = c.attention(pr.q.cuda(), kv_len, table, q_start=pr.q_start.cuda(), want_lse=True)
    paged.check(pr, o, lse, want)
    # the bounds a host program knows only share out the work
    o2, lse2 = c.attention(pr.q.cuda(), kv_len, table, q_start=pr.q_start.cuda(), max_new=max(new), max_kv=max(kv), want_lse=True)
    paged.check(pr, o2, lse2, want)
    o3, _ = c.attention(pr.q.cuda(), kv_len, table, q_start=pr.q_start.cuda(), max_new=max(new), max_kv=max(kv))
    assert torch.equal(o2, o3)                                        # the same bits every time


@pytest.mark.parametrize("dtype,d,P,hq,hkv,new,kv,window", [
    ("bf16", 128, 64, 8, 2, [1, 1], [500, 3], 100),
    ("bf16", 64, 16, 8, 2, [90], [400], 1),                           # itself only
    ("bf16", 128, 32, 4, 2, [100], [130], 33),
    ("fp32", 128, 16, 4, 2, [50, 1], [170, 90], 48),
])
def test_attention_window(dtype, d, P, hq, hkv, new, kv, window):
    pr = paged.Problem(window + d, dtype, d, P, hq, hkv, new, kv, garbage=float("inf"))
    kv_len, table = pr.args()
    o, lse = pr.cache().attention(pr.q.cuda(), kv_len, table, q_start=pr.q_start.cuda(), window=window, want_lse=True)
    paged.check(pr, o, lse, paged.attend(pr, window=window))


@pytest.mark.parametrize("dtype,new,window", [("bf16", 1, 0), ("bf16", 1, 40), ("bf16", 90, 0), ("bf16", 90, 30), ("fp32", 70, 50), ("fp32", 2, 300)])
def test_sequences_longer_than_their_table(dtype, new, window):
    """Tokens whose block lies behind the table's last one are masked; positions and windows are still those of the whole sequence."""
    pr = paged.Problem(18, dtype, 64, 16, 4, 2, [new, 3], [250, 20])
    pr.table = pr.table[:, :13].contiguous()                          # 208 of 250 positions
    kv_len, table = pr.args()
    o, lse = pr.cache().attention(pr.q.cuda(), kv_len, table, q_start=pr.q_start.cuda(), window=window, want_lse=True)
    paged.check(pr, o, lse, paged.attend(pr, window=window))


@pytest.mark.parametrize("new,kv", [([1, 1], [2000, 5]), ([40, 40], [100, 2000]), ([200], [1500])])
def test_attention_of_large_scores(new, kv):
    """Scores in the hundreds: a row's weight sits on one token or few, its maximum moves many times."""
    pr = paged.Problem(5, "bf16", 64, 32, 4, 2, new, kv, scale=8.0)
    kv_len, table = pr.args()
    o, lse = pr.cache().attention(pr.q.cuda(), kv_len, table, q_start=pr.q_start.cuda(), scale=1.0, want_lse=True)
    paged.check(pr, o, lse, paged.attend(pr, scale=1.0))


@pytest.mark.parametrize("dtype,new,kv", [("bf16", [10, 1], [4, 0]), ("fp32", [70, 3], [20, 3]), ("bf16", [200], [150])])
def test_rows_that_see_nothing(dtype, new, kv):
    """More new tokens than the sequence is long, lengths of zero: those rows are 0 with lse -inf."""
    pr = paged.Problem(1, dtype, 64, 16, 4, 2, new, kv, garbage=float("nan"))
    kv_len, table = pr.args()
    o, lse = pr.cache().attention(pr.q.cuda(), kv_len, table, q_start=pr.q_start.cuda(), want_lse=True)
    want = paged.attend(pr)
    assert torch.isinf(want[1]).any()
    paged.check(pr, o, lse, want)


@pytest.mark.parametrize("dtype,P,new", [("bf16", 16, [1, 1]), ("bf16", 64, [50, 120]), ("fp32", 32, [2, 40])])
def test_unmapped_pages_are_masked(dtype, P, new):
    pr = paged.Problem(2, dtype, 128, P, 8, 2, new, [300, 310], garbage=float("nan"))
    pr.table[0, 1] = -1
    pr.table[1, 0] = pr.n_pages
    pr.table[1, 2] = -(1 << 31)
    pr.table[1, 300 // P] = (1 << 31) - 1
    kv_len, table = pr.args()
    o, lse = pr.cache().attention(pr.q.cuda(), kv_len, table, q_start=pr.q_start.cuda(), want_lse=True)
    paged.check(pr, o, lse, paged.attend(pr))


@pytest.mark.parametrize("dtype,d,new", [("bf16", 64, 3), ("bf16", 128, 70), ("bf16", 256, 140), ("fp32", 128, 40), ("bf16", 128, 300)])
def test_infinities_and_nan_reach_only_rows_that_see_them(dtype, d, new):
    pr = paged.Problem(3, dtype, d, 32, 4, 2, [new], [new + 50])
    n = new + 50
    v, k = pr.rows_v[0], pr.rows_k[0]
    v[n - 1, 0, 5] = float("nan")
    v[n - 2, 0, 7] = float("inf")
    v[n - 3, 1, d - 1] = float("-inf")
    v[n - 2, 1, d - 1] = float("inf")                                  # both signs: the last two rows see NaN
    k[n - 1, 1, 3] = float("nan")                                      # the last row's score of itself
    kv_len, table = pr.args()
    o, lse = pr.cache().attention(pr.q.cuda(), kv_len, table, q_start=pr.q_start.cuda(), want_lse=True)
    out, l64, tol, ltol = paged.attend(pr)
    o, lse = o.cpu().to(torch.float64), lse.cpu().to(torch.float64)
    assert torch.equal(torch.isnan(o), torch.isnan(out)) and torch.equal(torch.isinf(o), torch.isinf(out))
    assert torch.equal(torch.isnan(lse), torch.isnan(l64))
    fin = torch.isfinite(out)
    assert torch.all((o - out).abs()[fin] <= tol[fin])


def test_strided_rows_and_another_stream():
    """Queries as a part of a wider projection, the block table a part of a wider one, work on a stream of its own."""
    pr = paged.Problem(4, "bf16", 128, 64, 8, 2, [1, 40], [77, 200])
    kv_len, table = pr.args()
    wide = torch.zeros(pr.T, 12, 128 + 16, dtype=torch.bfloat16, device="cuda")
    wide[:, 2:10, 8:136] = pr.q.cuda()
    roomy = torch.full((2, table.shape[1] + 5), -7, dtype=torch.int32, device="cuda")
    roomy[:, :table.shape[1]] = table
    c, qs = pr.cache(), pr.q_start.cuda()
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        o, lse = c.attention(wide[:, 2:10, 8:136], kv_len, roomy[:, :table.shape[1]], q_start=qs, want_lse=True)
    torch.cuda.current_stream().wait_stream(st)
    paged.check(pr, o, lse, paged.attend(pr))


@pytest.mark.parametrize("new", [[1], [40]])
def test_offsets_past_32_bits(new):
    """Pages whose bytes lie beyond 4 GiB of each array (only the pages in use are filled)."""
    import paper_2601_17702_amd as s3
    pr = paged.Problem(6, "bf16", 128, 64, 8, 2, new, [150], spare=0)
    k, v = pr.pack()
    per = k[0].numel() * 2
    n_pages = (5 << 30) // per
    c = s3.KVCache(n_pages, 64, 2, 128, signatures=True)
    far = torch.arange(n_pages - pr.n_pages, n_pages, device="cuda")
    c.k[far], c.v[far] = k.cuda(), v.cuda()
    kv_len, table = pr.args()
    table = torch.where(table >= 0, table + (n_pages - pr.n_pages), table)
    qs = pr.q_start.cuda()
    o, lse = c.attention(pr.q.cuda(), kv_len, table, q_start=qs, want_lse=True)
    want = paged.attend(pr)
    paged.check(pr, o, lse, want)
    sel = torch.full((pr.tiles(16), 2, 5), -1, dtype=torch.int32, device="cuda")
    sel[:, :, :3] = torch.arange(3, device="cuda")
    o, lse = c.block_attention(pr.q.cuda(), kv_len, table, sel, q_start=qs, q_block=16, want_lse=True)
    paged.check(pr, o, lse, want)
    n = new[0]
    x = torch.randn(n, 2, 128, device="cuda").to(torch.bfloat16)
    c.append(x, x, kv_len, table, q_start=qs)
    page, slot = int(table[0, 149 // 64]), 149 % 64
    assert torch.equal(c.k[page, :, :, slot].reshape(2, 128), x[-1]) and torch.equal(c.v[page, :, slot // 8, :, slot % 8], x[-1])
    del c


# ------------------------------------------------------------------------------------------------ append
def rotated(x, table, rot, pos, inter):
    """x [n, heads, d] CPU in its type -> (rotated in its type with every product and sum rounded to fp32, the same in 64 bits)."""
    if table is None:
        return x.clone(), x.to(torch.float64)
    res = []
    for dt in (torch.float32, torch.float64):
        y = x.to(dt, copy=True)
        c, s = table[pos][:, None, :rot // 2].to(dt), table[pos][:, None, rot // 2:].to(dt)
        i = torch.arange(rot // 2)
        ia, ib = (2 * i, 2 * i + 1) if inter else (i, i + rot // 2)
        a, b = y[..., ia].clone(), y[..., ib].clone()
        y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
        res.append(y)
    return res[0].to(x.dtype), res[1]


@pytest.mark.parametrize("dtype,d,P,hq,hkv,new,kv,rot,inter,explicit", [
    ("bf16", 128, 64, 32, 8, [1, 1, 1], [1, 64, 65], 128, False, False),
    ("bf16", 128, 64, 8, 2, [130, 0, 7], [300, 9, 7], 128, False, True),
    ("bf16", 64, 16, 7, 1, [33, 1], [40, 17], 32, True, False),
    ("bf16", 256, 32, 4, 4, [50], [50], 256, True, False),
    ("bf16", 256, 128, 2, 2, [200], [333], 64, False, False),
    ("fp32", 64, 256, 4, 2, [300, 2], [301, 256], 64, False, False),
    ("fp32", 128, 16, 4, 2, [19, 31, 1], [50, 32, 16], 96, True, True),
    ("fp32", 256, 64, 2, 1, [70], [190], 0, False, False),
    ("bf16", 128, 32, 2, 2, [12, 5], [7, 0], 128, False, False),      # more new tokens than the sequence is long
])
def test_append(dtype, d, P, hq, hkv, new, kv, rot, inter, explicit):
    import paper_2601_17702_amd as s3
    pr = paged.Problem(7 + d + P, dtype, d, P, hq, hkv, new, kv, garbage=3.0)
    kc, vc = pr.pack()
    sig = torch.full((pr.n_pages, hkv, d), 9.0, dtype=torch.bfloat16)
    c = s3.KVCache(pr.n_pages, P, hkv, d, pr.dtype, k=kc.cuda(), v=vc.cuda(), sig=sig.cuda())
    w = hq + 2 * hkv
    qkv = torch.randn(pr.T, w, d, generator=pr.g).to(pr.dtype)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    pos = torch.cat([torch.arange(m - n, m) for n, m in zip(new, kv)])
    seq = torch.cat([torch.full((n,), s) for s, n in enumerate(new)])
    at = pos
    if explicit:
        at = torch.randint(0, 900, (pr.T,), generator=pr.g)
    table = s3.rope_table(900, rot, 10000.0) if rot else None
    ang = torch.arange(900, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / max(rot, 1))
    if rot:
        # cos and sin of an angle below 900 in 64 bits, off by a few ulp of the angle, rounded once
        assert torch.all((table.cpu().to(torch.float64) - torch.cat([ang.cos(), ang.sin()], 1)).abs() <= 2.0 ** -25 + 1e-12)
    t_cpu = table.cpu() if rot else None
    dev = qkv.cuda()
    qr = c.append(dev[:, hq:hq + hkv], dev[:, hq + hkv:], pr.kv_len.cuda(), pr.table.cuda(), q_start=pr.q_start.cuda(), rope=table,
                  interleaved=inter, positions=at.to(torch.int32).cuda() if explicit else None, q=dev[:, :hq])
    k32, k64 = rotated(k, t_cpu, rot, at.clamp(0, 899), inter)
    q32, q64 = rotated(q, t_cpu, rot, at.clamp(0, 899), inter)
    assert torch.equal(qr.cpu(), q32)
    # against 64 bits: two products and a sum in fp32, 3 roundings of at most 2^-24 (|a| + |b|) each, then one to the type
    room = (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * q64.abs() * 1.01 + 3 * 2.0 ** -24 * 2 * float(q64.abs().max())
    assert torch.all((qr.cpu().to(torch.float64) - q64).abs() <= room)
    written = {}
    for i in range(pr.T):
        s, p = int(seq[i]), int(pos[i])
        if p < 0:
            continue
        page, slot = int(pr.table[s, p // P]), p % P
        kc[page, :, :, slot] = k32[i].view(hkv, d // pr.E, pr.E)
        vc[page, :, slot // pr.E, :, slot % pr.E] = v[i]
        written[page] = slot + 1
    for page, n in written.items():
        for h in range(hkv):
            rows = kc[page, h].transpose(0, 1).reshape(P, d)[:n]
            sig[page, h] = torch.from_numpy(paged.signature(rows)).to(torch.bfloat16)
    assert torch.equal(c.k.cpu(), kc) and torch.equal(c.v.cpu(), vc) and torch.equal(c.sig.cpu(), sig)


def test_append_token_by_token_equals_one_chunk():
    import paper_2601_17702_amd as s3
    pr = paged.Problem(8, "bf16", 128, 32, 4, 2, [100], [100])
    x = torch.randn(100, 4, 128, generator=pr.g).to(torch.bfloat16).cuda()
    k, v = x[:, :2], x[:, 2:]
    rope = s3.rope_table(100, 128)
    caches = [s3.KVCache(pr.n_pages, 32, 2, 128, signatures=True) for _ in range(3)]
    for c in caches:
        c.k.zero_(), c.v.zero_(), c.sig.zero_()
    table = pr.table.cuda()
    cuts = [[100], [1] * 100, [33, 1, 31, 35]]
    for c, cut in zip(caches, cuts):
        done = 0
        for n in cut:
            qs = torch.tensor([0, n], dtype=torch.int32, device="cuda")
            done += n
            c.append(k[done - n:done], v[done - n:done], torch.tensor([done], dtype=torch.int32, device="cuda"), table, q_start=qs, rope=rope)
    for c in caches[1:]:
        assert torch.equal(c.k, caches[0].k) and torch.equal(c.v, caches[0].v) and torch.equal(c.sig, caches[0].sig)


def test_append_leaves_unmapped_pages_alone():
    import paper_2601_17702_amd as s3
    pr = paged.Problem(9, "bf16", 64, 16, 2, 1, [40], [40])
    pr.table[0, 1] = pr.n_pages
    c = s3.KVCache(pr.n_pages, 16, 1, 64, signatures=True)
    c.k.fill_(5.0), c.v.fill_(5.0), c.sig.fill_(5.0)
    x = torch.randn(40, 2, 64, generator=pr.g).to(torch.bfloat16).cuda()
    c.append(x[:, :1], x[:, 1:], pr.kv_len.cuda(), pr.table.cuda(), q_start=pr.q_start.cuda())
    used = {int(pr.table[0, 0]), int(pr.table[0, 2])}
    for page in range(pr.n_pages):
        if page in used:
            assert not torch.all(c.sig[page] == 5.0)
        else:
            assert torch.all(c.k[page] == 5.0) and torch.all(c.v[page] == 5.0) and torch.all(c.sig[page] == 5.0)


@pytest.mark.parametrize("value", [0.0, float("nan"), float("inf"), 2.0 ** -41, 2.0 ** 50, 2.0 ** -40, 1.99 * 2.0 ** 49])
def test_signatures_at_the_ends_of_their_range(value):
    import paper_2601_17702_amd as s3
    c = s3.KVCache(1, 16, 1, 64, torch.float32, signatures=True)
    k = torch.zeros(1, 1, 64, device="cuda")
    k[0, 0, 3] = value
    one = torch.ones(1, dtype=torch.int32, device="cuda")
    c.append(k, k, one, torch.zeros(1, 1, dtype=torch.int32, device="cuda"))
    want = paged.grid8(k[0].cpu().numpy())
    assert np.array_equal(c.sig[0].cpu().to(torch.float64).numpy(), want)
    assert (np.abs(want).max() > 0) == (2.0 ** -40 <= value < 2.0 ** 50)


# ------------------------------------------------------------------------------------------------ selection, listed blocks
def draw_sig(pr):
    x = torch.randn(pr.n_pages, pr.hkv, pr.d, generator=pr.g) * 0.3
    return torch.from_numpy(paged.grid8(x.numpy())).to(torch.bfloat16)


@pytest.mark.parametrize("dtype,d,P,hq,hkv,new,kv,qb,top,lead,tail", [
    ("bf16", 128, 64, 32, 8, [1, 1, 1], [1, 640, 6400], 1, 8, 1, 1),
    ("bf16", 128, 16, 28, 4, [37, 0, 5], [500, 3, 5], 16, 12, 1, 2),
    ("bf16", 64, 32, 4, 4, [70], [900], 32, 9, 2, 3),
    ("fp32", 256, 16, 4, 2, [20], [300], 7, 6, 0, 0),                 # nothing is always taken
    ("fp32", 64, 16, 16, 1, [9, 1], [9, 160], 4, 5, 1, 1),
    ("bf16", 256, 32, 32, 1, [3], [2000], 2, 4, 1, 1),
    ("bf16", 128, 16, 8, 2, [1, 1], [20000, 15000], 1, 64, 1, 1),      # more candidates than one pass of threads
    ("bf16", 128, 16, 4, 2, [10], [3], 4, 4, 1, 1),                   # tiles before the sequence
    ("bf16", 64, 16, 8, 2, [300], [400], 256, 40, 1, 1),               # many rows a tile
    ("bf16", 128, 16, 28, 4, [100, 60], [900, 60], 1, 6, 1, 1),        # several tiles a workgroup, seven rows each
    ("bf16", 128, 32, 32, 8, [200, 3, 0, 77], [900, 300, 40, 80], 8, 6, 1, 1),
    ("fp32", 256, 16, 8, 4, [90], [2000], 4, 20, 1, 1),
    ("bf16", 64, 16, 2, 2, [1], [50000], 1, 96, 1, 1),                 # few tiles, a long context: through scratch
    ("fp32", 64, 16, 3, 1, [40], [40000], 16, 300, 1, 1),
    ("bf16", 64, 16, 2, 1, [600], [700], 2, 5, 1, 1),
])
def test_select(dtype, d, P, hq, hkv, new, kv, qb, top, lead, tail):
    pr = paged.Problem(11 + d + qb, dtype, d, P, hq, hkv, new, kv)
    sig = draw_sig(pr)
    kv_len, table = pr.args()
    c = pr.cache(sig=sig)
    sel = c.select(pr.q.cuda(), kv_len, table, top, q_start=pr.q_start.cuda(), q_block=qb, lead=lead, tail=tail)
    assert np.array_equal(sel.cpu().numpy(), paged.select(pr, sig, top, qb, lead, tail))
    sel = c.select(pr.q.cuda(), kv_len, table, top, q_start=pr.q_start.cuda(), q_block=qb, lead=lead, tail=tail, max_new=max(new), max_kv=max(kv))
    assert np.array_equal(sel.cpu().numpy(), paged.select(pr, sig, top, qb, lead, tail))


def test_select_ties_and_unmapped_blocks():
    """Equal signatures everywhere: the lowest blocks win; an unmapped block is no candidate, not even where it would always be taken;
    rows of zeros and of NaN score zero."""
    pr = paged.Problem(12, "bf16", 64, 16, 4, 1, [6], [800])
    sig = torch.ones(pr.n_pages, 1, 64, dtype=torch.bfloat16)
    pr.table[0, 0] = -1
    pr.table[0, 4] = pr.n_pages
    pr.q[2:4] = 0.0
    pr.q[4] = float("nan")
    kv_len, table = pr.args()
    sel = pr.cache(sig=sig).select(pr.q.cuda(), kv_len, table, 7, q_start=pr.q_start.cuda(), q_block=1)
    assert np.array_equal(sel.cpu().numpy(), paged.select(pr, sig, 7, 1, 1, 1))
    assert sel[2, 0].tolist() == [1, 2, 3, 5, 6, 7, 49]


@pytest.mark.parametrize("n_blocks,new,qb,top,kinds", [
    (300, 1, 1, 40, 0), (300, 1, 1, 40, 3),                           # through scratch; three different signatures only: ties everywhere
    (2000, 40, 8, 200, 0), (2000, 40, 8, 200, 5),
    (5000, 1, 1, 64, 0), (5000, 1, 1, 64, 2),                         # the pick of many candidates
    (20000, 3, 1, 700, 0), (20000, 3, 1, 700, 40),                    # more than it keeps in registers
    (20000, 1, 1, 4096, 0),
    (700, 130, 1, 30, 0), (700, 130, 1, 30, 2),                       # several tiles a workgroup
])
def test_select_of_many_candidates(n_blocks, new, qb, top, kinds):
    import paper_2601_17702_amd as s3
    kv = n_blocks * 16 - 3
    pr = paged.Problem(n_blocks + new, "bf16", 64, 16, 4, 2, [new], [kv])
    sig = draw_sig(pr)
    if kinds:
        sig = sig[torch.randint(0, kinds, (pr.n_pages,), generator=pr.g)]
    pr.table[0, 7] = -1
    c = s3.KVCache(pr.n_pages, 16, 2, 64, sig=sig.cuda())
    kv_len, table = pr.args()
    sel = c.select(pr.q.cuda(), kv_len, table, top, q_start=pr.q_start.cuda(), q_block=qb, lead=2, tail=2, max_new=new, max_kv=kv)
    assert np.array_equal(sel.cpu().numpy(), paged.select(pr, sig, top, qb, 2, 2))


@pytest.mark.parametrize("new,G,n_seq,listed", [(1, 4, 1200, False), (1, 4, 1200, True), (64, 4, 300, False), (64, 4, 300, True)])
def test_many_sequences_over_the_same_pages(new, G, n_seq, listed):
    """A shared prefix, and more work a workgroup than it looks up pages for at a time: every sequence has the same answer."""
    kv, P = 20000, 64
    pr = paged.Problem(n_seq + new, "bf16", 64, P, G, 1, [new], [kv])
    n_blocks = -(-kv // P)
    sel = np.arange(n_blocks, dtype=np.int32).reshape(1, 1, n_blocks) if listed else None
    want = paged.attend(pr, sel=sel, qb=new if listed else None)
    q = pr.q.cuda().repeat(n_seq, 1, 1)
    kv_len = torch.full((n_seq,), kv, dtype=torch.int32, device="cuda")
    table = pr.table.cuda().repeat(n_seq, 1)
    qs = torch.arange(n_seq + 1, dtype=torch.int32, device="cuda") * new
    c = pr.cache()
    if listed:
        tiles = (n_seq * new + n_seq * (new - 1)) // new               # the list's documented length; one tile a sequence is used
        dev = torch.from_numpy(sel).cuda().repeat(tiles, 1, 1)
        o, lse = c.block_attention(q, kv_len, table, dev, q_start=qs, q_block=new, want_lse=True)
    else:
        o, lse = c.attention(q, kv_len, table, q_start=qs, max_new=new, max_kv=kv, want_lse=True)
    o, lse = o.view(n_seq, new, G, 64), lse.view(n_seq, new, G)
    paged.check(pr, o[0], lse[0], want)
    tol = want[2].cuda().to(torch.float32) * 2
    assert torch.all((o.float() - o[:1].float()).abs() <= tol)         # where a workgroup's run ends differs, so do roundings
    for s in (1, n_seq // 2, n_seq - 1):
        paged.check(pr, o[s], lse[s], want)


@pytest.mark.parametrize("dtype,d,P,hq,hkv,new,kv,qb,top", [
    ("bf16", 128, 64, 32, 8, [1, 1], [640, 70], 1, 4),
    ("bf16", 128, 16, 28, 4, [37, 0, 5], [300, 3, 5], 16, 9),
    ("bf16", 64, 32, 8, 2, [70], [300], 64, 7),
    ("bf16", 128, 64, 8, 2, [130], [600], 128, 6),
    ("bf16", 256, 128, 4, 2, [20], [700], 8, 4),
    ("fp32", 128, 16, 4, 2, [40, 1], [200, 90], 16, 6),
    ("fp32", 256, 32, 2, 1, [70], [200], 64, 5),
    ("bf16", 128, 256, 8, 2, [5], [1500], 5, 3),
    ("bf16", 64, 16, 8, 2, [1, 1, 1], [90, 200, 7], 64, 5),            # tiles far larger than what a sequence brings
    ("fp32", 128, 16, 8, 2, [20, 3], [90, 200], 32, 5),                # 80 rows a tile
    ("bf16", 128, 16, 4, 1, [300], [400], 200, 9),                     # tiles of 800 rows
])
def test_block_attention(dtype, d, P, hq, hkv, new, kv, qb, top):
    pr = paged.Problem(13 + d + qb, dtype, d, P, hq, hkv, new, kv, garbage=float("nan"))
    rng = np.random.default_rng(d + P)
    n_blocks = max(-(-n // P) for n in kv)
    sel = rng.integers(-1, n_blocks + 1, (pr.tiles(qb), hkv, top)).astype(np.int32)      # holes, repeats, blocks past the sequence, any order
    sel[0, 0] = -1                                                     # a tile that reads nothing
    sel[-1, -1, 0] = 1 << 30
    kv_len, table = pr.args()
    c = pr.cache()
    dev = torch.from_numpy(sel).cuda()
    want = paged.attend(pr, sel=sel, qb=qb)
    o, lse = c.block_attention(pr.q.cuda(), kv_len, table, dev, q_start=pr.q_start.cuda(), q_block=qb, want_lse=True)
    paged.check(pr, o, lse, want)
    o2, lse2 = c.block_attention(pr.q.cuda(), kv_len, table, dev, q_start=pr.q_start.cuda(), q_block=qb, want_lse=True, max_new=max(new), max_kv=max(kv))
    paged.check(pr, o2, lse2, want)


def test_all_blocks_listed_is_attention():
    pr = paged.Problem(14, "bf16", 128, 32, 8, 2, [33, 1], [200, 150])
    sel = torch.arange(8, dtype=torch.int32, device="cuda").repeat(pr.tiles(16), 2, 1).contiguous()
    kv_len, table = pr.args()
    c, qs, q = pr.cache(), pr.q_start.cuda(), pr.q.cuda()
    o, lse = c.block_attention(q, kv_len, table, sel, q_start=qs, q_block=16, want_lse=True)
    paged.check(pr, o, lse, paged.attend(pr))


# ------------------------------------------------------------------------------------------------ graphs
@pytest.mark.parametrize("new", [[1, 1, 1], [40, 1, 100]])
def test_captured_in_a_graph(new):
    """Append, selection and both attentions recorded once; every replay, with other inputs in the same places and eager work
    between, equals the eager calls."""
    import paper_2601_17702_amd as s3
    pr = paged.Problem(15, "bf16", 128, 64, 8, 2, new, [200, 300, 1000])
    c = pr.cache(signatures=True)
    c.sig.zero_()
    kv_len, table = pr.args()
    qs = pr.q_start.cuda()
    rope = s3.rope_table(1000, 128)
    qkv = torch.randn(pr.T, 12, 128, device="cuda").to(torch.bfloat16)

    def step():
        q = c.append(qkv[:, 8:10], qkv[:, 10:], kv_len, table, q_start=qs, rope=rope, q=qkv[:, :8])
        o, _ = c.attention(q, kv_len, table, q_start=qs, max_new=max(new), max_kv=1000)
        sel = c.select(q, kv_len, table, 6, q_start=qs, q_block=16, max_kv=1000)
        ob, _ = c.block_attention(q, kv_len, table, sel, q_start=qs, q_block=16, max_new=max(new))
        return q, o, sel, ob

    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        step()
    torch.cuda.current_stream().wait_stream(st)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for _ in range(4):
        qkv.copy_(torch.randn(pr.T, 12, 128, device="cuda"))
        graph.replay()
        got = [t.clone() for t in out]
        torch.cuda.synchronize()
        for a, b in zip(got, step()):
            assert torch.equal(a, b)


# ------------------------------------------------------------------------------------------------ all of it together
def test_example_of_a_context_answered_from_a_part_of_it():
    """examples/paged_answer.py: lists hold blocks of the cache in ascending order, the named ones those of the spans; a part of
    the blocks cannot hold more than all of the weight, and holds more than its share of the cache where keys and question share a topic."""
    from examples import paged_answer
    r = paged_answer.run(context=3000, chunk=700, answer=3, n_q=8, n_kv=2, n_feat=1024, k=16, top_blocks=12, n_spans=6)
    assert torch.isfinite(r["hidden"].float()).all() and torch.isfinite(r["full"].float()).all()
    for sel in (r["named"], r["chosen"]):
        for row in sel.cpu().view(-1, 12).tolist():
            there = [b for b in row if b >= 0]
            assert there == sorted(set(there)) and there[0] == 0 and there[-1] == r["blocks"] - 1 and row[len(there):] == [-1] * (12 - len(there))
    named = set(r["named"].cpu().view(-1).tolist())
    spans = [int(s) for s in r["starts"].cpu() if s >= 0]
    assert spans and sum(s // 64 in named for s in spans) >= min(len(spans), 4)
    share = 12 / r["blocks"]
    assert share < r["chosen_share"] <= 1.0 + 1e-5 and 0.0 < r["span_share"] <= 1.0 + 1e-5


# ------------------------------------------------------------------------------------------------ refusals
def test_refusals():
    import paper_2601_17702_amd as s3
    pr = paged.Problem(16, "bf16", 128, 64, 8, 2, [1], [10])
    c = pr.cache()
    kv_len, table = pr.args()
    q = pr.q.cuda()
    for call in (
        lambda: s3.KVCache(4, 24, 2, 128).attention(q, kv_len, table),                       # page size
        lambda: s3.KVCache(4, 64, 2, 96).attention(q[:, :, :96], kv_len, table),              # d_head
        lambda: c.attention(q[:, :7], kv_len, table),                                         # heads
        lambda: c.attention(q, kv_len, table, scale=0.0),
        lambda: c.attention(q, kv_len, table, scale=float("nan")),
        lambda: c.attention(q, kv_len, table, window=-1),
        lambda: c.select(q, kv_len, table, 4),                                                # no signatures
        lambda: pr.cache(signatures=True).select(q, kv_len, table, 1),                        # no room for what is always taken
        lambda: pr.cache(signatures=True).select(q, kv_len, table, 5000),
        lambda: c.append(q[:, :2], q[:, 2:4], kv_len, table, rope=torch.zeros(4, 24, device="cuda")),
        lambda: s3.rope_table(4, 24),
        lambda: c.attention(torch.zeros(1, 8, 130, dtype=torch.bfloat16, device="cuda")[:, :, 1:129], kv_len, table),     # alignment
    ):
        with pytest.raises(s3.S3Error) as e:
            call()
        assert e.value.code == -1
    with pytest.raises(TypeError):
        s3.KVCache(4, 64, 2, 128, torch.float16)
    with pytest.raises(AssertionError):
        c.attention(q.float(), kv_len, table)


def test_no_tokens_is_a_no_op():
    pr = paged.Problem(17, "bf16", 128, 64, 8, 2, [0, 0], [10, 0])
    kv_len, table = pr.args()
    c = pr.cache(signatures=True)
    qs = pr.q_start.cuda()
    o, lse = c.attention(pr.q.cuda(), kv_len, table, q_start=qs, want_lse=True)
    assert o.shape == (0, 8, 128)
    x = torch.zeros(0, 2, 128, dtype=torch.bfloat16, device="cuda")
    c.append(x, x, kv_len, table, q_start=qs)
    sel = c.select(pr.q.cuda(), kv_len, table, 4, q_start=qs, q_block=16)
    assert torch.all(sel == -1)
