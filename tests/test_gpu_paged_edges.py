"""GPU checks of the paged cache at the ends of what its calls take, against the plain 64-bit forms (tests/paged.py)."""
import pytest
import torch

from tests import paged

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 30, 2 ** 30 - 1])
@pytest.mark.parametrize("dtype,new,kv", [("bf16", [10, 1], [4, 9]), ("bf16", [200], [150]), ("fp32", [150, 5], [90, 2])])
def test_windows_of_any_length(dtype, new, kv, window):
    """A window longer than every sequence hides nothing, also where some new tokens lie before the sequence's start: few rows and many."""
    pr = paged.Problem(19, dtype, 64, 16, 4, 2, new, kv, garbage=float("nan"))
    kv_len, table = pr.args()
    c, qs, q = pr.cache(), pr.q_start.cuda(), pr.q.cuda()
    o, lse = c.attention(q, kv_len, table, q_start=qs, window=window, want_lse=True)
    paged.check(pr, o, lse, paged.attend(pr))
    plain, _ = c.attention(q, kv_len, table, q_start=qs)
    if window >= 2 ** 30:
        assert torch.equal(o, plain)


@pytest.mark.parametrize("dtype,d,hq,hkv", [("bf16", 64, 3, 3), ("bf16", 128, 7, 1), ("fp32", 128, 2, 2), ("fp32", 256, 3, 1), ("bf16", 256, 5, 1)])
def test_an_odd_number_of_rows_in_parts(dtype, d, hq, hkv):
    """1, 3, 5 and 7 rows of single tokens whose keys more than one workgroup has."""
    pr = paged.Problem(20 + d, dtype, d, 32, hq, hkv, [1, 1, 1], [5000, 33, 3001], garbage=float("nan"))
    kv_len, table = pr.args()
    o, lse = pr.cache().attention(pr.q.cuda(), kv_len, table, want_lse=True)
    paged.check(pr, o, lse, paged.attend(pr))


@pytest.mark.parametrize("listed", [False, True])
@pytest.mark.parametrize("dtype,d,hq,new,kv,blocks", [
    ("bf16", 64, 4, [1, 1], [96, 4000], [3, 60]),         # one token that sees nothing else; the first of a workgroup's tokens, and whole workgroups'
    ("bf16", 128, 8, [150], [150], [2]),                  # a prompt: its first rows see nothing else
    ("bf16", 256, 4, [40, 5], [70, 64], [1, 2]),
    ("fp32", 64, 4, [70, 2], [2000, 64], [40, 2]),        # row tiles in parts
    ("fp32", 128, 4, [3, 100], [31, 200], [1, 4]),
    ("fp32", 256, 2, [90], [120], [2]),
])
def test_rows_that_see_scores_of_minus_infinity_only(dtype, d, hq, new, kv, blocks, listed):
    """The softmax of such a row is 0 / 0: NaN with lse -inf, not the zeros of a row that sees nothing.  Rows that see a finite score
    too are as if the others were not there.  An infinite key against queries of the other sign, in the first blocks of every sequence."""
    P = 32
    pr = paged.Problem(21 + d, dtype, d, P, hq, 2, new, kv, garbage=float("nan"))
    pr.q[..., 0] = -pr.q[..., 0].abs() - 1
    for rows, n in zip(pr.rows_k, blocks):
        rows[:n * P, :, 0] = float("inf")
    kv_len, table = pr.args()
    c, q, qs = pr.cache(), pr.q.cuda(), pr.q_start.cuda()
    for s, n in enumerate(blocks):
        pr.table[s, :n] = -1                                            # for the reference they are not there
    want, l64, tol, ltol = paged.attend(pr)
    if listed:
        sel = torch.arange(table.shape[1], dtype=torch.int32, device="cuda").repeat(pr.tiles(16), 2, 1).contiguous()
        o, lse = c.block_attention(q, kv_len, table, sel, q_start=qs, q_block=16, want_lse=True)
    else:
        o, lse = c.attention(q, kv_len, table, q_start=qs, max_new=max(new), max_kv=max(kv), want_lse=True)
    o, lse = o.cpu().to(torch.float64), lse.cpu().to(torch.float64)
    none = torch.isinf(l64)
    assert none.any()
    assert torch.isnan(o[none]).all() and torch.all(lse[none] == -float("inf"))
    assert torch.all((o - want).abs()[~none] <= tol[~none]) and torch.all((lse - l64).abs()[~none] <= ltol[~none])


def test_scratch_of_the_callers():
    """A workspace in host memory is refused by every call that takes one; one on the device serves all of them."""
    pr = paged.Problem(22, "bf16", 64, 16, 4, 2, [1, 40], [500, 90])
    kv_len, table = pr.args()
    c, q, qs = pr.cache(signatures=True), pr.q.cuda(), pr.q_start.cuda()
    c.sig.zero_()
    sel = c.select(q, kv_len, table, 6, q_start=qs, q_block=16)
    calls = (lambda ws: c.attention(q, kv_len, table, q_start=qs, ws=ws)[0], lambda ws: c.select(q, kv_len, table, 6, q_start=qs, q_block=16, ws=ws),
             lambda ws: c.block_attention(q, kv_len, table, sel, q_start=qs, q_block=16, ws=ws)[0])
    for call in calls:
        with pytest.raises(AssertionError):
            call(torch.empty(1 << 24, dtype=torch.uint8))
        assert torch.equal(call(torch.empty(1 << 28, dtype=torch.uint8, device="cuda")), call(None))


@pytest.mark.parametrize("new", [[1, 2], [90, 1]])
def test_sequences_without_pages(new):
    """A table of no columns: nothing is stored, every row sees nothing, no block is listed."""
    pr = paged.Problem(23, "bf16", 64, 16, 4, 2, new, [100, 3])
    c, q, qs, kv_len = pr.cache(signatures=True), pr.q.cuda(), pr.q_start.cuda(), pr.kv_len.cuda()
    before = [t.clone() for t in (c.k, c.v)]
    table = torch.empty(2, 0, dtype=torch.int32, device="cuda")
    c.append(q[:, :2], q[:, 2:], kv_len, table, q_start=qs)
    assert torch.equal(c.k, before[0]) and torch.equal(c.v, before[1])
    sel = c.select(q, kv_len, table, 5, q_start=qs, q_block=16)
    assert torch.all(sel == -1)
    for o, lse in (c.attention(q, kv_len, table, q_start=qs, want_lse=True), c.block_attention(q, kv_len, table, torch.zeros_like(sel), q_start=qs, q_block=16, want_lse=True)):
        assert torch.all(o == 0) and torch.all(lse == -float("inf"))


# ------------------------------------------------------------------------------------------------ what the kernels hold inside the arrays
def guarded(*shape, dtype, value):
    """(whole, inner): an array with 64 rows of `value` before and behind it, all of it `value`."""
    whole = torch.full((shape[0] + 128, *shape[1:]), value, dtype=dtype, device="cuda")
    return whole, whole[64:64 + shape[0]]


@pytest.mark.parametrize("dtype,new,kv", [("bf16", [1, 3], [70, 40]), ("bf16", [90, 2], [300, 31]), ("fp32", [40, 1], [64, 9])])
def test_rows_of_no_sequence_are_not_written(dtype, new, kv):
    """q_start begins at 3 and ends 5 rows before n_tokens."""
    import paper_2601_17702_amd as s3
    pr = paged.Problem(24, dtype, 64, 16, 4, 2, new, kv, garbage=2.0)
    c, table, kv_len = pr.cache(signatures=True), pr.table.cuda(), pr.kv_len.cuda()
    kc, vc = c.k.clone(), c.v.clone()
    T = pr.T + 8
    mine = torch.zeros(T, dtype=torch.bool)
    mine[3:3 + pr.T] = True
    q = torch.full((T, 4, 64), 7.0, dtype=pr.dtype)
    q[mine] = pr.q
    rows = [torch.full((T, 2, 64), 7.0, dtype=pr.dtype) for _ in range(2)]
    for x, r in zip(rows, (pr.rows_k, pr.rows_v)):
        x[mine] = torch.cat([r[s][m - n:] for s, (n, m) in enumerate(zip(new, kv))])          # the rows that are there already
    qs = (pr.q_start + 3).cuda()
    whole, out = guarded(T, 4, 64, dtype=pr.dtype, value=9.0)
    got = c.append(rows[0].cuda(), rows[1].cuda(), kv_len, table, q_start=qs, q=q.cuda(), q_out=out)
    assert torch.equal(out[mine.cuda()].cpu(), pr.q) and torch.all(whole[:67] == 9) and torch.all(whole[67 + pr.T:] == 9) and got is out
    assert torch.equal(c.k, kc) and torch.equal(c.v, vc)
    want = paged.attend(pr)
    whole, out = guarded(T, 4, 64, dtype=pr.dtype, value=9.0)
    _, lse = c.attention(q.cuda(), kv_len, table, q_start=qs, out=out, want_lse=True)
    paged.check(pr, out[mine.cuda()], lse[mine.cuda()], want)
    assert torch.all(whole[:67] == 9) and torch.all(whole[67 + pr.T:] == 9)
    tiles = s3.lib().s3_block_tiles(c._batch(T, kv_len, table, qs, None, None), 16)
    sel = torch.arange(table.shape[1], dtype=torch.int32, device="cuda").repeat(tiles, 2, 1).contiguous()
    whole, out = guarded(T, 4, 64, dtype=pr.dtype, value=9.0)
    _, lse = c.block_attention(q.cuda(), kv_len, table, sel, q_start=qs, q_block=16, out=out, want_lse=True)
    paged.check(pr, out[mine.cuda()], lse[mine.cuda()], want)
    assert torch.all(whole[:67] == 9) and torch.all(whole[67 + pr.T:] == 9)
    sig = torch.from_numpy(paged.grid8(torch.randn(pr.n_pages, 2, 64, generator=pr.g).numpy())).to(torch.bfloat16)
    c.sig.copy_(sig)
    got = c.select(q.cuda(), kv_len, table, 5, q_start=qs, q_block=16).cpu().numpy()
    ref = paged.select(pr, sig, 5, 16, 1, 1)
    n = sum(-(-x // 16) for x in new)
    assert (got[:n] == ref[:n]).all() and (got[n:] == -1).all()


@pytest.mark.parametrize("starts", [[0, 5, 60, 60], [0, 30, 10, 40], [0, 40, 90, 100], [2, -3, 8, 40]])
def test_starts_that_are_no_starts_write_nothing_else(starts):
    """Starts past n_tokens, that descend or are negative: which rows are written is open, but only rows of the call, lists that it has and pages of its
    tables are."""
    import paper_2601_17702_amd as s3
    T, P = 40, 16
    pr = paged.Problem(25, "bf16", 64, P, 4, 2, [20, 10, 10], [100, 60, 40])
    qs = torch.tensor(starts, dtype=torch.int32, device="cuda")
    kv_len, table = pr.args()
    q = pr.q.cuda()
    c = pr.cache(signatures=True)
    c.sig.zero_()
    unused = [p for p in range(pr.n_pages) if p not in set(pr.table.flatten().tolist())]
    before = [t[unused].clone() for t in (c.k, c.v, c.sig)]
    whole, out = guarded(T, 4, 64, dtype=pr.dtype, value=9.0)
    c.append(q[:, :2], q[:, 2:], kv_len, table, q_start=qs, q=q, q_out=out)
    assert torch.all(whole[:64] == 9) and torch.all(whole[64 + T:] == 9)
    assert all(torch.equal(t[unused], b) for t, b in zip((c.k, c.v, c.sig), before))
    for max_new in (40, 4):
        whole, out = guarded(T, 4, 64, dtype=pr.dtype, value=9.0)
        c.attention(q, kv_len, table, q_start=qs, max_new=max_new, out=out)
        assert torch.all(whole[:64] == 9) and torch.all(whole[64 + T:] == 9)
        for qb in (1, 8, 40):
            sel = c.select(q, kv_len, table, 6, q_start=qs, q_block=qb, lead=1, tail=0, max_new=max_new)
            assert torch.all((sel >= -1) & (sel < table.shape[1]))
            whole, lists = guarded(*sel.shape, dtype=torch.int32, value=-9)
            b = c._batch(T, kv_len, table, qs, max_new, None)
            ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
            assert s3.lib().s3_block_select(c._c, b, q.data_ptr(), 4, q.stride(0), q.stride(1), qb, 6, 1, 0, lists.data_ptr(), ws.data_ptr(), 1 << 24, s3._stream()) == 0
            assert torch.equal(lists, sel) and torch.all(whole[:64] == -9) and torch.all(whole[64 + len(sel):] == -9)
            whole, out = guarded(T, 4, 64, dtype=pr.dtype, value=9.0)
            c.block_attention(q, kv_len, table, sel, q_start=qs, q_block=qb, max_new=max_new, out=out)
            assert torch.all(whole[:64] == 9) and torch.all(whole[64 + T:] == 9)


@pytest.mark.parametrize("inter", [False, True])
def test_explicit_positions_outside_the_table(inter):
    """They are taken as the table's first or last row: in the four-token path, in the others and for keys."""
    import paper_2601_17702_amd as s3
    T, n_pos = 600, 50
    pr = paged.Problem(26, "bf16", 128, 64, 32, 2, [T], [T])
    c = pr.cache(signatures=True)
    pos = torch.randint(-60, 120, (T,), generator=pr.g, dtype=torch.int32)
    pos[:4] = torch.tensor([-(1 << 31), (1 << 31) - 1, -1, n_pos])
    rope = s3.rope_table(n_pos, 128)
    args = dict(q_start=pr.q_start.cuda(), rope=rope, interleaved=inter, q=pr.q.cuda())
    k = torch.cat(pr.rows_k).cuda()
    caches = []
    for p in (pos, pos.clamp(0, n_pos - 1)):
        out = c.append(k, k, pr.kv_len.cuda(), pr.table.cuda(), positions=p.cuda(), **args)
        caches.append((out.clone(), c.k.clone(), c.sig.clone()))
    assert all(torch.equal(a, b) for a, b in zip(*caches))
    short = s3.rope_table(T, 128)                                      # positions inside: another result
    out = c.append(k, k, pr.kv_len.cuda(), pr.table.cuda(), **{**args, "rope": short})
    assert not torch.equal(out, caches[0][0])


@pytest.mark.parametrize("dtype,d,new,kv", [("bf16", 64, [1], [70]), ("bf16", 128, [1], [3000]), ("bf16", 128, [150], [200]), ("fp32", 64, [90], [90]), ("fp32", 256, [3], [40])])
def test_an_infinite_value_of_next_to_no_weight(dtype, d, new, kv):
    """A token with a score hundreds below the others', an infinite value in one of its channels: that channel is infinite or NaN for the
    rows that see it, wherever in the call the token lies, the other channels are as without it."""
    for at in (0, kv[0] - new[0] // 2 - 1):
        pr = paged.Problem(27 + d, dtype, d, 32, 4, 2, new, kv)
        pr.q[..., 0] = 4.0
        pr.rows_k[0][..., 0] = 0.0
        pr.rows_k[0][at, :, 0] = -400.0                                # scaled by 1 below: 1600 under the others
        pr.rows_v[0][at, :, 5] = float("inf")
        kv_len, table = pr.args()
        o, _ = pr.cache().attention(pr.q.cuda(), kv_len, table, q_start=pr.q_start.cuda(), scale=1.0)
        o = o.cpu().to(torch.float64)
        sees = torch.arange(kv[0] - new[0], kv[0]) >= at
        alone = (torch.arange(kv[0] - new[0], kv[0]) == 0) & (at == 0)  # a prompt's first row sees nothing else
        assert not torch.isfinite(o[sees][:, :, 5]).any() and torch.isfinite(o[~sees]).all()
        pr.rows_v[0][at, :, 5] = 0.0
        want, _, tol, _ = paged.attend(pr, scale=1.0)
        rest = torch.arange(d) != 5
        assert torch.all((o - want).abs()[:, :, rest] <= tol[:, :, rest]) and (not alone.any() or torch.isinf(o[alone][:, :, 5]).all())


def test_starts_whose_counts_pass_31_bits():
    """2^15 sequences that all claim the same 2^16 tokens: the number of their lists wraps, where the array is written does not."""
    import paper_2601_17702_amd as s3
    T = n_seq = 1 << 16
    c = s3.KVCache(1, 16, 1, 64, signatures=True)
    c.sig.zero_()
    qs = (torch.arange(n_seq + 1, device="cuda") % 2 * T).to(torch.int32)
    kv_len = torch.full((n_seq,), 16, dtype=torch.int32, device="cuda")
    table = torch.zeros(n_seq, 1, dtype=torch.int32, device="cuda")
    q = torch.ones(T, 1, 64, dtype=torch.bfloat16, device="cuda")
    b = c._batch(T, kv_len, table, qs, T, 16)
    tiles = s3.lib().s3_block_tiles(b, 1)
    whole, sel = guarded(tiles, 1, 4, dtype=torch.int32, value=-9)
    assert s3.lib().s3_block_select_workspace(c._c, b, 1, 1, 4) == 0
    assert s3.lib().s3_block_select(c._c, b, q.data_ptr(), 1, 64, 64, 1, 4, 1, 1, sel.data_ptr(), None, 0, s3._stream()) == 0
    assert torch.all(whole[:64] == -9) and torch.all(whole[64 + tiles:] == -9) and torch.all((sel == -1) | (sel == 0))


@pytest.mark.parametrize("rot,theta", [(128, 10000.0), (64, 500000.0)])
def test_rotation_table_of_far_positions(rot, theta):
    """Angles up to 131071 radians: formed in 64 bits they are good to 1e-10, cos and sin are rounded once."""
    import paper_2601_17702_amd as s3
    n = 131072
    table = s3.rope_table(n, rot, theta).cpu().to(torch.float64)
    ang = torch.arange(n, dtype=torch.float64)[:, None] * theta ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    assert torch.all((table - torch.cat([ang.cos(), ang.sin()], 1)).abs() <= 2.0 ** -25 + 1e-9)


@pytest.mark.parametrize("dtype,d,n_seq,hkv,G,kv,top,fused", [
    ("bf16", 64, 32, 8, 4, 6500, 20, True),               # 256 lists of 407 candidates, one kernel
    ("bf16", 128, 80, 4, 2, 6399, 8, True),
    ("fp32", 64, 65, 4, 1, 7000, 40, True),
    ("bf16", 256, 32, 8, 3, 6401, 9, True),
    ("bf16", 64, 32, 8, 4, 6000, 20, False),              # 375 candidates: through scratch
    ("bf16", 128, 100, 8, 1, 300, 7, False),              # many short lists
    ("bf16", 64, 30, 8, 2, 9000, 33, False),              # 240 lists
])
def test_select_for_batches_of_single_tokens(dtype, d, n_seq, hkv, G, kv, top, fused):
    import numpy as np
    import paper_2601_17702_amd as s3
    pr = paged.Problem(28 + kv, dtype, d, 16, hkv * G, hkv, [1] * n_seq, [1] * n_seq, spare=600 - n_seq)
    pr.kv = [kv - 7 * s for s in range(n_seq)] if n_seq < 40 else [kv] * n_seq       # lengths that the pages below stand for
    nb = -(-kv // 16)
    pr.table = torch.randint(0, pr.n_pages, (n_seq, nb), generator=pr.g, dtype=torch.int32)
    pr.table[:, 5] = -1
    sig = torch.from_numpy(paged.grid8(torch.randn(pr.n_pages, hkv, d, generator=pr.g).numpy())).to(torch.bfloat16)
    c = s3.KVCache(pr.n_pages, 16, hkv, d, pr.dtype, sig=sig.cuda())
    kv_len, table = torch.tensor(pr.kv, dtype=torch.int32, device="cuda"), pr.table.cuda()
    b = c._batch(n_seq, kv_len, table, None, 1, kv)
    assert (s3.lib().s3_block_select_workspace(c._c, b, hkv * G, 1, top) == 0) == fused
    sel = c.select(pr.q.cuda(), kv_len, table, top, lead=2, tail=1, max_kv=kv)
    assert np.array_equal(sel.cpu().numpy(), paged.select(pr, sig, top, 1, 2, 1))
