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
