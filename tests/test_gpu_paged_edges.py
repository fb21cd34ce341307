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
