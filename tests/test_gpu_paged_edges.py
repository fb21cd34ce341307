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
