"""GPU checks at the ends of what the capped and 8-bit calls take: log-sum-exps under large caps, both forms of a cap on either side of where they change over, outputs at 16 modulo 32 bytes."""
import numpy as np
import pytest
import torch

from tests import paged, paged8

pytestmark = pytest.mark.gpu


def run(pr, c, **more):
    kv_len, table = pr.args()
    return c.attention(pr.q.cuda(), kv_len, table, q_start=pr.q_start.cuda(), want_lse=True, **more)


@pytest.mark.parametrize("cap", [5.0, 50.0, 200.0, 2048.0])
@pytest.mark.parametrize("dtype,d,hq,hkv,new,kv", [
    ("bf16", 128, 8, 2, [1, 1, 1], [1, 63, 3000]),            # 16 rows a tile, whole and joined
    ("e4m3", 128, 8, 2, [1, 1, 1], [1, 63, 3000]),
    ("e4m3", 64, 8, 2, [1, 1], [7, 900]),
    ("bf16", 256, 20, 1, [1, 2], [3, 2500]),                  # 32 rows a tile
    ("e4m3", 64, 16, 1, [3, 1], [1777, 40]),                  # two row sets
    ("bf16", 64, 4, 2, [150], [333]),                         # many rows
    ("e4m3", 128, 4, 1, [300], [301]),
    ("bf16", 128, 4, 1, [70], [9000]),                        # their tokens in parts
])
def test_lse_of_scores_of_zero(dtype, d, hq, hkv, new, kv, cap):
    """With queries of zero every score is 0 and a row's lse the logarithm of how many tokens it sees, whatever the cap: exp2(0), 1 / 2 and the weights' sum
    are exact.  What is left is log2 (a unit of 2^-23 of itself at most), ln 2 as a constant (2^-25) and their product (2^-24): 2^-22 in all."""
    pr = paged8.problem(dtype, d + len(kv), d, 32, hq, hkv, new, kv)
    pr.q.zero_()
    sees = torch.cat([torch.arange(m - n + 1, m + 1) for n, m in zip(new, kv)]).to(torch.float64)
    for bounds in ({}, {"max_new": max(new), "max_kv": max(kv)}):
        _, lse = run(pr, pr.cache(), softcap=cap, **bounds)
        want = torch.log(sees)[:, None]
        assert torch.all((lse.cpu().to(torch.float64) - want).abs() <= 2.0 ** -22 * want)


LEVELS = [0.0, 0.1, 0.3, 0.34, 0.36, 0.5, 1.0, 2.0, 3.0]


@pytest.mark.parametrize("cap", [2048.0, float(np.nextafter(np.float32(2048.0), np.float32(1e9))), 4096.0])
@pytest.mark.parametrize("dtype,d,hq,hkv,new,n", [
    ("bf16", 64, 8, 2, 1, 700), ("bf16", 128, 16, 1, 1, 90), ("bf16", 256, 32, 1, 1, 300), ("bf16", 64, 16, 1, 4, 200), ("bf16", 128, 8, 2, 150, 400),
    ("e4m3", 128, 8, 2, 1, 700), ("e4m3", 64, 16, 2, 2, 90), ("e4m3", 256, 20, 1, 1, 300), ("e4m3", 64, 16, 1, 4, 200), ("e4m3", 64, 9, 3, 150, 400),
    ("fp32", 64, 9, 1, 2, 300), ("fp32", 128, 8, 1, 100, 200),
])
def test_caps_where_the_form_changes(dtype, d, hq, hkv, new, n, cap):
    """Rows of bf16 take one form of the cap up to 2048 and the other above, which has a series for |z| < 0.35 and an exponential beyond.  A query has two channels that are not zero: with
    the first, over keys of 1 there, it sets its row's z = score / cap between -3 and 3, neighbouring rows on either side of 0.35, and with the second it spreads the
    capped scores by about 1, so that many tokens count.

    A score is a sum of two products, off by 2 2^-24 of their magnitudes; capped it is off by 2^-20 of itself, its scaled value by 2^-23, and up to 2048 over bf16 by 2^-22 of the cap; exp2
    is good to 2^-21; weights, sums, logarithm and results are as in paged.attend."""
    pr = paged8.problem(dtype, d + new, d, 32, hq, hkv, [new], [n])
    pr.rows_k[0][:, :, 0] = 1.0
    if dtype == "e4m3":
        pr.quantise()
    assert torch.all(pr.rows_k[0][:, :, 0] == 1.0)
    level = torch.tensor(LEVELS, dtype=torch.float64)[torch.arange(new * hq) % 9] * torch.where(torch.arange(new * hq) % 2 == 0, 1.0, -1.0)
    pr.q.zero_()
    pr.q[:, :, 0] = (cap * level).view(new, hq).to(pr.dtype)
    pr.q[:, :, 1] = (1.0 / (1.0 - torch.tanh(level) ** 2)).view(new, hq).to(pr.dtype)
    out, lse = (x.cpu().to(torch.float64) for x in run(pr, pr.cache(), softcap=cap, scale=1.0, max_new=new, max_kv=n))
    fp = dtype == "fp32"
    G, bits = hq // hkv, 0.0 if fp else 2.0 ** -8
    hidden = torch.arange(n)[None] > n - new + torch.arange(new)[:, None]
    for h in range(hq):
        K, V = pr.rows_k[0][:, h // G].to(torch.float64), pr.rows_v[0][:, h // G].to(torch.float64)
        a, b = pr.q[:, h, :1].to(torch.float64), pr.q[:, h, 1:2].to(torch.float64) * K[:, 1]
        s = cap * torch.tanh((a + b) / cap)
        e = 2.0 ** -23 * (a.abs() + b.abs()) + (2.0 ** -20 + 2.0 ** -23) * s.abs() + (2.0 ** -22 * cap if not fp and cap <= 2048 else 0.0)
        e = e.masked_fill(hidden, 0.0).amax(1, keepdim=True) + 2.0 ** -21
        s = s.masked_fill(hidden, -float("inf"))
        p = torch.softmax(s, 1)
        o, l64 = p @ V, torch.logsumexp(s, 1)
        tol = (2 * e + n * 2.0 ** -24 + bits) * (p @ V.abs()) + (bits or 2.0 ** -24) * 1.01 * o.abs()
        assert torch.all((out[:, h] - o).abs() <= tol), (h, float(((out[:, h] - o).abs() / tol).max()))
        assert torch.all((lse[:, h] - l64).abs() <= e[:, 0] + n * 2.0 ** -24 + 2.0 ** -22 * l64.abs()), h


@pytest.mark.parametrize("dtype", ["e4m3", "bf16", "fp32"])
@pytest.mark.parametrize("d,new", [(64, 40), (128, 3), (256, 33)])
def test_read_into_outputs_aligned_to_16_bytes(dtype, d, new):
    """k_out and v_out that begin 16 bytes into their storage, rows in order and far apart: the same bits, and nothing beside them."""
    pr = paged8.problem(dtype, 31 + d, d, 32, 2, 2, [new], [new + 60])
    c = pr.cache()
    kv_len, table = pr.args()
    e = 16 // pr.dtype.itemsize
    for positions in (None, torch.arange(new, dtype=torch.int32, device="cuda") * 37 % (new + 60)):
        same = dict(q_start=pr.q_start.cuda(), positions=positions)
        want = c.read(kv_len, table, new, **same)
        rooms = [torch.full((new * 2 * d + 2 * e,), 3.0, dtype=pr.dtype, device="cuda") for _ in "kv"]
        outs = [x[e:-e].view(new, 2, d) for x in rooms]
        assert all(x.data_ptr() % 32 == 16 for x in outs)
        c.read(kv_len, table, new, k_out=outs[0], v_out=outs[1], **same)
        for room, out, w in zip(rooms, outs, want):
            assert torch.equal(out, w) and torch.all(room[:e] == 3.0) and torch.all(room[-e:] == 3.0)
