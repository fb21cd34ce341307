"""GPU checks at the ends of what the capped and 8-bit calls take: log-sum-exps under large caps, outputs at 16 modulo 32 bytes."""
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
