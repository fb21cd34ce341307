"""CPU-only checks of the 8-bit cache's entry points and those beside it: bad arguments are refused on the host, before anything touches a GPU; and
of the plain forms that the GPU checks hold them to."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2601_17702_amd as s3
from tests import paged8
from tests.test_paged_args import ONE, batch
from tests.test_paged_args import cache as cache16


def cache(k=ONE, v=ONE, scale=ONE, sig=ONE, n_pages=8, page=64, heads=2, d=128):
    return s3._KV8_CACHE.pack(k, v, scale, sig, n_pages, page, heads, d)


def norm(q=ONE, k=ONE, qs=0, ks=0, eps=1e-6):
    return s3._KV_NORM.pack(q, k, qs, ks, eps)


LONG = dict(max_kv=4096, max_pages=64, stride=64)       # of which no workgroup takes a tile whole


def attend(c=None, b=None, q=ONE, n_q=8, ts=1024, hs=128, scale=0.1, cap=0.0, window=0, out=ONE, ws=ONE, ws_bytes=1 << 40):
    return s3.lib().s3_kv8_attention(c or cache(), b or batch(), q, n_q, ts, hs, scale, cap, window, out, None, ws, ws_bytes, None)


def listed(c=None, b=None, sel=ONE, q_block=16, top=4, ws=ONE, ws_bytes=1 << 40, n_q=8, cap=0.0):
    return s3.lib().s3_kv8_block_attention(c or cache(), b or batch(), ONE, n_q, 1024, 128, sel, q_block, top, 0.1, cap, ONE, None, ws, ws_bytes, None)


def append(c=None, b=None, k=ONE, kt=256, kh=128, v=ONE, rope=None, n_pos=100, rot=128, q=None, n_q=8, q_out=ONE, qt=1024, w=None, eight=True):
    fn = s3.lib().s3_kv8_append if eight else s3.lib().s3_kv_append_norm
    return fn(c or (cache() if eight else cache16()), b or batch(), k, kt, kh, v, 256, 128, rope, n_pos, rot, 0, None, q, n_q, qt, 128, q_out, w, None)


def read(c=None, b=None, pos=None, k=ONE, v=ONE, eight=True):
    return s3.lib().s3_kv8_read(c or cache(), b or batch(), pos, k, v, None) if eight else s3.lib().s3_kv_read(c or cache16(), b or batch(), pos, k, v, None)


def capped(c=None, b=None, cap=30.0, scale=0.1, window=0, ws=ONE, ws_bytes=1 << 40):
    return s3.lib().s3_paged_attention_capped(c or cache16(), b or batch(), ONE, 8, 1024, 128, scale, cap, window, ONE, None, ws, ws_bytes, None)


@pytest.mark.parametrize("bad", [
    dict(k=0), dict(v=0), dict(scale=0), dict(k=ONE + 16), dict(scale=ONE + 64), dict(sig=ONE + 2), dict(n_pages=0), dict(page=8), dict(page=48),
    dict(page=512), dict(heads=0), dict(heads=5000), dict(d=96), dict(d=32)])
def test_bad_caches(bad):
    for call in (attend, listed, append, read):
        assert call(c=cache(**bad)) == -1
    assert s3.lib().s3_kv8_attention_workspace(cache(**bad), batch(), 8) == 0
    assert s3.lib().s3_kv8_block_attention_workspace(cache(**bad), batch(), 8, 1, 4) == 0


@pytest.mark.parametrize("bad", [
    dict(kv_len=0), dict(table=0), dict(n_seq=-1), dict(n_tokens=-1), dict(max_pages=-1), dict(stride=15), dict(max_new=-1), dict(max_kv=-1),
    dict(qs=0), dict(max_pages=1 << 25, stride=1 << 25), dict(n_tokens=(1 << 24) + 1), dict(n_seq=(1 << 20) + 1)])
def test_bad_batches(bad):
    for call in (attend, listed, append, read, capped):
        assert call(b=batch(**bad)) == -1
    assert append(b=batch(**bad), eight=False, w=norm()) == -1 and read(b=batch(**bad), eight=False) == -1


def test_bad_arguments_of_each_call():
    nan, inf = float("nan"), float("inf")
    assert all(attend(**x) == -1 for x in (dict(q=0), dict(q=ONE + 8), dict(n_q=7), dict(n_q=0), dict(n_q=66), dict(ts=1020), dict(hs=130), dict(hs=64),
                                           dict(ts=-1024), dict(scale=0.0), dict(scale=nan), dict(scale=inf), dict(window=-1), dict(out=0), dict(out=ONE + 8),
                                           dict(ws=0, b=batch(**LONG)), dict(ws=ONE + 128, b=batch(**LONG)), dict(cap=-1.0), dict(cap=nan), dict(cap=inf), dict(cap=2e30), dict(cap=1e-20, scale=1e20)))
    assert b"s3_kv8_attention" in s3.lib().s3_last_error()
    assert attend(ws_bytes=16, b=batch(**LONG)) == -3
    assert all(listed(**x) == -1 for x in (dict(sel=0), dict(q_block=0), dict(top=0), dict(top=4097), dict(n_q=3), dict(ws=0, q_block=4, top=40), dict(cap=-0.5)))
    assert listed(ws_bytes=16, q_block=4, top=40) == -3
    assert all(capped(**x) == -1 for x in (dict(cap=0.0), dict(cap=-1.0), dict(cap=nan), dict(cap=inf), dict(window=-1), dict(ws=0), dict(scale=0.0)))
    assert capped(ws_bytes=16) == -3
    L = s3.lib()
    assert L.s3_block_attention_capped(cache16(), batch(), ONE, 8, 1024, 128, ONE, 16, 4, 0.1, 0.0, ONE, None, ONE, 1 << 40, None) == -1
    assert L.s3_block_attention_capped(cache16(), batch(), ONE, 8, 1024, 128, None, 16, 4, 0.1, 9.0, ONE, None, ONE, 1 << 40, None) == -1
    for eight in (True, False):
        more = dict(eight=eight, w=norm())
        assert all(append(**more, **x) == -1 for x in (dict(k=0), dict(v=0), dict(k=ONE + 4), dict(kt=257), dict(kh=100), dict(rope=ONE, rot=24), dict(rope=ONE, rot=0),
                                                       dict(rope=ONE, rot=144), dict(rope=ONE, n_pos=0), dict(rope=ONE + 4), dict(q=ONE, n_q=7),
                                                       dict(q=ONE, q_out=0), dict(q=ONE, qt=1021)))
        assert all(append(eight=eight, w=norm(**x)) == -1 for x in (dict(eps=0.0), dict(eps=-1.0), dict(eps=nan), dict(eps=inf), dict(q=ONE + 4), dict(k=ONE + 8),
                                                                    dict(qs=130), dict(ks=64), dict(ks=-128)))
        assert all(read(eight=eight, **x) == -1 for x in (dict(k=ONE + 8), dict(v=ONE + 2)))
        assert read(eight=eight, b=batch(n_tokens=1 << 24, n_seq=1), c=(cache if eight else cache16)(heads=4096)) == -1
    assert append(eight=False, w=None) == -1
    assert attend(c=None, b=batch()) != 0 and L.s3_kv8_attention(None, batch(), ONE, 8, 1024, 128, 0.1, 0.0, 0, ONE, None, ONE, 1 << 40, None) == -1


def test_nothing_to_do():
    empty = batch(n_seq=0, n_tokens=0)
    assert attend(b=empty, q=0, out=0, ws=0, ws_bytes=0) == 0 and append(b=empty, k=0, v=0) == 0 and read(b=empty, k=0, v=0) == 0
    assert append(b=empty, k=0, v=0, w=norm(), eight=False) == 0 and read(b=empty, eight=False) == 0 and capped(b=empty, ws=0, ws_bytes=0) == 0
    assert read(k=0, v=0) == 0


def test_sizes():
    assert s3._KV8_CACHE.size == 48 and s3._KV_NORM.size == 40 and C.sizeof(C.c_void_p) == 8
    L = s3.lib()
    for b, n_q in ((batch(n_tokens=600, max_new=600), 32), (batch(qs=0, n_tokens=2, max_new=1, max_kv=2000, max_pages=32, stride=32), 8)):
        assert L.s3_kv8_attention_workspace(cache(), b, n_q) == L.s3_paged_attention_workspace(cache16(), b, n_q) > 0


def test_scratch_of_tiles_that_one_workgroup_has():
    """None, where nothing is joined: few rows, and a bound of 1024 tokens, or of 2048 and a workgroup for every compute unit (lists: 8192)."""
    def need(n_seq, max_kv, max_new=1, heads=8, n_q=32):
        pages = -(-max_kv // 64)
        b = batch(qs=0 if max_new == 1 else ONE, n_seq=n_seq, n_tokens=n_seq * max_new, max_new=max_new, max_pages=pages, stride=pages, max_kv=max_kv)
        return s3.lib().s3_kv8_attention_workspace(cache(heads=heads), b, n_q)
    assert need(1, 1024) == need(32, 2048) == need(1, 1000, max_new=4) == 0
    assert need(1, 1025) > 0 and need(31, 2048) > 0 and need(64, 2049) > 0 and need(1, 1000, max_new=5) > 0
    lists = lambda top, n_seq: s3.lib().s3_kv8_block_attention_workspace(cache(heads=8), batch(qs=0, n_seq=n_seq, n_tokens=n_seq, max_new=1), 32, 1, top)  # noqa: E731
    assert lists(16, 1) == lists(128, 32) == 0 and lists(17, 1) > 0 and lists(129, 32) > 0


def test_plain_form_of_8_bits():
    """The values and codes that the GPU checks compare with, against torch's e4m3 and by hand."""
    assert np.array_equal(paged8.VALUES, torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy())
    g = torch.Generator().manual_seed(1)
    x = (torch.randn(500, 64, generator=g) * torch.exp(4 * torch.randn(500, 1, generator=g))).numpy()
    b, c = paged8.to8(x)
    y = torch.from_numpy(x).double() * torch.exp2(127.0 - torch.from_numpy(c).double())[:, None]
    assert float(y.abs().max()) <= 448 and torch.all(y.abs().amax(1) > 224)
    assert np.array_equal(y.float().to(torch.float8_e4m3fn).view(torch.uint8).numpy(), b)
    big = np.float32(448 * 2.0 ** 7)
    assert paged8.to8(np.array([[big], [np.nextafter(big, np.float32(1e9))], [0.0], [1e-44]]))[1].tolist() == [134, 135, 1, 1]
    b, c = paged8.to8(np.array([[np.inf, 448.0, np.nan, -1.0]]))
    assert c[0] == 127 and b[0, 0] == b[0, 2] == 0x7f and np.isnan(paged8.of8(b, c)[0, 0]) and paged8.of8(b, c)[0, 1] == 448.0


def test_plain_form_of_capped_scores():
    """A cap far above the scores changes nothing; one far below leaves the sign."""
    from tests import paged
    pr = paged.Problem(1, "fp32", 64, 16, 4, 2, [3], [20])
    for a, b in zip(paged8.attend(pr, 1e9)[:2], paged.attend(pr)[:2]):
        assert torch.allclose(a, b, rtol=1e-9, atol=1e-12)
    out, lse, _, _ = paged8.attend(pr, 1e-9)
    assert torch.allclose(lse[2], torch.full((4,), float(np.log(20.0)), dtype=torch.float64))
    assert torch.allclose(out[2, 0], pr.rows_v[0][:, 0].double().mean(0))
