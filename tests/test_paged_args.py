"""CPU-only checks of the paged cache's entry points: bad arguments are refused on the host, before anything touches a GPU; sizes
of workspaces and lists."""
import ctypes as C

import pytest

import paper_2601_17702_amd as s3

ONE = 4096                                   # an address that is never followed: validation fails first


def cache(k=ONE, v=ONE, sig=ONE, dtype=0, n_pages=8, page=64, heads=2, d=128):
    return s3._KV_CACHE.pack(k, v, sig, dtype, n_pages, page, heads, d)


def batch(qs=ONE, kv_len=ONE, table=ONE, stride=16, n_seq=2, n_tokens=10, max_pages=16, max_new=10, max_kv=1024):
    return s3._KV_BATCH.pack(qs, kv_len, table, stride, n_seq, n_tokens, max_pages, max_new, max_kv)


def attend(c=None, b=None, q=ONE, n_q=8, ts=1024, hs=128, scale=0.1, window=0, out=ONE, ws=ONE, ws_bytes=1 << 40):
    return s3.lib().s3_paged_attention(c or cache(), b or batch(), q, n_q, ts, hs, scale, window, out, None, ws, ws_bytes, None)


def listed(c=None, b=None, sel=ONE, q_block=16, top=4, ws=ONE, ws_bytes=1 << 40, n_q=8):
    return s3.lib().s3_block_attention(c or cache(), b or batch(), ONE, n_q, 1024, 128, sel, q_block, top, 0.1, ONE, None, ws, ws_bytes, None)


def choose(c=None, b=None, q_block=16, top=8, lead=1, tail=1, sel=ONE, ws=ONE, ws_bytes=1 << 40, n_q=8):
    return s3.lib().s3_block_select(c or cache(), b or batch(), ONE, n_q, 1024, 128, q_block, top, lead, tail, sel, ws, ws_bytes, None)


def append(c=None, b=None, k=ONE, kt=256, kh=128, v=ONE, rope=None, n_pos=100, rot=128, q=None, n_q=8, q_out=ONE, qt=1024):
    return s3.lib().s3_kv_append(c or cache(), b or batch(), k, kt, kh, v, 256, 128, rope, n_pos, rot, 0, None, q, n_q, qt, 128, q_out, None)


@pytest.mark.parametrize("bad", [
    dict(k=0), dict(v=0), dict(k=ONE + 16), dict(sig=ONE + 2), dict(dtype=2), dict(n_pages=0), dict(page=8), dict(page=48), dict(page=512),
    dict(heads=0), dict(heads=5000), dict(d=96), dict(d=32)])
def test_bad_caches(bad):
    for call in (attend, listed, choose, append):
        assert call(c=cache(**bad)) == -1
    assert s3.lib().s3_paged_attention_workspace(cache(**bad), batch(), 8) == 0
    assert s3.lib().s3_block_select_workspace(cache(**bad), batch(), 8, 1, 4) == 0


@pytest.mark.parametrize("bad", [
    dict(kv_len=0), dict(table=0), dict(n_seq=-1), dict(n_tokens=-1), dict(max_pages=-1), dict(stride=15), dict(max_new=-1), dict(max_kv=-1),
    dict(qs=0), dict(max_pages=1 << 25, stride=1 << 25), dict(n_tokens=(1 << 24) + 1), dict(n_seq=(1 << 20) + 1)])
def test_bad_batches(bad):
    for call in (attend, listed, choose, append):
        assert call(b=batch(**bad)) == -1


def test_bad_arguments_of_each_call():
    assert all(attend(**x) == -1 for x in (dict(q=0), dict(q=ONE + 8), dict(n_q=7), dict(n_q=0), dict(n_q=66), dict(ts=1020), dict(hs=130), dict(hs=64),
                                           dict(ts=-1024), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
                                           dict(window=-1), dict(out=0), dict(out=ONE + 8), dict(ws=0), dict(ws=ONE + 128)))
    assert b"s3_paged_attention" in s3.lib().s3_last_error()
    assert attend(ws_bytes=16) == -3
    assert all(listed(**x) == -1 for x in (dict(sel=0), dict(q_block=0), dict(top=0), dict(top=4097), dict(n_q=3), dict(ws=0, q_block=4)))
    assert listed(ws_bytes=16, q_block=4) == -3
    assert all(choose(**x) == -1 for x in (dict(q_block=0), dict(top=0), dict(top=4097), dict(lead=-1), dict(tail=-1), dict(top=2), dict(lead=9, tail=0),
                                           dict(sel=0), dict(c=cache(sig=0)), dict(n_q=9)))
    assert all(append(**x) == -1 for x in (dict(k=0), dict(v=0), dict(k=ONE + 4), dict(kt=257), dict(kh=100), dict(rope=ONE, rot=24), dict(rope=ONE, rot=0),
                                           dict(rope=ONE, rot=144), dict(rope=ONE, n_pos=0), dict(rope=ONE + 4), dict(q=ONE, n_q=7), dict(q=ONE, q_out=0),
                                           dict(q=ONE, qt=1021)))
    L = s3.lib()
    assert all(L.s3_rope_table(*x, None) == -1 for x in ((0, 4, 64, 1e4), (ONE, -1, 64, 1e4), (ONE, 4, 24, 1e4), (ONE, 4, 272, 1e4), (ONE, 4, 64, 0.0),
                                                         (ONE, 4, 64, float("nan")), (ONE + 4, 4, 64, 1e4)))
    assert L.s3_paged_attention(None, batch(), ONE, 8, 1024, 128, 0.1, 0, ONE, None, ONE, 1 << 40, None) == -1


def test_nothing_to_do():
    empty = batch(n_seq=0, n_tokens=0)
    assert attend(b=empty, q=0, out=0, ws=0, ws_bytes=0) == 0 and append(b=empty, k=0, v=0) == 0 and choose(b=empty, sel=0, ws=0) == 0
    assert s3.lib().s3_rope_table(ONE, 0, 64, 1e4, None) == 0


def test_sizes():
    L = s3.lib()
    assert L.s3_block_tiles(batch(n_seq=3, n_tokens=10), 1) == 10
    assert L.s3_block_tiles(batch(n_seq=3, n_tokens=10), 4) == (10 + 9) // 4 and L.s3_block_tiles(batch(), 0) == 0
    small = L.s3_paged_attention_workspace(cache(), batch(n_tokens=2, max_new=1), 8)
    assert 0 < small <= L.s3_paged_attention_workspace(cache(), batch(n_tokens=64, max_new=63), 8) and small % 256 == 0
    assert C.sizeof(C.c_void_p) == 8 and s3._KV_CACHE.size == 48 and s3._KV_BATCH.size == 56
