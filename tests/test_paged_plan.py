"""CPU-only checks of how much scratch the paged cache's calls ask for (heads of 128 channels in bf16 unless said)."""
import pytest

import paper_2601_17702_amd as s3
from tests.test_paged_args import batch, cache


def scratch(n_seq, n_tokens, max_new, max_kv, n_q=32, heads=8, d=128, dtype=0):
    c = cache(n_pages=1 << 20, heads=heads, d=d, dtype=dtype)
    pages = -(-max_kv // 64)
    return s3.lib().s3_paged_attention_workspace(c, batch(n_seq=n_seq, n_tokens=n_tokens, max_pages=pages, stride=pages, max_new=max_new, max_kv=max_kv), n_q)


@pytest.mark.parametrize("n_seq,n_tokens,max_new,max_kv,n_q,heads", [
    (64, 64, 64, 32768, 32, 8),              # single tokens with starts, the bound of a sequence's new tokens left at its default
    (256, 256, 256, 32768, 32, 8),
    (16, 16, 16, 131072, 32, 8),
    (43, 298, 256, 131072, 8, 8),            # one chunk beside single tokens
    (9, 2048 + 240, 2048, 131072, 32, 8),    # a long chunk beside short turns
    (64, 4096, 4096, 32768, 28, 4),
])
def test_scratch_of_parts_is_bounded(n_seq, n_tokens, max_new, max_kv, n_q, heads):
    """Parts are cut until some 2048 workgroups are there, whatever the bounds of a call say, and only for row tiles that can be there: a part of 256
    rows holds 256 * 130 floats, so 2048 of them 273 MB; the streaming kernel's two per workgroup 34 MB at most beside that."""
    assert scratch(n_seq, n_tokens, max_new, max_kv, n_q, heads) <= 2048 * 256 * 130 * 4 + 1024 * 32 * 130 * 4


def test_scratch_of_a_decoding_batch_without_a_bound():
    """64 single tokens of which the host says only that there are 64: at most 7 sequences can have the 33 rows that make a chunk."""
    assert scratch(64, 64, 64, 32768) <= 128 << 20
    assert scratch(64, 64, 1, 32768) <= 4 << 20


@pytest.mark.parametrize("G", [1, 3, 7, 8])
@pytest.mark.parametrize("d,dtype", [(64, 0), (128, 0), (256, 1)])
def test_slots_of_the_streaming_kernel_are_whole_pieces(G, d, dtype):
    """512 workgroups have two slots each, which are written and read 16 bytes at a time, for odd numbers of rows, too."""
    slot, rest = divmod(scratch(4, 4, 1, 4096, 2 * G, 2, d, dtype), 1024)
    assert rest == 0 and slot % 16 == 0 and slot >= G * (d + 2) * 4


def attend(b, heads, G=1):
    return s3.lib().s3_paged_attention(cache(heads=heads), b, 4096, heads * G, 1 << 20, 128, 0.1, 0, 4096, None, 4096, 1 << 50, None)


def test_calls_too_large_for_one_launch_are_refused_before_any():
    """S3_EINVAL on the host, with nothing launched (where there is no GPU a launch gives S3_EHIP)."""
    wide = dict(max_pages=16, stride=16, max_kv=1024)
    # 2^20 single tokens of 8 heads: a join of 2^23 workgroups
    assert attend(batch(qs=0, n_seq=1 << 20, n_tokens=1 << 20, max_new=1, **wide), 8) == -1
    # short turns are few, but not the tiles of the chunks beside them: the kernel of the short ones is not launched either
    assert attend(batch(n_seq=3, n_tokens=300000, max_new=150000, **wide), 4096) == -1
    assert b"too many" in s3.lib().s3_last_error()
    def choose(n_tokens, heads, max_kv, page=16):
        pages = -(-max_kv // page)
        b = batch(n_seq=1, n_tokens=n_tokens, max_new=n_tokens, max_pages=pages, stride=pages, max_kv=max_kv)
        return s3.lib().s3_block_select(cache(page=page, heads=heads), b, 4096, heads * 32, 1 << 20, 128, 1, 16, 1, 1, 4096, 4096, 1 << 50, None)
    # 2^23 lists of 512 threads are 2^32 threads
    assert choose(1 << 13, 1 << 10, 1024) == -1
    assert b"too many" in s3.lib().s3_last_error()
    assert choose(1 << 15, 8, 1 << 20) == -1 and choose(1, 1, 1 << 30) == -1


def test_scratch_in_host_memory_is_refused():
    """A kernel would follow its address."""
    import torch
    q, c = torch.zeros(1, 8, 128), s3.KVCache.__new__(s3.KVCache)
    with pytest.raises(AssertionError):
        c._out(q, None, True, 256, torch.zeros(4096, dtype=torch.uint8))
    assert c._out(q, None, False, 0, None)[2] is None


def test_a_table_without_columns_is_no_error():
    """Sequences that have no page yet: the table is empty, and so is its address."""
    L, b = s3.lib(), batch(table=0, max_pages=0, stride=0)
    assert L.s3_paged_attention_workspace(cache(), b, 8) > 0 and L.s3_block_attention_workspace(cache(), b, 8, 1, 4) > 0
    assert L.s3_paged_attention_workspace(cache(), batch(table=0, max_pages=1, stride=1), 8) == 0


def test_which_choices_go_through_scratch():
    """Scores of a decoding batch's lists are left in scratch unless there is a list for every compute unit, and 400 candidates in it."""
    def scratch_of(n_seq, nb, max_new=1, n_tokens=None, q_block=1, heads=8):
        b = batch(n_seq=n_seq, n_tokens=n_tokens or n_seq, max_new=max_new, max_pages=nb, stride=nb, max_kv=nb * 64)
        return s3.lib().s3_block_select_workspace(cache(heads=heads), b, 32, q_block, 32)
    for n_seq, nb in ((8, 2000), (8, 8000), (16, 3000), (32, 300), (512, 100), (1, 100)):
        assert scratch_of(n_seq, nb) >= n_seq * 8 * nb * 4, (n_seq, nb)
    for n_seq, nb in ((32, 500), (64, 512), (512, 500), (64, 8000)):
        assert scratch_of(n_seq, nb) == 0, (n_seq, nb)
    assert scratch_of(1, 2000, 16, 16, 16) > 0 and scratch_of(1, 200, 16, 16, 16) == 0 and scratch_of(1, 2000, 256, 256, 16) == 0
