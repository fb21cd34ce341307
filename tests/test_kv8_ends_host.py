"""CPU-only checks beside tests/test_gpu_kv8_ends.py."""
import glob
import os
import re

import pytest

import paper_2601_17702_amd as s3
from tests.conftest import ROOT
from tests.test_kv8_args import cache as cache8
from tests.test_paged_args import ONE, batch
from tests.test_paged_args import cache as cache16

BYTES = {"__bf16": 2, "float": 4, "unsigned": 4, "int": 4, "_Float16": 2, "double": 8}


def test_no_access_is_wider_than_what_callers_align():
    """Callers align to 16 bytes: no memory is read or written through a vector type of more, whose own alignment is its size."""
    sources = {f: open(f).read() for p in ("*.hip", "*.h", "*.inc") for f in glob.glob(os.path.join(ROOT, "paper_2601_17702_amd/csrc", p))}
    wide = set()
    for text in sources.values():
        for n, of, name in re.findall(r"typedef __attribute__\(\(ext_vector_type\((\d+)\)\)\) (\w+) (\w+);", text):
            if of in BYTES and int(n) * BYTES[of] > 16:
                wide.add(name)
    assert "kv_f32x16" in wide                            # the matrix instructions' accumulators
    for f, text in sources.items():
        for name in wide:
            assert not re.search(r"\((?:const )?%s\s*\*\)" % name, text), (f, name)


@pytest.mark.parametrize("dtype", [s3.S3_BF16, s3.S3_FP32, "e4m3"])
@pytest.mark.parametrize("d,heads,G", [(64, 1, 1), (128, 8, 4), (256, 2, 7), (128, 3, 16), (64, 4, 32), (256, 64, 2)])
def test_scratch_of_one_tile_is_enough_for_any_lists_of_few_rows(dtype, d, heads, G):
    """Of listed blocks the batch that takes most is one tile of queries, whatever the chunks' lengths."""
    L = s3.lib()
    c = cache8(heads=heads, d=d) if dtype == "e4m3" else cache16(heads=heads, d=d, dtype=dtype)
    need = L.s3_kv8_block_attention_workspace if dtype == "e4m3" else L.s3_block_attention_workspace
    for q_block in {1, 2, 32 // G, 64}:
        for max_new in (1, 2, 5, 64, 1000):
            t = min(max_new, q_block)
            if t < 1 or t * G > 32:
                continue
            for top in (1, 16, 17, 128, 129, 4096):
                one = need(c, batch(n_seq=1, n_tokens=t, max_new=t), heads * G, q_block, top)
                for n_seq, n_tokens in ((1, 1), (1, t), (1, max_new), (2, 1), (2, max_new + 1), (3, 3 * max_new), (40, 40), (40, 40 * max_new), (300, 300 * max_new)):
                    assert need(c, batch(n_seq=n_seq, n_tokens=n_tokens, max_new=max_new), heads * G, q_block, top) <= one, (q_block, max_new, top, n_seq, n_tokens)


@pytest.mark.parametrize("dtype", [s3.S3_BF16, s3.S3_FP32, "e4m3"])
@pytest.mark.parametrize("d,heads,G", [(64, 1, 1), (128, 8, 4), (256, 2, 7), (128, 3, 16), (64, 4, 32), (256, 64, 2)])
def test_scratch_of_one_sequence_is_enough_for_any_batch_of_few_rows(dtype, d, heads, G):
    """A buffer that a program keeps while sequences come and go: sized for one sequence, it holds for every number of them, and for shorter bounds than its own."""
    L = s3.lib()
    c = cache8(heads=heads, d=d) if dtype == "e4m3" else cache16(heads=heads, d=d, dtype=dtype)
    all_of = L.s3_kv8_attention_workspace if dtype == "e4m3" else L.s3_paged_attention_workspace

    def many(n_seq, max_new, max_kv):
        pages = -(-max_kv // 64)
        return batch(qs=ONE, n_seq=n_seq, n_tokens=n_seq * max_new, max_new=max_new, max_pages=pages, stride=pages, max_kv=max_kv)
    seen = set()
    for max_new in {1, 2, 32 // G}:
        if not 1 <= max_new * G <= 32:
            continue
        for max_kv in (1, 1000, 1024, 1025, 2048, 2049, 8192, 8193, 131072):
            one = all_of(c, many(1, max_new, max_kv), heads * G)
            for n_seq in (1, 2, 3, 4, 31, 32, 33, 64, 85, 86, 255, 256, 257, 1000):
                need = all_of(c, many(n_seq, max_new, max_kv), heads * G)
                seen.add(need == one)
                assert need <= one, (max_new, max_kv, n_seq)
                assert all_of(c, many(n_seq, max_new, max(1, max_kv // 3)), heads * G) <= one
    assert seen == {True, False} if dtype == "e4m3" and G < 32 else seen == {True}      # over 8 bits there are batches that need none
