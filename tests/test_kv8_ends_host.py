"""CPU-only checks beside tests/test_gpu_kv8_ends.py."""
import glob
import os
import re

from tests.conftest import ROOT

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
