"""The pick of a wavefront hands keys from lane to lane through LDS: a fence stands behind the keys' first pass and behind the keys that it ranks."""
from tests.test_lds_fences import wavefront_fences


def test_pick_fences_its_hand_overs():
    found = {f: n for f, n in wavefront_fences("kv_select.hip").items() if "sel_fused_kernel" in f}
    assert found and all(n >= 2 for n in found.values()), found
