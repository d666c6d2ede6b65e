"""Sizes that mpv_evict_positions refuses because its kernels count in 32 bits (no GPU)."""

import ctypes

import pytest

import paper_2602_16994_amd as mpv
from paper_2602_16994_amd import binding as bd
from tests.test_abi_cpu import code

MOST = 2 ** 31 - 1 - (1 << 16)                     # positions, kept or in a table


def need_of(**over):
    f = dict(layers=1, B=1, kv_heads=1, score_heads=1, head_dim=8, dtype=1, num_pages=4, page_size=16, table_width=4, budget=20, trigger=30, sinks=2, recent=4,
             score_width=64, cache_layer_stride=512, page_stride=128, slot_stride=8)
    need = ctypes.c_size_t()
    return mpv.load_library().mpv_evict_positions_workspace_bytes(ctypes.byref(bd._Eviction(**{**f, **over})), ctypes.byref(need))


@pytest.mark.parametrize("sizes,fine", [
    (dict(budget=MOST, trigger=2 ** 31 - 1), True), (dict(budget=MOST + 1, trigger=2 ** 31 - 1), False), (dict(budget=2 ** 31 - 1, trigger=2 ** 31 - 1), False),
    (dict(trigger=2 ** 31 - 1), True),
    (dict(page_size=1, table_width=MOST, score_width=MOST), True), (dict(page_size=1, table_width=MOST + 1, score_width=MOST + 1), False),
    (dict(num_pages=1, page_size=MOST, table_width=1, score_width=MOST), True), (dict(num_pages=1, page_size=2 ** 31 - 1, table_width=1, score_width=2 ** 31 - 1), False),
])
def test_loops_over_positions_do_not_pass_32_bits(sizes, fine):
    """They go on in steps of some thousands beyond the last position."""
    assert need_of(**sizes) == (0 if fine else code("MPV_ERR_UNSUPPORTED"))
