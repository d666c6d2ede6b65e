"""Numbers that do not fit the 32 bits in which the library takes them (no GPU needed: they are refused before anything else)."""

import pytest
import torch

import paper_2602_16994_amd as mpv

I = torch.zeros(2, dtype=torch.int32)


def attention(parent=(-1, 0, 0), **kw):
    q, k, c = torch.zeros(2, 3, 4, 64), torch.zeros(2, 3, 2, 64), torch.zeros(8, 16, 2, 64)
    return mpv.mpv_tree_attention(list(parent), q, k, k, c, c, torch.zeros(2, 4, dtype=torch.int32), I, **kw)


@pytest.mark.parametrize("number", [2 ** 31, 2 ** 32 + 8, -2 ** 31 - 1, 2 ** 63])
def test_attention(number):
    for name in ("window", "sinks"):
        with pytest.raises(ValueError, match=f"{name} must fit 32 bits"):
            attention(**{name: number})
    with pytest.raises(ValueError, match=r"parent\[2\] must fit 32 bits"):
        attention(parent=(-1, 0, number))


@pytest.mark.parametrize("number", [2 ** 31, 2 ** 32 + 8])
def test_chains_and_tables(number):
    with pytest.raises(ValueError, match="max_depth must fit 32 bits"):
        mpv.mpv_verify_chains(torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, 3, 9), None, torch.zeros(2, 3), max_depth=number)
    for name in ("page_size", "extra"):
        with pytest.raises(ValueError, match=f"{name} must fit 32 bits"):
            mpv.mpv_extend_tables(torch.zeros(2, 4, dtype=torch.int32), I, I, torch.zeros(8, dtype=torch.int32), I[:1],
                                  slot_map=torch.zeros(2, 3, dtype=torch.int64), **{"page_size": 16, "extra": 0, name: number})
