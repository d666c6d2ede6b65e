"""Batches of no trees (needs an MI355X)."""

import pytest
import torch

import paper_2602_16994_amd as mpv

pytestmark = pytest.mark.gpu

PARENT = mpv.delayed_tree(3, 1, 2)


def test_counters_of_no_trees():
    print("[case] no trees", flush=True)
    N, V = len(PARENT), 50
    z = torch.randn(0, N, V, device="cuda")
    tokens, u = torch.zeros(0, N, dtype=torch.int32, device="cuda"), torch.zeros(0, N, device="cuda")
    one = torch.randn(1, N, V, device="cuda")
    old = mpv.mpv_verify(PARENT, torch.zeros(1, N, dtype=torch.int32, device="cuda"), one, one, 1.0, torch.zeros(1, N, device="cuda"),
                         mpv.MPV_METHOD_TRAVERSAL)
    old.counters.fill_(7)
    res = mpv.mpv_verify(PARENT, tokens, z, z, 1.0, u, mpv.MPV_METHOD_TRAVERSAL, out=old)
    res.raise_on_timeout()
    assert res.counters.tolist() == [0] * 8
    pieces = [torch.full((8,), 7, dtype=torch.int32, device="cuda") for _ in range(50)]
    del pieces
    res = mpv.mpv_block_efficiency(PARENT, tokens, z, z, 1.0, mpv.MPV_METHOD_SPECINFER)
    res.raise_on_timeout()
    assert res.counters.tolist() == [0] * 8 and res.expected.numel() == 0
    pieces = [torch.full((8,), 7, dtype=torch.int32, device="cuda") for _ in range(50)]
    del pieces
    alpha, counters = mpv.mpv_acceptance_rates(PARENT, z, z, 1.0, mpv.MPV_METHOD_SPECINFER)
    assert counters.tolist() == [0] * 8 and alpha.numel() == 0
