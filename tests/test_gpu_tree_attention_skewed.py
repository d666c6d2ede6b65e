"""mpv_tree_attention on batches in which one context is much longer than the others, so that its units have many parts although there are
more units than teams of workgroups (needs an MI355X).  Tolerance: that of test_gpu_tree_attention.py."""

import numpy as np
import pytest
import torch

from paper_2602_16994_amd import TreeAttentionResult
from tests.test_gpu_tree_attention import CHAIN3, DELAYED15, TYPES, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,parent,H,KV,D", [(300, CHAIN3, 4, 2, 32), (300, DELAYED15, 8, 2, 32), (130, [-1], 12, 6, 128), (150, CHAIN3, 8, 4, 136)])
def test_one_long_context_among_many_short_ones(B, parent, H, KV, D, dtype):
    print("[case] skewed", B, len(parent), H, KV, D, dtype, flush=True)
    rng = np.random.default_rng(B + D)
    context = rng.integers(0, 20, B).tolist()
    context[B // 3] = 9000
    nodes = rng.integers(0, len(parent) + 1, B).tolist()
    nodes[B // 3] = len(parent)
    case = Case(B, parent, H, KV, D, dtype, [16] * B, 16, nodes=nodes, seed=B)
    # (a block table as wide as the longest context needs; the others' rows are not read that far)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(B)
    pages = 9000 // 16 + 1
    cache = [torch.cat([t, torch.randn(pages, 16, KV, D, generator=gen, device="cuda").to(dtype)]) for t in (case.ck, case.cv)]
    table = torch.full((B, pages), -1, dtype=torch.int32, device="cuda")
    table[:, :1] = case.table
    table[:, 1] = case.table[:, 0].flip(0)
    table[B // 3] = case.pages + torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    case.ck, case.cv, case.table, case.pages = *cache, table, case.pages + pages
    case.context = torch.tensor(context, dtype=torch.int32, device="cuda")
    case.out = TreeAttentionResult(out=torch.full_like(case.q, 7.0))
    got = case.check(case.run(out=case.out).out)
    for b, n in enumerate(nodes):
        assert (got[b, n:] == 7.0).all()
