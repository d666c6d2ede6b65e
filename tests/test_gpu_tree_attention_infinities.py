"""Infinite values whose weight vanishes, in tiles that all nodes of a tree see alike and in others (needs an MI355X): that column of every
node that sees them is no finite number, everything else is as it was."""

import pytest
import torch

from tests.test_gpu_tree_attention import TREE7, TYPES, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("where", ["context", "window's edge", "tree"])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_an_infinite_value_without_weight(sign, where, dtype):
    print("[case] infinite without weight", sign, where, dtype, flush=True)
    L = 300
    case = Case(1, TREE7, 4, 2, 64, dtype, [L], 16, seed=31, window=200 if where == "window's edge" else 0, scale=1.0)
    case.q[:] = 0.0
    case.q[..., 0] = 30.0
    for k in (case.ck, case.tk):
        k[..., 0] = 0.0
    at = L - 199 if where == "window's edge" else 40          # (the root sees the edge, its children do not)
    key, value = (case.tk[0, 1], case.tv[0, 1]) if where == "tree" else [t[case.table[0, at // 16], at % 16] for t in (case.ck, case.cv)]
    key[:, 0] = -200.0                             # a product of -6000: its weight is 0 in any type
    clean = case.run().out.clone()
    assert torch.isfinite(clean).all()
    value[1, 9] = sign * float("inf")              # cache head 1, query heads 2 and 3
    got = case.run().out
    nodes = {"context": range(7), "window's edge": [0], "tree": [1, 2, 3]}[where]
    spoiled = torch.zeros_like(got, dtype=torch.bool)
    for n in nodes:
        spoiled[0, n, 2:, 9] = True
    assert not torch.isfinite(got[spoiled]).any()
    assert torch.equal(got[~spoiled], clean[~spoiled])
