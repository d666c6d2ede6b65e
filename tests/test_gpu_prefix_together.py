"""mpv_prefix_attention where prefixes are read for all trees together (needs an MI355X).  That goes by the room that the prefixes have, so
short ones in a wide table take that path, too.  Definition and bounds: tests/test_gpu_prefix_attention.py."""

import numpy as np
import pytest
import torch

import paper_2602_16994_amd as mpv
from paper_2602_16994_amd import binding as bd
from tests.test_gpu_prefix_attention import Case as Plain
from tests.test_gpu_tree_attention import CHAIN3, DELAYED15, TREE7, TYPES

pytestmark = pytest.mark.gpu
ROOM = 1 << 26                                     # positions that a prefix has room for


class Case(Plain):
    def __init__(self, parent, H, KV, D, dtype, prefix_of, prefix_len, context, page, **kw):
        super().__init__(parent, H, KV, D, dtype, prefix_of, prefix_len, context, page, **kw)
        wide = torch.full((len(prefix_len), ROOM // page), -1, dtype=torch.int32, device="cuda")
        wide[:, :self.prefix_table.shape[1]] = self.prefix_table
        self.prefix_table = wide

    def expected(self):                            # (the definition reads as many pages as there are)
        wide, self.prefix_table = self.prefix_table, self.prefix_table[:, :4096]
        want = super().expected()
        self.prefix_table = wide
        return want

    def check(self, result=None):
        assert reads_together(self)
        return super().check(result)


def reads_together(case):
    """The workspace holds the rows' states then.  (Of batches that fill the card: otherwise its size depends on the room in the tables.)"""
    args = (case.parent, case.q, case.tk, case.tv, case.ck, case.cv, case.table, case.context, case.scale, case.window, case.sinks, case.nodes,
            case.shapes)
    return bd._prefixed_plan(*args, case.prefix_of, case.prefix_table, case.prefix_len, None).need != \
        bd._prefixed_plan(*args, case.prefix_of, case.prefix_table[:, :1].contiguous(), case.prefix_len, None).need


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("parent,H,KV,D,prefix_of,prefix_len,context,page", [
    ([-1], 4, 1, 64, [0, 0], [17], [1, 0], 1),
    ([-1], 8, 2, 128, [0, 0, 0, 0, 0], [700], [30, 0, 64, 1, 200], 16),
    (CHAIN3, 6, 2, 64, [0, 0, 1, 2, 2, 2], [64, 1, 129], [0, 63, 64, 5, 100, 1], 16),
    (TREE7, 8, 8, 80, [1, 1, -1, 0], [65, 300], [65, 3, 40, 12], 24),
    (DELAYED15, 4, 2, 128, [0, 0, 0, 5, -7, 1], [127, 0], [0, 1, 127, 129, 20, 50], 32),
    ([-1], 32, 1, 40, [0, 0, 0], [333], [40, 2, 0], 16),
    (TREE7, 12, 4, 192, [0, 0], [900], [150, 20], 256),
    ([-1], 3, 3, 256, [0] * 7, [100], 9, 8),
    (TREE7, 4, 2, 256, [0] * 9, [70], 20, 16),
])
def test_shapes(parent, H, KV, D, prefix_of, prefix_len, context, page, dtype):
    print("[case] together: shapes", len(prefix_of), len(parent), H, KV, D, prefix_len, context, page, dtype, flush=True)
    Case(parent, H, KV, D, dtype, prefix_of, prefix_len, context, page, seed=len(parent) + page).check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,parent,H,KV,D", [(130, [-1, 0, 0, 1, 2], 32, 8, 64), (200, [-1, 0, 0, 1, 2], 32, 8, 40), (110, CHAIN3, 64, 16, 136),
                                             (65, [-1], 2, 2, 128), (130, CHAIN3, 2, 1, 64), (70, DELAYED15, 4, 2, 64)])
def test_every_size_of_the_blocks(B, parent, H, KV, D, dtype):
    """Blocks of 16 to 192 rows; trees that cross a multiple of 64, and units of several blocks."""
    print("[case] together: blocks", B, len(parent), H, KV, D, dtype, flush=True)
    Case(parent, H, KV, D, dtype, [0] * B, [50], [b % 7 for b in range(B)], 16, seed=B).check()


@pytest.mark.parametrize("dtype", TYPES)
def test_a_long_prefix_that_many_workgroups_share(dtype):
    print("[case] together: long prefix", dtype, flush=True)
    Case([-1], 4, 1, 128, dtype, [0, 0, 0, -1, 1], [20000, 5000], [5, 700, 0, 3, 9], 64, seed=3).check()


@pytest.mark.parametrize("order", [[0, 1, 0, 1, 2, 0], [2, 2, 1, 1, 0, 0], [-1, 0, -1, 0, 7, 0], [-1] * 6])
def test_any_order(order):
    print("[case] together: order", order, flush=True)
    Case(TREE7, 4, 2, 64, torch.float16, order, [90, 33, 128], [10, 0, 64, 5, 31, 2], 16, seed=len(set(order))).check()


@pytest.mark.parametrize("dtype", TYPES)
def test_many_prefixes(dtype):
    """Every tree has its own, and some share: as many units as trees, in every chunk of 64."""
    print("[case] together: many prefixes", dtype, flush=True)
    B = 150
    case = Case([-1], 4, 2, 64, dtype, [b if b % 5 else -1 for b in range(B)], [b % 40 for b in range(B)], [b % 9 for b in range(B)], 256, seed=7)
    case.check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sinks", [0, 5, 7000])
def test_windows(sinks, dtype):
    """Windows that end inside a prefix, for some trees behind its first tile and for some before."""
    print("[case] together: window", sinks, dtype, flush=True)
    B = 60
    case = Case(CHAIN3, 2, 1, 64, dtype, [0] * 20 + [1] * 20 + [2] * 20, [16100, 16500, 40], [b * 9 for b in range(B)], 16, window=16300, sinks=sinks, seed=8)
    case.check()


@pytest.mark.parametrize("dtype", TYPES)
def test_windows_that_leave_nothing_of_a_prefix(dtype):
    print("[case] together: window past the prefix", dtype, flush=True)
    case = Case([-1], 2, 1, 64, dtype, [0] * 60, [30], [16400] * 3 + [b for b in range(57)], 64, window=16300, sinks=0, seed=9)
    case.check()


@pytest.mark.parametrize("dtype", TYPES)
def test_trees_of_their_own_shapes_and_sizes(dtype):
    print("[case] together: own shapes", dtype, flush=True)
    N, B = 9, 6
    rng = np.random.default_rng(4)
    shapes = [[-1] + [int(rng.integers(0, n)) for n in range(1, N)] for _ in range(B)]
    nodes = [9, 0, 3, 1, 0, 7]
    case = Case([-1] * N, 8, 2, 64, dtype, [0, 0, 0, 1, 1, 1], [50, 99], [5, 0, 70, 1, 12, 64], 16, nodes=nodes, shapes=shapes, seed=5)
    out = mpv.PrefixAttentionResult(out=torch.full_like(case.q, 7.0), lse=torch.full(case.q.shape[:3], 7.0, device="cuda"))
    case.check(case.run(out=out))
    for b, n in enumerate(nodes):
        assert (out.out[b, n:] == 7.0).all() and (out.lse[b, n:] == 7.0).all()
    case.nodes = torch.zeros(B, dtype=torch.int32, device="cuda")
    out.out.fill_(7.0)
    case.run(out=out)
    assert (out.out == 7.0).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_slices_of_a_projection_and_interleaved_caches(dtype):
    print("[case] together: strides", dtype, flush=True)
    Case(TREE7, 8, 2, 128, dtype, [0, 0, 1], [100, 31], [100, 33, 260], 16, seed=11, spread=True).check()


@pytest.mark.parametrize("scale,gain", [(0.0, 1.0), (-0.1, 1.0), (0.5, 1.0), (0.125, 40.0)])
def test_scales(scale, gain):
    print("[case] together: scale", scale, gain, flush=True)
    Case(CHAIN3, 4, 2, 64, torch.bfloat16 if gain == 1.0 else torch.float32, [0, 0], [77], [9, 30], 16, scale=scale, gain=gain, seed=12).check()


@pytest.mark.parametrize("dtype", TYPES)
def test_pages_that_are_none(dtype):
    print("[case] together: bad pages", dtype, flush=True)
    case = Case(CHAIN3, 4, 2, 64, dtype, [0, 0, 1], [100, 50], [40, 64, 20], 16, seed=14)
    case.prefix_table[0, 2] = -1
    case.prefix_table[0, 4] = case.pages
    case.prefix_len[1] = -3
    case.check()
    case.prefix_table.fill_(-1)                    # nothing of the prefix is there: its rows' states are empty
    case.check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
def test_what_is_not_seen_does_not_reach_an_output(value, dtype):
    print("[case] together: unseen", value, dtype, flush=True)
    B = 60
    case = Case(CHAIN3, 2, 1, 64, dtype, [0] * B, [16350], [b for b in range(B)], 16, window=16300, sinks=2, seed=16)
    last = int(case.prefix_table[0, 16350 // 16])
    case.ck[last, 16350 % 16:] = value
    case.cv[last, 16350 % 16:] = value
    first = int(case.prefix_table[0, 0])           # positions 3 to 15: the first window begins at 16350 + 0 + 1 - 16300
    case.cv[first, 3:] = value
    case.ck[first, 3:] = value
    case.check()
    # in the windows of the first trees alone: position 60 is seen by nodes at 16359 and before
    page = int(case.prefix_table[0, 60 // 16])
    case.cv[page, 60 % 16, 0, 5] = value
    out = case.run().out.double().cpu().numpy()
    for b in range(B):
        for n, depth in enumerate((0, 1, 2)):
            assert np.isfinite(out[b, n, :, :5]).all() and np.isfinite(out[b, n, :, 6:]).all()
            assert np.isfinite(out[b, n, :, 5]).all() == (16350 + b + depth - 16300 + 1 > 60), (b, n)


def test_outputs_repeat():
    print("[case] together: repeat", flush=True)
    case = Case(TREE7, 8, 2, 128, torch.bfloat16, [0] * 40, [3000], [b * 7 for b in range(40)], 16, seed=21)
    first = case.run()
    for _ in range(3):
        again = case.run()
        assert torch.equal(first.out, again.out) and torch.equal(first.lse, again.lse)
    assert case.run(lse=False).lse is None
