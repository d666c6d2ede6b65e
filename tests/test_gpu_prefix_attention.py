"""mpv_prefix_attention against the definition in 64 bits (needs an MI355X).

Outputs are held to the bound of tests/test_gpu_tree_attention.py: behind a prefix the sums are rescaled and added up once more per part,
which its 2 (n + 64) e covers.  The logarithm of the sum, with e = 2^-24, S the largest sum of absolute products of a key (scaled), n keys:
  a product's sum in float32                           (D + 1) e S
  the exponent's rounding and its exponential          2 (S + 4) e
  the sum over the keys, rescaled on the way           2 (n + 64) e
  reference + logarithm, turned into natural units     8 e (|lse| + S + 8)
"""

import numpy as np
import pytest
import torch

import paper_2602_16994_amd as mpv
from oracle import prefix_oracle as po
from tests.test_gpu_tree_attention import CHAIN3, DELAYED15, FULL64, HALF, TREE41, TREE7, TYPES

pytestmark = pytest.mark.gpu


class Case:
    def __init__(self, parent, H, KV, D, dtype, prefix_of, prefix_len, context, page, window=0, sinks=0, nodes=None, shapes=None, seed=1,
                 spread=False, scale=None, gain=1.0, width=None, prefix_width=None):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        N, B, G = len(parent), len(prefix_of), len(prefix_len)
        self.parent, self.window, self.sinks, self.dtype = parent, window, sinks, dtype
        self.scale = D ** -0.5 if scale is None else scale
        context = [context] * B if isinstance(context, int) else list(context)
        width = -(-max(context) // page) if width is None else width
        many = -(-max([0, *prefix_len]) // page) if prefix_width is None else prefix_width
        self.pages = B * width + G * many + 3

        def rand(*shape):
            return torch.randn(*shape, generator=gen, device="cuda")

        if spread:
            qkv = rand(B, N, H + 2 * KV, D).to(dtype)
            self.q, self.tk, self.tv = qkv[:, :, :H], qkv[:, :, H:H + KV], qkv[:, :, H + KV:]
            cache = rand(self.pages, 2, page, KV, D).to(dtype)
            self.ck, self.cv = cache[:, 0], cache[:, 1]
        else:
            self.q, self.tk, self.tv = rand(B, N, H, D).to(dtype), rand(B, N, KV, D).to(dtype), rand(B, N, KV, D).to(dtype)
            self.ck, self.cv = rand(self.pages, page, KV, D).to(dtype), rand(self.pages, page, KV, D).to(dtype)
        self.q *= gain
        order = torch.randperm(self.pages, generator=gen, device="cuda").to(torch.int32)
        self.table = order[:B * width].view(B, width)
        self.prefix_table = order[B * width:B * width + G * many].view(G, many)

        def whole(x):
            return None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")

        self.prefix_of, self.prefix_len, self.context = whole(prefix_of), whole(prefix_len), whole(context)
        self.nodes, self.shapes = whole(nodes), whole(shapes)

    def run(self, **kw):
        args = dict(window=self.window, sinks=self.sinks, num_nodes=self.nodes, tree_parent=self.shapes, scale=self.scale, lse=True)
        args.update(kw)
        return mpv.mpv_prefix_attention(self.parent, self.q, self.tk, self.tv, self.ck, self.cv, self.table, self.context, self.prefix_of,
                                        self.prefix_table, self.prefix_len, **args)

    def expected(self):
        B, N = self.q.shape[:2]
        f = [t.double().cpu().numpy() for t in (self.q, self.tk, self.tv, self.ck, self.cv)]
        parents = [self.parent] * B if self.shapes is None else self.shapes.tolist()
        nodes = [N] * B if self.nodes is None else self.nodes.tolist()
        return po.prefix_attention(*f, self.table.cpu().numpy(), self.context.tolist(), parents, nodes, self.prefix_of.tolist(),
                                   self.prefix_table.cpu().numpy(), self.prefix_len.tolist(), self.window, self.sinks, self.scale)

    def check(self, result=None):
        result = self.run() if result is None else result
        got = result.out.double().cpu().numpy()
        want, A, S, n, lse = self.expected()
        h, e, D = HALF[self.dtype], 2.0 ** -24, self.q.shape[3]
        if result.lse is not None:
            bound = ((D + 1) * S + 2 * (S + 4) + 2 * (n + 64) + 8 * (np.abs(lse) + S + 8)) * e
            real = ~np.isnan(lse)
            off = (np.abs(result.lse.double().cpu().numpy() - lse) / bound)[real]
            print("[lse: largest error over its bound] %.3f" % off.max(), flush=True)
            assert off.max() <= 1.0
        S, n = S[..., None], n[..., None]
        tol = h * np.abs(want) + (h + 2 * (D + 1) * e * S + 4 * (S + 4) * e + 2 * (n + 64) * e) * A
        if self.dtype == torch.float16:
            tol = tol + n * 2.0 ** -24 * max(float(t.double().abs().nan_to_num().max()) if t.numel() else 0.0 for t in (self.cv, self.tv))
        real = ~np.isnan(want)
        assert np.isfinite(got[real]).all()
        off = (np.abs(got - want) / (tol + 1e-300))[real]
        print("[largest error over its bound] %.3f" % off.max(), flush=True)
        assert off.max() <= 1.0
        return got


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("parent,H,KV,D,prefix_of,prefix_len,context,page", [
    ([-1], 1, 1, 8, [0], [1], 0, 16),
    ([-1], 4, 1, 64, [0, 0], [17], [1, 0], 1),
    ([-1], 8, 2, 128, [0, 0, 0, 0, 0], [700], [30, 0, 64, 1, 200], 16),
    (CHAIN3, 6, 2, 64, [0, 0, 1, 2, 2, 2], [64, 1, 129], [0, 63, 64, 5, 100, 1], 16),
    (TREE7, 8, 8, 80, [1, 1, -1, 0], [65, 300], [65, 3, 40, 12], 24),
    (DELAYED15, 8, 2, 128, [0, 0, 0, 5, -7, 1], [127, 0], [0, 1, 127, 129, 20, 50], 32),
    (DELAYED15, 16, 1, 96, [0, 0, 0], [511], [257, 8, 0], 7),
    (TREE41, 4, 2, 256, [0, 0], [200], [31, 70], 64),
    (FULL64, 8, 1, 128, [0, 0, 0, 0], [300], [130, 0, 1, 64], 128),
    ([-1], 64, 1, 40, [0, 0, 0], [333], [40, 2, 0], 16),
    (TREE7, 12, 4, 192, [0, 0], [900], [150, 20], 256),
    ([-1], 3, 3, 256, [0] * 7, [100], 9, 8),
])
def test_shapes(parent, H, KV, D, prefix_of, prefix_len, context, page, dtype):
    print("[case] prefix shapes", len(prefix_of), len(parent), H, KV, D, prefix_len, context, page, dtype, flush=True)
    Case(parent, H, KV, D, dtype, prefix_of, prefix_len, context, page, seed=len(parent) + page).check()


@pytest.mark.parametrize("B,parent,H,KV", [(64, [-1], 4, 1), (65, [-1], 2, 2), (130, CHAIN3, 2, 1), (70, DELAYED15, 8, 2), (20, TREE41, 8, 1)])
def test_many_trees_behind_one_prefix(B, parent, H, KV):
    """Runs of trees that cross a multiple of 64, several row blocks and several units a cache head."""
    print("[case] many trees", B, len(parent), H, KV, flush=True)
    Case(parent, H, KV, 64, torch.bfloat16, [0] * B, [150], [b % 40 for b in range(B)], 16, seed=B).check()


def test_a_long_prefix_that_many_teams_share():
    print("[case] long prefix", flush=True)
    Case([-1], 4, 1, 128, torch.bfloat16, [0, 0, 0], [20000], [5, 700, 0], 64, seed=3).check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H,KV,D", [(16, 2, 80), (5, 1, 128), (8, 2, 256), (4, 1, 256)])
def test_several_row_blocks_of_long_rows(H, KV, D, dtype):
    """Trees whose rows take several blocks: 328, 205, 164 rows a cache head."""
    print("[case] prefix row blocks", H, KV, D, dtype, flush=True)
    Case(TREE41, H, KV, D, dtype, [0, 0, 1], [140, 33], [100, 0, 37], 16, seed=D).check()


@pytest.mark.parametrize("order", [[0, 1, 0, 1, 2, 0], [2, 2, 1, 1, 0, 0], [-1, 0, -1, 0, 7, 0], [-1] * 6])
def test_any_order(order):
    print("[case] order", order, flush=True)
    Case(TREE7, 4, 2, 64, torch.float16, order, [90, 33, 128], [10, 0, 64, 5, 31, 2], 16, seed=len(set(order))).check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 3), (2, 1), (64, 4), (100, 0), (100, 70), (255, 17), (430, 390), (5000, 2)])
def test_window_and_sinks(window, sinks, dtype):
    print("[case] prefix window", window, sinks, dtype, flush=True)
    Case(mpv.delayed_tree(3, 2, 6), 4, 2, 64, dtype, [0, 0, 1, -1, 2], [400, 7, 300], [50, 0, 99, 20, 301], 16, window=window, sinks=sinks,
         seed=window).check()


@pytest.mark.parametrize("dtype", TYPES)
def test_trees_of_their_own_shapes_and_sizes(dtype):
    print("[case] prefix own shapes", dtype, flush=True)
    N, B = 9, 6
    rng = np.random.default_rng(4)
    shapes = [[-1] + [int(rng.integers(0, n)) for n in range(1, N)] for _ in range(B)]
    shapes[2][5] = 70                               # no node: a root of its own
    case = Case([-1] * N, 8, 2, 64, dtype, [0, 0, 0, 1, 1, 1], [50, 99], [5, 0, 70, 1, 12, 64], 16, window=40, sinks=2, nodes=[9, 0, 3, 1, 0, 7],
                shapes=shapes, seed=5)
    out = mpv.PrefixAttentionResult(out=torch.full_like(case.q, 7.0), lse=torch.full(case.q.shape[:3], 7.0, device="cuda"))
    case.check(case.run(out=out))
    for b, nodes in enumerate([9, 0, 3, 1, 0, 7]):
        assert (out.out[b, nodes:] == 7.0).all() and (out.lse[b, nodes:] == 7.0).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_slices_of_a_projection_and_interleaved_caches(dtype):
    print("[case] prefix strides", dtype, flush=True)
    Case(DELAYED15, 8, 2, 128, dtype, [0, 0, 1], [100, 31], [100, 33, 260], 16, seed=11, spread=True).check()


@pytest.mark.parametrize("scale", [0.0, -0.1, 0.5])
def test_scales(scale):
    print("[case] prefix scale", scale, flush=True)
    Case(CHAIN3, 4, 2, 64, torch.bfloat16, [0, 0], [77], [9, 30], 16, scale=scale, seed=12).check()


def test_large_products():
    """Scores of several hundred: references move, and the part without the largest key vanishes."""
    print("[case] prefix large products", flush=True)
    Case(CHAIN3, 4, 2, 64, torch.float32, [0, 0], [77], [90, 30], 16, gain=40.0, seed=13).check()


@pytest.mark.parametrize("dtype", TYPES)
def test_pages_that_are_none_and_lengths_that_do_not_fit(dtype):
    print("[case] prefix bad pages", dtype, flush=True)
    case = Case(CHAIN3, 4, 2, 64, dtype, [0, 0, 1], [100, 50], [40, 64, 20], 16, seed=14)
    case.prefix_table[0, 2] = -1
    case.prefix_table[0, 4] = case.pages
    case.table[1, 1] = 1 << 30
    case.prefix_len[0] = 5000
    case.prefix_len[1] = -3
    case.context[2] = -1
    case.check()


@pytest.mark.parametrize("dtype", TYPES)
def test_no_pages_at_all(dtype):
    """A prefix of which nothing is there gives nothing: its rows' states are empty."""
    print("[case] prefix without pages", dtype, flush=True)
    case = Case(CHAIN3, 4, 2, 64, dtype, [0, 0], [100], [40, 0], 16, seed=15)
    case.prefix_table.fill_(-1)
    case.check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
def test_what_is_not_seen_does_not_reach_an_output(value, dtype):
    print("[case] prefix unseen", value, dtype, flush=True)
    case = Case(CHAIN3, 4, 2, 64, dtype, [0, 0, 1, 1], [100, 70], [40, 3, 17, 90], 16, window=60, sinks=2, seed=16)
    # behind the lengths, and between the sinks and the windows of all trees
    for p, n in ((0, 100), (1, 70)):
        last = int(case.prefix_table[p, n // 16])
        case.ck[last, n % 16:] = value
        case.cv[last, n % 16:] = value
    case.cv[int(case.prefix_table[0, 0]), 3:16] = value      # positions 3 to 15: the first window begins at 100 + 3 + 1 - 60
    case.ck[int(case.prefix_table[0, 0]), 3:16] = value
    case.check()


@pytest.mark.parametrize("dtype", TYPES)
def test_what_only_some_trees_see(dtype):
    """A value that is no number, in the window of the tree with the short context alone."""
    print("[case] prefix seen by some", dtype, flush=True)
    case = Case([-1], 4, 2, 64, dtype, [0, 0], [100], [0, 60], 16, window=50, sinks=0, seed=17)
    at = 60                                        # tree 0 sees positions 51 to 100, tree 1 those from 111 on
    case.cv[int(case.prefix_table[0, at // 16]), at % 16, 1, 5] = float("inf")
    got = case.run()
    out = got.out.double().cpu().numpy()
    assert np.isinf(out[0, 0, 2:, 5]).all() and np.isfinite(out[0, 0, :2]).all() and np.isfinite(out[1]).all()
    case.cv[int(case.prefix_table[0, at // 16]), at % 16, 1, 5] = 0.0
    want = case.expected()[0]
    assert np.allclose(out[1], want[1], atol=0.05) and np.allclose(out[0, 0, :2], want[0, 0, :2], atol=0.05)


def test_without_prefixes_it_is_tree_attention_with_lse():
    print("[case] no prefixes", flush=True)
    case = Case(TREE7, 8, 2, 128, torch.bfloat16, [-1, -1], [1], [100, 7], 16, seed=18)
    want = case.run()
    got = mpv.mpv_prefix_attention(case.parent, case.q, case.tk, case.tv, case.ck, case.cv, case.table, case.context, lse=True)
    plain = mpv.mpv_tree_attention(case.parent, case.q, case.tk, case.tv, case.ck, case.cv, case.table, case.context)
    assert torch.equal(got.out, want.out) and torch.equal(got.lse, want.lse)
    assert (got.out.float() - plain.out.float()).abs().max() <= 2 * HALF[torch.bfloat16] * plain.out.float().abs().max()
    case.check(got)
    assert case.run(lse=False).lse is None


def test_an_empty_batch_and_an_empty_list():
    print("[case] prefix empty", flush=True)
    case = Case(TREE7, 8, 2, 64, torch.bfloat16, [], [5], [], 16, seed=19, width=1)
    assert case.run().out.shape == (0, 7, 8, 64)
    case = Case(TREE7, 8, 2, 64, torch.bfloat16, [0, 0], [], [4, 9], 16, seed=20, prefix_width=2)
    case.check()


def test_outputs_repeat():
    print("[case] prefix repeat", flush=True)
    case = Case(TREE7, 8, 2, 128, torch.bfloat16, [0] * 40, [3000], [b * 7 for b in range(40)], 16, seed=21)
    first = case.run()
    for _ in range(3):
        again = case.run()
        assert torch.equal(first.out, again.out) and torch.equal(first.lse, again.lse)
