"""mpv_tree_attention against the definition in 64 bits (needs an MI355X).

Tolerance, per element, with h half a step of the type (bf16 2^-8, f16 2^-11, f32 2^-24), e = 2^-24, A = sum of the weights times
the absolute values, S = the largest sum of absolute products of a key (scaled) and n keys seen:
  the output's rounding                                h |out|
  a weight's rounding to the type                      h A       (f16: and 2^-24 a weight below its smallest normal number, n 2^-24 max|v|
                                                                  against a sum of weights of at least 1)
  a product's sum in float32, in any order             (D + 1) e S, as an exponent in the weight and in the sum of weights: 2 (D + 1) e S A
  the exponent's own rounding and its exponential      2 (S + 4) 2 e A
  sums over the keys, rescaled on the way              2 (n + 64) e A
"""

import numpy as np
import pytest
import torch

import paper_2602_16994_amd as mpv
from oracle import serving_oracle as so

pytestmark = pytest.mark.gpu

HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TYPES = [torch.bfloat16, torch.float16, torch.float32]


class Case:
    def __init__(self, B, parent, H, KV, D, dtype, context, page, window=0, sinks=0, nodes=None, shapes=None, seed=1, spread=False,
                 spare=0, scale=None, gain=1.0):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        N = len(parent)
        self.parent, self.window, self.sinks, self.dtype = parent, window, sinks, dtype
        self.scale = D ** -0.5 if scale is None else scale
        context = [context] * B if isinstance(context, int) else list(context)
        width = max(1, -(-max(context) // page)) + spare
        self.pages = B * width + 3

        def rand(*shape):
            return torch.randn(*shape, generator=gen, device="cuda")

        # spread: nodes are slices of one projection's output, keys and values of a slot lie in one tensor
        if spread:
            qkv = rand(B, N, H + 2 * KV, D).to(dtype)
            self.q, self.tk, self.tv = qkv[:, :, :H], qkv[:, :, H:H + KV], qkv[:, :, H + KV:]
            cache = rand(self.pages, 2, page, KV, D).to(dtype)
            self.ck, self.cv = cache[:, 0], cache[:, 1]
        else:
            self.q, self.tk, self.tv = rand(B, N, H, D).to(dtype), rand(B, N, KV, D).to(dtype), rand(B, N, KV, D).to(dtype)
            self.ck, self.cv = rand(self.pages, page, KV, D).to(dtype), rand(self.pages, page, KV, D).to(dtype)
        self.q *= gain
        self.table = torch.randperm(self.pages, generator=gen, device="cuda")[:B * width].view(B, width).to(torch.int32)
        self.context = torch.tensor(context, dtype=torch.int32, device="cuda")
        self.nodes = None if nodes is None else torch.tensor(nodes, dtype=torch.int32, device="cuda")
        self.shapes = None if shapes is None else torch.tensor(shapes, dtype=torch.int32, device="cuda")
        self.out = None

    def run(self, **kw):
        args = dict(window=self.window, sinks=self.sinks, num_nodes=self.nodes, tree_parent=self.shapes, scale=self.scale)
        args.update(kw)
        return mpv.mpv_tree_attention(self.parent, self.q, self.tk, self.tv, self.ck, self.cv, self.table, self.context, **args)

    def expected(self):
        B, N = self.q.shape[:2]
        f = [t.double().cpu().numpy() for t in (self.q, self.tk, self.tv, self.ck, self.cv)]
        parents = [self.parent] * B if self.shapes is None else self.shapes.tolist()
        nodes = [N] * B if self.nodes is None else self.nodes.tolist()
        return so.tree_attention(*f, self.table.cpu().numpy(), self.context.tolist(), parents, nodes, self.window, self.sinks, self.scale)

    def check(self, out=None):
        got = (self.run().out if out is None else out).double().cpu().numpy()
        want, A, S, n = self.expected()
        h, e, D = HALF[self.dtype], 2.0 ** -24, self.q.shape[3]
        S, n = S[..., None], n[..., None]
        tol = h * np.abs(want) + (h + 2 * (D + 1) * e * S + 4 * (S + 4) * e + 2 * (n + 64) * e) * A
        if self.dtype == torch.float16:
            tol = tol + n * 2.0 ** -24 * max(float(self.cv.double().abs().nan_to_num().max()) if self.cv.numel() else 0.0,
                                             float(self.tv.double().abs().nan_to_num().max()))
        real = ~np.isnan(want)
        assert np.isfinite(got[real]).all()
        off = (np.abs(got - want) / (tol + 1e-300))[real]
        print("[largest error over its bound] %.3f" % off.max(), flush=True)
        assert off.max() <= 1.0
        return got


CHAIN3 = [-1, 0, 1]
TREE7 = mpv.root_tree(2, 3)
DELAYED15 = mpv.delayed_tree(4, 2, 3)
TREE41 = mpv.root_tree(8, 5)
FULL64 = mpv.delayed_tree(9, 0, 7)
DEEP64 = list(range(-1, 63))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,parent,H,KV,D,context,page", [
    (1, [-1], 1, 1, 8, 0, 16),
    (1, [-1], 4, 1, 64, 1, 1),
    (2, [-1], 8, 2, 128, [1000, 37], 16),
    (3, CHAIN3, 6, 2, 64, [0, 63, 64], 16),
    (2, TREE7, 8, 8, 80, [65, 300], 24),
    (4, DELAYED15, 8, 2, 128, [0, 1, 127, 129], 32),
    (2, DELAYED15, 16, 1, 96, [511, 257], 7),
    (2, TREE41, 4, 2, 256, [200, 31], 64),
    (1, FULL64, 8, 1, 128, [130], 128),
    (2, DEEP64, 3, 3, 72, [5, 95], 5),
    (1, TREE7, 12, 4, 192, [1500], 256),
    (1, [-1], 64, 1, 40, [333], 16),
])
def test_shapes(B, parent, H, KV, D, context, page, dtype):
    print("[case] shapes", B, len(parent), H, KV, D, context, page, dtype, flush=True)
    Case(B, parent, H, KV, D, dtype, context, page, seed=B + len(parent)).check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 3), (2, 1), (5, 0), (64, 4), (100, 0), (100, 70), (255, 17), (5000, 2)])
def test_window_and_sinks(window, sinks, dtype):
    print("[case] window", window, sinks, dtype, flush=True)
    Case(3, mpv.delayed_tree(3, 2, 6), 4, 2, 64, dtype, [400, 0, 99], 16, window=window, sinks=sinks, seed=window).check()


@pytest.mark.parametrize("dtype", TYPES)
def test_a_window_over_a_long_context(dtype):
    print("[case] long window", dtype, flush=True)
    Case(1, [-1, 0, 0], 4, 1, 64, dtype, [20000], 16, window=700, sinks=4, seed=9).check()


@pytest.mark.parametrize("dtype", TYPES)
def test_long_and_short_contexts_in_one_batch(dtype):
    print("[case] ragged", dtype, flush=True)
    Case(6, TREE7, 8, 2, 64, dtype, [5000, 0, 3, 64, 700, 1], 16, seed=10).check()


@pytest.mark.parametrize("dtype", TYPES)
def test_slices_of_a_projection_and_interleaved_caches(dtype):
    print("[case] strides", dtype, flush=True)
    Case(3, DELAYED15, 8, 2, 128, dtype, [100, 33, 260], 16, seed=11, spread=True).check()


@pytest.mark.parametrize("dtype", TYPES)
def test_trees_of_their_own_shapes_and_sizes(dtype):
    print("[case] own shapes", dtype, flush=True)
    rng = np.random.default_rng(4)
    shapes = [[-1] + [int(rng.integers(0, n)) for n in range(1, 20)] for _ in range(5)]
    shapes[1][7] = 7                              # a parent that cannot be: a root of its own
    shapes[2][3] = -5
    case = Case(5, list(range(-1, 19)), 4, 2, 64, dtype, [70, 0, 1, 200, 64], 16, nodes=[20, 13, 7, 1, 0], shapes=shapes, seed=12, window=50, sinks=2)
    case.out = mpv.TreeAttentionResult(out=torch.full_like(case.q, 7.0))
    got = case.check(case.run(out=case.out).out)
    for b, n in enumerate([20, 13, 7, 1, 0]):
        assert (got[b, n:] == 7.0).all()          # rows behind a tree's last node


@pytest.mark.parametrize("dtype", TYPES)
def test_large_products_and_a_dominant_key(dtype):
    print("[case] large products", dtype, flush=True)
    Case(2, TREE7, 4, 2, 64, dtype, [300, 140], 16, seed=13, gain=30.0).check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("fill", [float("nan"), float("inf"), -float("inf"), "lowest"])
def test_what_is_not_seen_does_not_count(dtype, fill):
    """Slots behind the context, unused pages, slots between the sinks and the window, nodes behind a tree's last: whatever they hold."""
    print("[case] not seen", dtype, fill, flush=True)
    fill = torch.finfo(dtype).min if fill == "lowest" else fill
    case = Case(3, TREE7, 4, 2, 64, dtype, [201, 30, 0], 16, nodes=[7, 4, 2], seed=14, window=20, sinks=3, spare=2)
    clean = case.check()
    used = torch.zeros(case.pages, 16, dtype=torch.bool, device="cuda")
    for b, L in enumerate([201, 30, 0]):
        for j in range(L):
            if j < 3 or j > L - 20:
                used[case.table[b, j // 16], j % 16] = True
    for t in (case.ck, case.cv):
        t[~used] = fill
    for b, n in enumerate([7, 4, 2]):
        case.tk[b, n:] = fill
        case.tv[b, n:] = fill
        case.q[b, n:] = fill
    got = case.run().out.double().cpu().numpy()
    for b, n in enumerate([7, 4, 2]):
        assert np.array_equal(got[b, :n], clean[b, :n])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("fill", [float("nan"), float("inf")])
def test_what_another_node_sees_does_not_count(dtype, fill):
    """A sibling's keys and values, and a cached position at the window's edge that the root sees and its children do not."""
    print("[case] not seen by this node", dtype, fill, flush=True)
    case = Case(1, TREE7, 4, 2, 64, dtype, [90], 16, seed=15, window=20, sinks=0)
    clean = case.run().out.clone()
    case.tv[0, 3] = fill                          # seen by node 3 alone
    case.tk[0, 6] = fill                          # seen by node 6 alone
    edge = 90 - 19                                # the root's first position in the cache
    case.cv[case.table[0, edge // 16], edge % 16, :, 5] = fill
    got = case.run().out
    for n in (1, 2, 4, 5):
        assert torch.equal(got[0, n], clean[0, n]), n
    assert not torch.isfinite(got[0, 3]).any()
    assert torch.isnan(got[0, 6]).all()
    column = torch.arange(64, device="cuda") == 5
    assert not torch.isfinite(got[0, 0][:, column]).any() and torch.equal(got[0, 0][:, ~column], clean[0, 0][:, ~column])


@pytest.mark.parametrize("dtype", TYPES)
def test_pages_out_of_range_are_not_seen(dtype):
    print("[case] bad pages", dtype, flush=True)
    case = Case(3, CHAIN3, 4, 2, 64, dtype, [200, 70, 64], 16, seed=16)
    case.table[0, 3] = -1
    case.table[0, 5] = case.pages
    case.table[1, 0] = 2 ** 31 - 1
    case.table[2, :] = -7                         # nothing of the context is left
    case.check()


def test_lengths_out_of_range():
    print("[case] lengths", flush=True)
    case = Case(3, CHAIN3, 4, 2, 64, torch.bfloat16, [200, 70, 64], 16, seed=17)
    case.context[:] = torch.tensor([10 ** 9, -5, 64], device="cuda")     # more than the block table holds: all of it; less than nothing
    case.nodes = torch.tensor([99, 3, -1], dtype=torch.int32, device="cuda")
    case.check()


def test_no_cache_at_all():
    print("[case] no cache", flush=True)
    case = Case(2, TREE7, 4, 2, 64, torch.bfloat16, [0, 0], 16, seed=18)
    case.ck, case.cv, case.table = case.ck[:0], case.cv[:0], case.table[:, :0].contiguous()
    case.check()
    empty = Case(1, TREE7, 4, 2, 64, torch.bfloat16, [5], 16)
    empty.q, empty.tk, empty.tv = empty.q[:0], empty.tk[:0], empty.tv[:0]
    empty.table, empty.context = empty.table[:0], empty.context[:0]
    assert empty.run().out.shape[0] == 0


def test_two_calls_agree_bit_by_bit_and_another_stream_waits_for_nobody():
    print("[case] streams", flush=True)
    case = Case(8, DELAYED15, 8, 2, 128, torch.bfloat16, [3000, 5, 900, 64, 0, 1200, 33, 2500], 16, seed=19)
    first = case.run().out
    kept = case.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = mpv.TreeAttentionResult(out=torch.empty_like(first))
    case.run(out=other, stream=side)
    again = case.run(out=kept).out
    torch.cuda.synchronize()
    assert torch.equal(first, again) and torch.equal(first, other.out)


def test_captured_and_replayed_with_new_lengths():
    """A graph holds one call; lengths, tables and inputs change between the replays, with eager calls in between."""
    print("[case] graph", flush=True)
    case = Case(4, TREE7, 8, 2, 64, torch.bfloat16, [900, 900, 900, 900], 16, seed=20)
    kept = case.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        case.run(out=kept)
    for lengths in ([900, 1, 0, 64], [3, 899, 512, 77], [0, 0, 0, 0], [900, 900, 900, 900]):
        case.context.copy_(torch.tensor(lengths, dtype=torch.int32))
        case.q.normal_()
        eager = case.run().out
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(kept.out, eager), lengths
        case.check(kept.out)


def test_a_cache_whose_offsets_pass_32_bits():
    """8 GiB of keys: the last pages lie behind 2^31 elements."""
    print("[case] far offsets", flush=True)
    pages, page, KV, D = 9000, 512, 8, 128        # 4.7e9 elements of keys, as many of values
    ck = torch.empty(pages, page, KV, D, dtype=torch.bfloat16, device="cuda")
    cv = torch.empty_like(ck)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(21)
    used = [pages - 1, 17, pages - 2]
    for p in used:
        ck[p] = torch.randn(page, KV, D, generator=gen, device="cuda").to(torch.bfloat16)
        cv[p] = torch.randn(page, KV, D, generator=gen, device="cuda").to(torch.bfloat16)
    q = torch.randn(1, 3, 16, D, generator=gen, device="cuda").to(torch.bfloat16)
    tk, tv = torch.randn(2, 1, 3, KV, D, generator=gen, device="cuda").to(torch.bfloat16)
    context = torch.tensor([1300], dtype=torch.int32, device="cuda")
    far = mpv.mpv_tree_attention(CHAIN3, q, tk, tv, ck, cv, torch.tensor([used], dtype=torch.int32, device="cuda"), context).out
    near = mpv.mpv_tree_attention(CHAIN3, q, tk, tv, ck[used].clone(), cv[used].clone(),
                                  torch.tensor([[0, 1, 2]], dtype=torch.int32, device="cuda"), context).out
    torch.cuda.synchronize()
    assert torch.equal(far, near)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("N,H,KV", [(5, 3, 1), (10, 3, 1), (20, 3, 1), (33, 3, 1), (52, 3, 1), (43, 9, 1)])
def test_numbers_of_rows(N, H, KV, D, dtype):
    """15, 30, 60, 99, 156 and 387 rows a cache head, none of them a whole number of 16: every number of waves and of blocks."""
    print("[case] rows", N, H, KV, D, dtype, flush=True)
    rng = np.random.default_rng(N)
    parent = [-1] + [int(rng.integers(max(0, n - 4), n)) for n in range(1, N)]
    Case(2, parent, H, KV, D, dtype, [150, 77], 16, window=100, sinks=2, seed=N + D).check()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,KV", [(70, 1), (150, 8), (333, 2)])
def test_many_trees(B, KV, dtype):
    """More trees than a wave has lanes, more units than there are workgroups; empty trees among them."""
    print("[case] many trees", B, KV, dtype, flush=True)
    rng = np.random.default_rng(B)
    context = rng.integers(0, 90, B).tolist()
    context[B // 2] = 1500
    nodes = rng.integers(0, 4, B).tolist()
    case = Case(B, CHAIN3, KV, KV, 32, dtype, context, 16, nodes=nodes, seed=B)
    case.out = mpv.TreeAttentionResult(out=torch.full_like(case.q, 7.0))
    got = case.check(case.run(out=case.out).out)
    for b, n in enumerate(nodes):
        assert (got[b, n:] == 7.0).all()


def test_no_tree_has_a_node():
    print("[case] all empty", flush=True)
    case = Case(5, CHAIN3, 4, 2, 64, torch.bfloat16, [90, 0, 3, 64, 700], 16, nodes=[0, 0, -1, 0, 0], seed=22)
    out = mpv.TreeAttentionResult(out=torch.full_like(case.q, 7.0))
    assert (case.run(out=out).out == 7.0).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scale", [0.0, -0.2, 1.0])
def test_scales(scale, dtype):
    print("[case] scale", scale, dtype, flush=True)
    Case(2, TREE7, 4, 2, 64, dtype, [300, 40], 16, seed=23, scale=scale, gain=0.3).check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("fill", [float("nan"), float("inf"), -float("inf")])
def test_what_all_see_reaches_all(dtype, fill):
    """A value in the context that is no number spoils its column in every node of its tree, and nothing else."""
    print("[case] seen by all", dtype, fill, flush=True)
    case = Case(2, TREE7, 4, 2, 64, dtype, [500, 90], 16, seed=24)
    clean = case.run().out.clone()
    case.cv[case.table[0, 3], 5, 1, 9] = fill
    got = case.run().out
    spoiled = torch.zeros_like(got, dtype=torch.bool)
    spoiled[0, :, 2:, 9] = True
    assert torch.equal(got[~spoiled], clean[~spoiled])
    assert not torch.isfinite(got[spoiled]).any() and (fill == fill or torch.isnan(got[spoiled]).all())


def test_a_key_of_minus_infinity_has_no_weight():
    print("[case] infinite key", flush=True)
    case = Case(1, TREE7, 2, 2, 64, torch.float32, [70], 16, seed=25)
    case.q.abs_()
    case.tk[0, 1] = -float("inf")                 # its products are -inf: seen by nodes 1, 2 and 3, without weight
    got = case.run().out.clone()
    assert torch.isfinite(got).all()
    case.tv[0, 1] += 5.0
    assert torch.equal(case.run().out, got)


def test_pages_of_one_slot_and_of_many():
    """The same context in pages of other sizes: the same results, bit by bit."""
    print("[case] page sizes", flush=True)
    first = Case(1, TREE7, 4, 2, 64, torch.bfloat16, [900], 1, seed=26)
    k, v = torch.randn(2, 900, 2, 64, device="cuda").to(torch.bfloat16)
    at = torch.arange(900, device="cuda")
    outs = []
    for page in (1, 3, 16, 1000):
        case = Case(1, TREE7, 4, 2, 64, torch.bfloat16, [900], page, seed=26)
        case.q, case.tk, case.tv = first.q, first.tk, first.tv
        case.ck[case.table[0, at // page].long(), at % page] = k
        case.cv[case.table[0, at // page].long(), at % page] = v
        outs.append(case.run().out)
    assert all(torch.equal(o, outs[0]) for o in outs)
