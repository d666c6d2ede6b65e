"""mpv_score_positions and mpv_evict_positions against their definitions in 64 bits (needs an MI355X).

A score is a sum of weights e^(s - lse), with D products of a sum in float32, s and lse as large as the definition's `bound` adds up.  With
e = 2^-24: the products' sum (D + 1) e of the absolute products; the difference and its turn into log2 units 2 e (|s| + |lse|) + 2 e |s - lse|;
the exponential 4 e; sums over n rows and lanes (n + 8) e; the old score's product 2 e.  All are below (D + 8 + rows) e times
`bound` + 8 (rows + D) e times the score.  What is evicted is copied: exact.
"""

import numpy as np
import pytest
import torch

import paper_2602_16994_amd as mpv
from oracle import eviction_oracle as eo

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16, torch.float32]


def generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


class Scores:
    def __init__(self, layers, N, H, KV, D, dtype, context, page, accept, path, per_head=True, seed=1, spare=1, layered=True):
        gen = generator(seed)
        B = len(context)
        width = -(-max(context) // page) + spare
        self.pages = B * width + 2

        def rand(*shape):
            return torch.randn(*shape, generator=gen, device="cuda").to(dtype)

        lead = (layers,) if layered else ()
        self.q, self.tree_k, self.cache_k = rand(*lead, B, N, H, D), rand(*lead, B, N, KV, D), rand(*lead, self.pages, page, KV, D)
        self.lse = 3.0 + torch.rand(*lead, B, N, H, generator=gen, device="cuda")
        self.scores = torch.rand(*lead, B, KV if per_head else 1, width * page + 3, generator=gen, device="cuda")
        self.table = torch.randperm(self.pages, generator=gen, device="cuda")[:B * width].view(B, width).to(torch.int32)
        self.context = torch.tensor(context, dtype=torch.int32, device="cuda")
        self.accept = None if accept is None else torch.tensor(accept, dtype=torch.int32, device="cuda")
        self.path = None if path is None else torch.tensor(path, dtype=torch.int32, device="cuda")
        self.layered, self.N = layered, N

    def check(self, scale=None, decay=1.0):
        def host(t):
            t = t if self.layered else t.unsqueeze(0)
            return t.double().cpu().numpy()

        D = self.q.shape[-1]
        B = self.context.shape[0]
        accept = [0] * B if self.accept is None else [min(max(int(a), 0), self.N - 1 if self.path is None else min(self.path.shape[1], self.N - 1)) for a in self.accept]
        path = [list(range(1, self.N))] * B if self.path is None else self.path.tolist()
        want, bound = eo.score_positions(host(self.q), host(self.tree_k), host(self.cache_k), self.table.cpu().numpy(), self.context.tolist(),
                                         host(self.lse), host(self.scores), accept, path, D ** -0.5 if scale is None else scale, decay)
        mpv.mpv_score_positions(self.q, self.tree_k, self.cache_k, self.table, self.context, self.lse, self.scores, accept_len=self.accept,
                                path_nodes=self.path, scale=scale, decay=decay)
        got, e = host(self.scores), 2.0 ** -24
        rows = (max(accept, default=0) + 1) * self.q.shape[-2] + 8
        tol = (D + 8 + rows) * e * bound + 8 * (rows + D) * e * np.abs(want) + 1e-300
        off = (np.abs(got - want) / tol)[~np.isnan(want)]
        print("[largest error over its bound] %.3f" % off.max(), flush=True)
        assert np.array_equal(np.isnan(got), np.isnan(want)) and off.max() <= 1.0


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layers,N,H,KV,D,context,page,accept,path,per_head", [
    (1, 1, 1, 1, 8, [0], 16, None, None, True),
    (1, 1, 4, 1, 64, [1, 15, 16, 17], 1, None, None, True),
    (2, 5, 8, 2, 128, [100, 0, 63], 16, [4, 0, 2], [[1, 2, 3, 4], [-1] * 4, [1, 4, -1, -1]], True),
    (2, 5, 8, 2, 128, [100, 0, 63], 16, [4, 0, 2], [[1, 2, 3, 4], [-1] * 4, [1, 4, -1, -1]], False),
    (1, 4, 6, 2, 80, [130, 257], 24, [3, 1], None, True),
    (1, 7, 24, 2, 96, [77], 7, [3], [[2, 5, 6]], True),
    (3, 3, 12, 12, 72, [65, 5], 32, [1, 2], [[2, -1], [1, 2]], False),
    (1, 2, 3, 1, 192, [300], 64, [1], [[1]], True),
    (1, 2, 4, 4, 256, [90, 500], 128, [0, 1], None, True),
    (1, 20, 16, 1, 40, [33], 16, [19], None, True),
])
def test_scores(layers, N, H, KV, D, context, page, accept, path, per_head, dtype):
    print("[case] scores", layers, N, H, KV, D, context, page, per_head, dtype, flush=True)
    Scores(layers, N, H, KV, D, dtype, context, page, accept, path, per_head, seed=D + N).check(decay=0.9)


def test_scores_of_one_layer_without_its_dimension():
    print("[case] scores one layer", flush=True)
    case = Scores(1, 3, 4, 2, 64, torch.bfloat16, [50, 9], 16, [2, 0], [[1, 2], [-1, -1]], layered=False)
    case.check(scale=-0.3, decay=0.0)


def test_scores_of_pages_nodes_and_lengths_out_of_range():
    print("[case] scores out of range", flush=True)
    case = Scores(2, 4, 4, 2, 64, torch.float16, [50, 40, 20], 16, [3, 9, -2], [[1, 4, 2], [3, -1, 1], [-1] * 3], spare=0)
    case.table[0, 1] = -1
    case.table[1, 2] = case.pages
    case.context[2] = 1000                          # taken as the row's 64 slots: the path does not fit the scores
    case.check()


@pytest.mark.parametrize("dtype", TYPES)
def test_scores_of_rows_that_saw_nothing_or_no_number(dtype):
    print("[case] scores lse", dtype, flush=True)
    case = Scores(1, 2, 4, 2, 64, dtype, [50], 16, [1], [[1]])
    case.lse[0, 0, 0, 1] = -float("inf")
    case.lse[0, 0, 1, 0] = float("inf")
    case.cache_k[0, int(case.table[0, 1]), 3, 0, 5] = float("nan")         # position 19, the first cache head: its score alone
    before = case.scores.clone()
    mpv.mpv_score_positions(case.q, case.tree_k, case.cache_k, case.table, case.context, case.lse, case.scores, case.accept, case.path)
    nan = torch.isnan(case.scores)
    assert nan.sum() == 1 and nan[0, 0, 0, 19]
    case.cache_k[0, int(case.table[0, 1]), 3, 0, 5] = 0.0
    case.scores.copy_(before)
    case.check()


def test_scores_follow_the_attention():
    """With lse of mpv_prefix_attention the weights of a node add up to the number of its query heads, the prefix's share aside."""
    print("[case] scores sum", flush=True)
    gen = generator(4)
    B, N, H, KV, D, page = 3, 4, 8, 2, 64, 16
    t = torch.bfloat16
    q, k, v = (torch.randn(B, N, n, D, generator=gen, device="cuda").to(t) for n in (H, KV, KV))
    ck, cv = (torch.randn(20, page, KV, D, generator=gen, device="cuda").to(t) for _ in range(2))
    table = torch.randperm(20, generator=gen, device="cuda")[:15].view(B, 5).to(torch.int32)
    context = torch.tensor([70, 0, 33], dtype=torch.int32, device="cuda")
    accept = torch.tensor([3, 0, 1], dtype=torch.int32, device="cuda")
    lse = mpv.mpv_prefix_attention([-1, 0, 1, 2], q, k, v, ck, cv, table, context, lse=True).lse
    scores = torch.zeros(B, KV, 96, device="cuda")
    mpv.mpv_score_positions(q, k, ck, table, context, lse, scores, accept_len=accept)
    for b, a in enumerate([3, 0, 1]):
        n = int(context[b]) + a + 1
        assert torch.allclose(scores[b, :, :n].sum(dim=1), torch.full((KV,), (a + 1.0) * H / KV, device="cuda"), rtol=1e-4)
        assert (scores[b, :, n:] == 0).all()


# ---------------------------------------------------------------- eviction


class Evict:
    def __init__(self, layers, KV, D, dtype, context, page, budget, trigger, sinks, recent, per_head=True, seed=1, levels=0, spread=False, spare=0,
                 layered=True):
        gen = generator(seed)
        B = len(context)
        width = -(-max(context) // page) + spare
        self.pages = B * width + 4
        lead = (layers,) if layered else ()

        def rand(*shape):
            return torch.randn(*shape, generator=gen, device="cuda").to(dtype)

        if spread:
            both = rand(*lead, self.pages, 2, page, KV, D)
            self.k, self.v = both.select(-4, 0), both.select(-4, 1)
        else:
            self.k, self.v = rand(*lead, self.pages, page, KV, D), rand(*lead, self.pages, page, KV, D)
        shape = (*lead, B, KV if per_head else 1, width * page + 5)
        self.scores = torch.rand(shape, generator=gen, device="cuda") - 0.2
        if levels:
            self.scores = torch.randint(0, levels, shape, generator=gen, device="cuda").float()
        order = torch.randperm(self.pages, generator=gen, device="cuda").to(torch.int32)
        self.table = order[:B * width].view(B, width).clone()
        self.free = torch.full((self.pages,), -1, dtype=torch.int32, device="cuda")
        self.free[:4] = order[B * width:]
        self.free_count = torch.tensor([4], dtype=torch.int32, device="cuda")
        self.context = torch.tensor(context, dtype=torch.int32, device="cuda")
        self.args = (budget, trigger, sinks, recent)
        self.layered = layered

    def call(self, **kw):
        budget, trigger, sinks, recent = self.args
        return mpv.mpv_evict_positions(self.k, self.v, self.table, self.context, self.scores, self.free, self.free_count, budget, trigger=trigger,
                                       sinks=sinks, recent=recent, **kw)

    def check(self, **kw):
        def host(t):
            return (t if self.layered else t.unsqueeze(0)).double().cpu().numpy()

        k, v, new, kept, free, after = eo.evict_positions(host(self.k), host(self.v), self.table.cpu().numpy(), self.context.tolist(), host(self.scores),
                                                          self.free.tolist(), int(self.free_count), *self.args)
        old_scores, table = self.scores.clone(), self.table.clone()
        r = self.call(**kw)
        assert np.array_equal(host(r.kept), kept)
        assert np.array_equal(host(self.k), k, equal_nan=True) and np.array_equal(host(self.v), v, equal_nan=True)
        assert r.context_len.tolist() == after and int(r.free_count) == len(free) and self.free[:len(free)].tolist() == free
        assert torch.equal(self.table, table)
        got = host(r.scores)
        there = np.zeros(got.shape, dtype=bool)
        for b, n in enumerate(after):
            there[:, b, :, :n] = True
        assert np.array_equal(got[there], np.where(np.isnan(new), host(r.scores), new)[there], equal_nan=True)
        assert (np.isnan(new) == ~there).all() or np.isnan(host(old_scores)).any()
        return r


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layers,KV,D,context,page,budget,trigger,sinks,recent,per_head", [
    (1, 1, 8, [2], 1, 1, 1, 0, 0, True),
    (1, 1, 64, [40, 17, 0, 16], 16, 16, 16, 0, 0, True),
    (2, 2, 128, [100, 64, 65, 200], 16, 64, 64, 4, 16, True),
    (2, 2, 128, [100, 64, 65, 200], 16, 64, 64, 4, 16, False),
    (1, 3, 80, [700, 30, 511], 24, 100, 300, 0, 100, True),
    (1, 3, 80, [700, 30, 511], 24, 100, 300, 50, 50, False),
    (3, 2, 72, [90, 91], 7, 90, 90, 1, 2, True),
    (1, 2, 256, [1500], 64, 1000, 1000, 3, 10, True),
    (1, 1, 40, [5000, 4097, 100], 128, 33, 4096, 33, 0, False),
    (1, 4, 192, [260], 5, 259, 259, 0, 0, True),
])
def test_eviction(layers, KV, D, context, page, budget, trigger, sinks, recent, per_head, dtype):
    print("[case] evict", layers, KV, D, context, page, budget, trigger, sinks, recent, per_head, dtype, flush=True)
    Evict(layers, KV, D, dtype, context, page, budget, trigger, sinks, recent, per_head, seed=budget).check()


@pytest.mark.parametrize("inplace", [False, True])
def test_in_place_and_not(inplace):
    print("[case] evict in place", inplace, flush=True)
    case = Evict(2, 2, 64, torch.bfloat16, [900, 100, 300], 16, 200, 250, 2, 20, seed=3)
    before = case.context.clone(), case.free_count.clone(), case.scores.clone()
    r = case.check(inplace=inplace)
    assert (r.scores is case.scores) == inplace and (r.context_len is case.context) == inplace
    if not inplace:
        for was, now in zip(before, (case.context, case.free_count, case.scores)):
            assert torch.equal(was, now)
        again = case.call(out=r)                   # the same lists; its own buffers
        assert again is r and r.scores is not case.scores


@pytest.mark.parametrize("levels", [1, 2, 7])
def test_equal_scores(levels):
    print("[case] evict ties", levels, flush=True)
    Evict(2, 2, 64, torch.bfloat16, [3000, 700], 16, 500, 500, 3, 30, seed=levels, levels=levels).check()


def test_scores_that_are_no_numbers():
    print("[case] evict nan", flush=True)
    case = Evict(1, 2, 64, torch.float32, [300], 16, 100, 100, 0, 0, seed=8)
    case.scores[0, 0, 0, :250] = float("nan")
    case.scores[0, 0, 0, 5] = -float("inf")
    case.scores[0, 0, 1, 10:20] = float("inf")
    case.scores[0, 0, 1, 30:40] = -0.0
    case.scores[0, 0, 1, 40:50] = 0.0
    case.check()


def test_one_layer_and_interleaved_caches():
    print("[case] evict layout", flush=True)
    Evict(1, 2, 64, torch.bfloat16, [90, 40], 16, 32, 50, 1, 4, layered=False).check()
    Evict(2, 2, 64, torch.float16, [90, 400], 16, 32, 50, 1, 4, spread=True).check()


def test_pages_that_are_none_and_a_list_that_is_full():
    print("[case] evict bad pages", flush=True)
    case = Evict(1, 2, 64, torch.bfloat16, [90, 200], 16, 32, 50, 0, 0, seed=5)
    case.table[0, 0] = -1
    case.table[1, 3] = case.pages
    case.free_count.fill_(case.pages - 3)
    case.free.copy_(torch.arange(case.pages, device="cuda"))
    case.context[1] = 100000
    case.check()


def test_many_requests():
    print("[case] evict many", flush=True)
    rng = np.random.default_rng(1)
    Evict(1, 1, 8, torch.bfloat16, [int(x) for x in rng.integers(0, 60, 700)], 4, 20, 30, 1, 3, seed=6).check()


def test_lengths_and_pages_without_layers():
    print("[case] evict no layers", flush=True)
    case = Evict(0, 2, 64, torch.bfloat16, [90, 200, 3], 16, 32, 50, 0, 0, seed=7)
    r = case.call()
    assert r.context_len.tolist() == [32, 32, 3] and int(r.free_count) == 4 + 4 + 11


def test_an_empty_batch():
    print("[case] evict empty", flush=True)
    case = Evict(1, 2, 64, torch.bfloat16, [20], 16, 4, 4, 0, 0)
    case.table, case.context, case.scores = case.table[:0], case.context[:0], case.scores[:, :0].contiguous()
    r = case.call()
    assert int(r.free_count) == 4 and r.context_len.shape == (0,)
    s = Scores(1, 1, 1, 1, 8, torch.bfloat16, [0], 16, None, None)
    mpv.mpv_score_positions(s.q[:, :0], s.tree_k[:, :0], s.cache_k, s.table[:0], s.context[:0], s.lse[:, :0].contiguous(), s.scores[:, :0].contiguous())
