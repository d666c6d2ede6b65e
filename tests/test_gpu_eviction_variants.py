"""mpv_evict_positions in each of its kernels: lists of every length, rows of every width (needs an MI355X).

The definition is written out for what a call has to leave: kept positions by sorting, the caches' rows by indexing.  All of it is exact, and
positions that are there are compared whatever their score is, NaN among them.
"""

import numpy as np
import pytest
import torch

import paper_2602_16994_amd as mpv

pytestmark = pytest.mark.gpu


def kept_positions(scores, context, budget, sinks, recent):
    """The kept positions of one list, in order: of equal scores the first, NaN less than any number."""
    middle = scores[sinks:context - recent].astype(np.float64)
    value = np.where(np.isnan(middle), -np.inf, middle)
    order = np.lexsort((np.arange(len(middle)), np.isnan(middle), -value))[:budget - sinks - recent]
    return np.concatenate([np.arange(sinks), np.sort(order) + sinks, np.arange(context - recent, context)]).astype(np.int64)


class Case:
    def __init__(self, layers, KV, D, dtype, context, page, width, per_head, seed, levels=0):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.layers, self.B, self.G, self.page, self.width = layers, len(context), KV if per_head else 1, page, width
        self.pages = self.B * width + 3

        def rand(*shape):
            return torch.randn(*shape, generator=gen, device="cuda").to(dtype)

        self.k, self.v = (rand(layers, self.pages, page, KV, D) for _ in range(2))
        shape = (layers, self.B, self.G, width * page + 3)
        self.scores = torch.randn(shape, generator=gen, device="cuda")
        if levels:
            self.scores = torch.randint(0, levels, shape, generator=gen, device="cuda").float()
        order = torch.randperm(self.pages, generator=gen, device="cuda").to(torch.int32)
        self.table = order[:self.B * width].view(self.B, width).clone()
        self.free = torch.full((self.pages,), -1, dtype=torch.int32, device="cuda")
        self.free[:3] = order[self.B * width:]
        self.count = torch.tensor([3], dtype=torch.int32, device="cuda")
        self.context = torch.tensor(context, dtype=torch.int32, device="cuda")

    def check(self, budget, trigger, sinks, recent, **kw):
        lengths, old = self.context.tolist(), self.scores.clone()
        want_scores, scores = old.clone(), old.cpu().numpy()
        want_kept = torch.full((self.layers, self.B, self.G, budget), -1, dtype=torch.int32)
        free, table = self.free[:int(self.count)].tolist(), self.table.cpu().numpy()
        flat = [t.clone().flatten(1, 2) for t in (self.k, self.v)]
        want = [t.clone() for t in flat]
        after = []
        for b, length in enumerate(lengths):
            after.append(budget if length > trigger else length)
            if length <= trigger:
                continue
            free += [int(x) for x in table[b, -(-budget // self.page):-(-length // self.page)]]
            slot = torch.from_numpy((table[b].astype(np.int64)[:, None] * self.page + np.arange(self.page)).reshape(-1)).cuda()
            for layer in range(self.layers):
                for g in range(self.G):
                    keep = kept_positions(scores[layer, b, g], length, budget, sinks, recent)
                    want_kept[layer, b, g] = torch.from_numpy(keep)
                    at = torch.from_numpy(keep).cuda()
                    want_scores[layer, b, g, :budget] = old[layer, b, g, at]
                    heads = slice(g, g + 1) if self.G > 1 else slice(None)
                    for new, was in zip(want, flat):
                        new[layer, slot[:budget], heads] = was[layer, slot[at], heads]
        r = mpv.mpv_evict_positions(self.k, self.v, self.table, self.context, self.scores, self.free, self.count, budget, trigger=trigger, sinks=sinks,
                                    recent=recent, **kw)
        assert torch.equal(r.kept.cpu(), want_kept)
        assert torch.equal(self.k.flatten(1, 2), want[0]) and torch.equal(self.v.flatten(1, 2), want[1])
        assert r.context_len.tolist() == after and int(r.free_count) == len(free) and self.free[:len(free)].tolist() == free
        assert torch.equal(self.table.cpu(), torch.from_numpy(table))
        got, there = r.scores, torch.zeros(old.shape, dtype=torch.bool, device="cuda")
        for b, length in enumerate(after):
            there[:, b, :, :length] = True
        same = (got == want_scores) | (torch.isnan(got) & torch.isnan(want_scores))
        assert bool(same[there].all())
        if kw.get("inplace"):
            assert r.scores is self.scores
        else:
            assert bool(((self.scores == old) | (torch.isnan(self.scores) & torch.isnan(old))).all())


@pytest.mark.parametrize("inplace", [False, True])
@pytest.mark.parametrize("kind", ["random", "ties", "nan", "first and last"])
@pytest.mark.parametrize("width,page", [(1024, 1), (205, 5), (512, 16), (8193, 1), (1000, 32), (4096, 8), (2185, 15), (10001, 4)])
def test_lists_of_every_length(width, page, kind, inplace):
    """Room for 1024, 1025, 8192, 8193, 32 000, 32 768, 32 775 and 40 004 positions: the borders of the kernels that select."""
    print("[case] evict lists", width, page, kind, inplace, flush=True)
    room = width * page
    context = [room, room - 1, room * 2 // 3, 900, 3]
    case = Case(1, 2, 8, torch.bfloat16, context, page, width, True, seed=room, levels=3 if kind == "ties" else 0)
    if kind == "nan":
        case.scores[0, 0, 0, ::2] = float("nan")
        case.scores[0, 0, 1, 5:room - 7] = float("nan")
        case.scores[0, 1, 0, ::3] = -float("inf")
        case.scores[0, 1, 1, ::5] = float("inf")
        case.scores[0, 2, 0] = 0.0
        case.scores[0, 2, 0, 1::2] = -0.0
    if kind == "first and last":
        case.check(600, 700, 250, 350, inplace=inplace)
    else:
        case.check(room // 2 + 1, max(room // 2 + 1, 850), 4, 30, inplace=inplace)


# (bytes of a row, budget): what reaches a slice of 4, 8, 16, 32 and 64 pieces of 16 bytes, with 256 and with 1024 threads, of some hundred lists;
# two slices, the second of one piece; several slices
@pytest.mark.parametrize("KV,D,budget,requests", [
    (1, 32, 20, 300), (1, 32, 600, 300), (1, 64, 20, 300), (1, 64, 1100, 300), (1, 128, 20, 300), (1, 128, 520, 300), (2, 128, 20, 300), (2, 128, 260, 300),
    (4, 128, 20, 300), (4, 128, 135, 300), (5, 104, 40, 300), (5, 104, 140, 300), (16, 128, 30, 200), (1, 256, 700, 40), (8, 128, 400, 20),
])
def test_rows_of_every_width(KV, D, budget, requests):
    print("[case] evict rows", KV, D, budget, requests, flush=True)
    rng = np.random.default_rng(KV * D + budget)
    page = 16
    width = -(-(budget + budget // 3 + 9) // page)
    context = [int(x) for x in rng.integers(budget // 2, width * page + 1, requests)]
    Case(1, KV, D, torch.float16, context, page, width, False, seed=D + budget).check(budget, budget + 2, 2, 5)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_cache_heads_of_many_layers(dtype):
    """A head's part of a row is a slice of its own; rows of 512 bytes (float32) of 256 lists."""
    print("[case] evict heads", dtype, flush=True)
    Case(8, 4, 128, dtype, [300, 100, 257, 299, 30, 280, 260, 300], 16, 19, True, seed=9).check(100, 120, 4, 20, inplace=True)


def test_more_lists_than_workgroups_of_1024_threads():
    """80 layers of 20 000 requests, whole slots of 2048 bytes, a budget that takes 1024 threads a workgroup where a launch can have as many: none is cut."""
    print("[case] evict many lists", flush=True)
    layers, B, budget = 80, 20000, 300
    cache = torch.zeros(layers, 1, 1, 8, 128, dtype=torch.bfloat16, device="cuda")
    table = torch.zeros(B, 1, dtype=torch.int32, device="cuda")
    context = torch.ones(B, dtype=torch.int32, device="cuda")
    scores = torch.arange(layers * B, dtype=torch.float32, device="cuda").view(layers, B, 1, 1)
    free, count = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    r = mpv.mpv_evict_positions(cache, cache.clone(), table, context, scores, free, count, budget)
    assert torch.equal(r.context_len, context) and int(r.free_count) == 0 and torch.equal(r.scores, scores)
    assert int(r.kept.amax()) == -1 and int(r.kept.amin()) == -1


@pytest.mark.parametrize("inplace", [False, True])
@pytest.mark.parametrize("requests,width,short", [(1, 40, 0), (5, 300, 0), (70, 500, 0), (5, 300, 100), (3, 3000, 0)])
def test_entries_that_are_no_pages_do_not_become_free(requests, width, short, inplace):
    """What stands in a row of the block table behind the kept pages and is no page is not handed out; the pages around it are, in order, as far as the list
    holds them (`short`: places that it lacks)."""
    print("[case] evict no pages", requests, width, short, inplace, flush=True)
    rng = np.random.default_rng(width + requests)
    page, budget = 2, 30
    context = [int(x) for x in rng.integers(1, width * page + 1, requests)]
    context[0] = width * page
    case = Case(1, 1, 8, torch.bfloat16, context, page, width, True, seed=requests)
    table = case.table.cpu().numpy()
    strange = rng.random(table.shape) < 0.2
    strange[:, :16] = False                        # (a row that has no page does not move; here all of them do)
    table[strange] = rng.choice([-1, case.pages, 2 ** 31 - 1, -2 ** 31], int(strange.sum()))
    # kept positions lie anywhere: scores fall with the position, so that those that are kept are the first ones
    case.scores.copy_(-torch.arange(case.scores.shape[-1], device="cuda").float().expand_as(case.scores))
    case.table.copy_(torch.from_numpy(table))
    start = case.pages - short if short else 3
    start = max(3, start)
    case.free[:start] = torch.arange(start, dtype=torch.int32, device="cuda")
    case.count.fill_(start)
    free = list(range(start))
    for b, length in enumerate(context):
        if length > budget:
            free += [int(x) for x in table[b, budget // page:-(-length // page)] if 0 <= x < case.pages]
    free = free[:case.pages]
    behind = case.free[len(free):].clone()
    r = mpv.mpv_evict_positions(case.k, case.v, case.table, case.context, case.scores, case.free, case.count, budget, inplace=inplace)
    assert int(r.free_count) == len(free) and case.free[:len(free)].tolist() == free
    assert torch.equal(case.free[len(free):], behind)
    assert r.context_len.tolist() == [min(x, budget) for x in context]
