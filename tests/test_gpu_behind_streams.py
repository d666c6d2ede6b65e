"""Attention behind prefixes, log probabilities, scores and eviction on other streams than the current one, in graphs, and with workspaces
that two graphs share (needs an MI355X)."""

import pytest
import torch

import paper_2602_16994_amd as mpv
from tests.test_gpu_eviction import Evict, Scores
from tests.test_gpu_logprobs import random
from tests.test_gpu_prefix_attention import Case
from tests.test_gpu_serving_streams import keep_busy, places
from tests.test_gpu_prefix_together import reads_together
from tests.test_gpu_tree_attention import TREE7

pytestmark = pytest.mark.gpu


def shared():
    """Enough to save that the prefixes are read together (single tokens, see mpv_behind.hip)."""
    return Case([-1], 8, 2, 128, torch.bfloat16, [0] * 90 + [1] * 100, [4000, 3000], [b % 70 for b in range(190)], 64, seed=31)


def own():
    return Case(TREE7, 8, 2, 128, torch.bfloat16, [0, 0, 1, -1], [300, 77], [100, 0, 31, 64], 16, seed=32)


def logprobs():
    logits, tokens = random(6, 5, 70001, torch.bfloat16, 33)
    return lambda **kw: mpv.mpv_token_logprobs(logits, tokens, top=9, **kw)


def evict(**kw):
    case = Evict(2, 2, 64, torch.bfloat16, [900, 100, 300], 16, 200, 250, 2, 20, seed=34)
    return case.call(**kw)


CALLS = {
    "shared": (lambda: shared().run, ("out", "lse")),
    "own": (lambda: own().run, ("out", "lse")),
    "logprobs": (logprobs, ("logprob", "entropy", "rank", "top_tokens", "top_logprobs")),
    "evict": (lambda: evict, ("context_len", "free_count", "kept")),
}


def test_prefixes_are_read_together_where_the_tests_mean_it():
    print("[case] shared state", flush=True)
    case, other = shared(), own()
    assert reads_together(case)
    case.check()
    other.check()


@pytest.mark.parametrize("kind", CALLS)
def test_what_is_allocated_is_not_still_in_use_on_the_current_stream(kind):
    print("[case] behind: allocated for another stream", kind, flush=True)
    make, names = CALLS[kind]
    call = make()
    want = call()
    side, here = torch.cuda.Stream(), torch.cuda.current_stream()
    busy = torch.zeros(64 << 20, device="cuda")
    if kind == "evict":                            # (its caches are changed by a call: another one's, made beforehand)
        case = Evict(2, 2, 64, torch.bfloat16, [900, 100, 300], 16, 200, 250, 2, 20, seed=34)
        call = case.call
    torch.cuda.synchronize()
    keep_busy(here, busy)
    given_back = [torch.empty_like(getattr(want, n)) for n in (*names, "workspace") for _ in range(64)]
    for t in given_back:
        t.zero_()
    taken = {t.data_ptr() for t in given_back}
    del given_back, t
    kw = {} if kind in ("logprobs", "evict") else dict(lse=True)
    res = call(stream=side, **kw)
    assert not here.query() and not taken & places(res, (*names, "workspace"))
    torch.cuda.synchronize()
    for n in names:
        assert torch.equal(getattr(res, n), getattr(want, n)), n


def captured(calls):
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        calls()
    return graph


@pytest.mark.parametrize("kind", ["shared", "own"])
def test_attention_replayed_from_two_graphs_that_share_a_workspace(kind):
    print("[case] behind: graphs", kind, flush=True)
    case = shared() if kind == "shared" else own()
    a = case.run()
    b = mpv.PrefixAttentionResult(out=torch.empty_like(a.out), lse=torch.empty_like(a.lse), workspace=a.workspace)
    q = case.q                                     # (the first graph reads it)
    other = case.q.flip(0).contiguous()
    torch.cuda.synchronize()
    first = captured(lambda: case.run(out=a))
    case.q = other
    case.run(out=b)
    torch.cuda.synchronize()
    second = captured(lambda: case.run(out=b))
    assert a.workspace is b.workspace
    for turn in range(3):
        case.context.copy_((case.context + 1) % 65)
        case.prefix_len.sub_(17)
        case.q = q
        want = case.run()
        case.q = other
        want_other = case.run()
        torch.cuda.synchronize()
        for x in (a.out, a.lse, b.out, b.lse):
            x.fill_(7.0)
        first.replay()
        second.replay()
        first.replay()
        torch.cuda.synchronize()
        for got, w in ((a, want), (b, want_other)):
            assert torch.equal(got.out, w.out) and torch.equal(got.lse, w.lse), turn
    case.q = other
    case.check(b)


def test_scores_and_eviction_replayed():
    """A call in place, over and over, eagerly and from a graph: lengths, scores, lists of free pages and caches stay the same."""
    print("[case] behind: eviction in a graph", flush=True)
    cases = [Evict(2, 2, 64, torch.bfloat16, [90, 40, 64], 8, 30, 40, 2, 6, seed=35, spare=2) for _ in range(2)]
    scores = Scores(2, 3, 4, 2, 64, torch.bfloat16, [90, 40, 64], 8, [2, 0, 1], [[1, 2], [-1, -1], [2, -1]], seed=36, spare=2)

    def step(case, out=None):
        mpv.mpv_score_positions(scores.q, scores.tree_k, case.k, case.table, case.context, scores.lse, case.scores, accept_len=scores.accept,
                                path_nodes=scores.path, decay=0.5)
        out = case.call(inplace=True, out=out)
        case.context.add_(9)                       # as if tokens were appended, into pages that the table still names
        return out

    outs = [step(case) for case in cases]
    torch.cuda.synchronize()
    state = [x.clone() for x in (cases[1].k, cases[1].v, cases[1].scores, cases[1].context, cases[1].free, cases[1].free_count)]
    graph = captured(lambda: step(cases[1], outs[1]))
    for x, y in zip((cases[1].k, cases[1].v, cases[1].scores, cases[1].context, cases[1].free, cases[1].free_count), state):
        assert torch.equal(x, y)                   # capturing ran nothing
    cut = 0
    for turn in range(5):
        outs[0] = step(cases[0], outs[0])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0].kept, outs[1].kept), turn
        for name in ("k", "v", "scores", "context", "free", "free_count"):
            assert torch.equal(getattr(cases[0], name), getattr(cases[1], name)), (turn, name)
        cut += int((outs[0].kept[:, :, :, 0] == 0).sum())
    assert cut > 8


def test_two_calls_at_once_on_two_streams():
    print("[case] behind: two streams", flush=True)
    cases = [shared(), own()]
    logp = logprobs()
    want = [c.run() for c in cases] + [logp()]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        got = [c.run(stream=s) for c, s in zip(cases, streams)] + [logp(stream=streams[2])]
        torch.cuda.synchronize()
        for g, w in zip(got[:2], want[:2]):
            assert torch.equal(g.out, w.out) and torch.equal(g.lse, w.lse)
        assert torch.equal(got[2].top_tokens, want[2].top_tokens) and torch.equal(got[2].logprob, want[2].logprob)
