"""A serving loop with requests behind shared prefixes whose own caches are kept within a budget (needs an MI355X): attention, verification,
log probabilities, scores, room, accepted rows, eviction."""

import numpy as np
import pytest
import torch

import paper_2602_16994_amd as mpv
from oracle import eviction_oracle as eo
from oracle import logprobs_oracle as lo
from oracle import prefix_oracle as po

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("per_head", [True, False])
@pytest.mark.parametrize("graph", [False, True])
def test_a_loop_that_evicts(graph, per_head):
    """After every step: the attention over prefix, cache and tree is the definition's; scores are the definition's, from the attention's own
    sums; what is evicted is what the scores say, and the cache holds the rows that they kept."""
    print("[case] evicting loop", graph, per_head, flush=True)
    torch.manual_seed(5)
    B, layers, H, KV, D, V, size, steps, budget, trigger, sinks, recent = 5, 2, 4, 2, 64, 97, 8, 7, 12, 15, 2, 4
    parent = mpv.delayed_tree(2, 1, 2)
    N, depth, width, dev = len(parent), 3, 4, "cuda"
    G = KV if per_head else 1
    pages = B * width + 2 * 4
    ck, cv = torch.randn(2, layers, pages, size, KV, D, device=dev).to(torch.bfloat16)
    order = torch.randperm(pages, device=dev).to(torch.int32)
    prefix_table, prefix_len = order[:8].view(2, 4).clone(), torch.tensor([29, 11], dtype=torch.int32, device=dev)
    prefix_of = torch.tensor([0, 0, 1, -1, 1], dtype=torch.int32, device=dev)
    table = torch.full((B, width), -1, dtype=torch.int32, device=dev)
    free = torch.full((pages,), -1, dtype=torch.int32, device=dev)
    free[:B * width] = order[8:]
    count = torch.tensor([B * width], dtype=torch.int32, device=dev)
    context = torch.zeros(B, dtype=torch.int32, device=dev)
    slots = torch.full((B, depth + 1), -1, dtype=torch.int64, device=dev)
    q = torch.empty(layers, B, N, H, D, device=dev, dtype=torch.bfloat16)
    tk, tv = torch.empty(2, layers, B, N, KV, D, device=dev, dtype=torch.bfloat16)
    lse = torch.empty(layers, B, N, H, device=dev)
    scores = torch.zeros(layers, B, G, width * size, device=dev)
    target, draft = torch.empty(B, N, V, device=dev), torch.empty(B, N, V, device=dev)
    tokens, u = torch.empty(B, N, dtype=torch.int32, device=dev), torch.empty(B, N, device=dev)
    outs = [mpv.PrefixAttentionResult(out=torch.empty(B, N, H, D, device=dev, dtype=torch.bfloat16), lse=lse[i]) for i in range(layers)]
    held = {}

    def step():
        for i in range(layers):
            mpv.mpv_prefix_attention(parent, q[i], tk[i], tv[i], ck[i], cv[i], table, context, prefix_of, prefix_table, prefix_len, out=outs[i])
        held["res"] = r = mpv.mpv_verify(parent, tokens, target, draft, 1.0, u, mpv.MPV_METHOD_TRAVERSAL, out=held.get("res"))
        held["logp"] = mpv.mpv_token_logprobs(target, r.path_tokens, top=3, accept_len=r.accept_len, path_nodes=r.path_nodes,
                                              bonus_token=r.bonus_token, out=held.get("logp"))
        mpv.mpv_score_positions(q, tk, ck, table, context, lse, scores, accept_len=r.accept_len, path_nodes=r.path_nodes, decay=0.75)
        held["tables"] = mpv.mpv_extend_tables(table, context, r.accept_len, free, count, size, slots, extra=1, inplace=True, out=held.get("tables"))
        mpv.mpv_append_paths(tk, tv, ck, cv, slots, r.accept_len, path_nodes=r.path_nodes)
        held["evict"] = mpv.mpv_evict_positions(ck, cv, table, context, scores, free, count, budget, trigger=trigger, sinks=sinks, recent=recent,
                                                inplace=True, out=held.get("evict"))

    state = (table, free, count, context, slots, ck, cv, scores)
    g, cut = None, 0

    def host(x):
        return x.double().cpu().numpy()

    for t in range(steps):
        for x in (q, tk, tv):
            x.normal_()
        target.normal_()
        draft.copy_(target + 0.3 * torch.randn_like(target))
        q_draft = torch.softmax(draft, -1)
        for n in range(1, N):
            tokens[:, n] = torch.multinomial(q_draft[:, parent[n]], 1).squeeze(1).to(torch.int32)
        tokens[:, 0] = 0
        u.uniform_()
        before = [x.clone() for x in state]
        if graph and t == 1:
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                step()
            for x, y in zip(state, before):
                assert torch.equal(x, y)
        g.replay() if g is not None else step()
        torch.cuda.synchronize()
        r = held["res"]
        r.raise_on_timeout()
        accept = r.accept_len.tolist()
        table0, _, _, context0, _, ck0, cv0, scores0 = before
        # attention
        for i in range(layers):
            want, A, S, seen, sums = po.prefix_attention(host(q[i]), host(tk[i]), host(tv[i]), host(ck0[i]), host(cv0[i]), table0.cpu().numpy(),
                                                         context0.tolist(), [parent] * B, [N] * B, prefix_of.tolist(), prefix_table.cpu().numpy(),
                                                         prefix_len.tolist(), 0, 0, D ** -0.5)
            assert (np.abs(host(outs[i].out) - want) <= 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2.0 ** -12) * A).all()
            assert np.abs(host(lse[i]) - sums).max() < 1e-4
        # log probabilities of what was emitted
        logp = held["logp"]
        for b in range(B):
            for i in range(accept[b] + 1):
                node = 0 if i == 0 else int(r.path_nodes[b, i - 1])
                token = int(r.bonus_token[b]) if i == accept[b] else int(r.path_tokens[b, i])
                lp, entropy, rank, best, _ = lo.row(host(target[b, node]), token, 1.0, 3)
                assert abs(float(logp.logprob[b, i]) - lp) < 1e-5 and abs(float(logp.entropy[b, i]) - entropy) < 1e-4
                assert int(logp.rank[b, i]) == rank and logp.top_tokens[b, i].tolist() == list(best)
        # scores, room and accepted rows, eviction: the definitions on the state before the step
        path = r.path_nodes.tolist()
        given, _ = eo.score_positions(host(q), host(tk), host(ck0), table0.cpu().numpy(), context0.tolist(), host(lse), host(scores0), accept, path,
                                      D ** -0.5, 0.75)
        k, v = host(ck0), host(cv0)
        long = [int(c) + a + 1 for c, a in zip(context0.tolist(), accept)]
        rows = table.cpu().numpy()
        for b in range(B):
            for i, n in enumerate([0] + path[b][:accept[b]]):
                at = int(context0[b]) + i
                k[:, rows[b, at // size], at % size] = host(tk[:, b, n])
                v[:, rows[b, at // size], at % size] = host(tv[:, b, n])
        k, v, new, kept, _, after = eo.evict_positions(k, v, rows, long, given, [], 0, budget, trigger, sinks, recent)
        assert context.tolist() == after
        cut += sum(n > trigger for n in long)
        assert int(count) == B * width - sum(-(-n // size) for n in after) and len(set(free[:int(count)].tolist())) == int(count)
        got = host(scores)
        for b in range(B):
            assert np.allclose(got[:, b, :, :after[b]], new[:, b, :, :after[b]], rtol=1e-4, atol=1e-6)
            for i in range(after[b]):
                page = rows[b, i // size]
                assert np.array_equal(host(ck[:, page, i % size]), k[:, page, i % size])
                assert np.array_equal(host(cv[:, page, i % size]), v[:, page, i % size])
        assert np.array_equal(held["evict"].kept.cpu().numpy(), kept)
    assert cut > 3
