"""mpv_verify_chains against the definition in 64 bits (needs an MI355X).  Whole numbers have to be equal: the tests of tokens
are exact in doubles, a bonus token can differ only where the drawn point lies within the rounding of sums in doubles (V 2^-53,
relative) of a step of the cumulative mass, and no such draw is among the seeds (asserted)."""

import numpy as np
import pytest
import torch

import paper_2602_16994_amd as mpv
from oracle import serving_oracle as so

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]


def make(B, N, V, dtype, draft=True, seed=1, pad=0, sharp=2.5):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def rows():
        z = torch.randn(B, N, V + pad, generator=gen, device="cuda") * sharp
        return torch.softmax(z, dim=-1).to(dtype)[:, :, :V]

    q = rows()
    p = torch.softmax(torch.log(q.float() + 1e-9) + 0.7 * torch.randn(B, N, V, generator=gen, device="cuda"), dim=-1).to(dtype)
    if pad:
        wide = torch.zeros(B, N, V + pad, dtype=dtype, device="cuda")
        wide[:, :, :V] = p
        p = wide[:, :, :V]
    tokens = torch.zeros(B, N, dtype=torch.int32, device="cuda")
    for n in range(1, N):
        tokens[:, n] = torch.multinomial(q[:, n - 1].float() + 1e-12, 1, generator=gen).squeeze(1).to(torch.int32)
    return tokens, p, q if draft else None, torch.rand(B, N, generator=gen, device="cuda")


def check(tokens, p, q, u, nodes=None, res=None):
    B, N, V = p.shape
    num = None if nodes is None else torch.tensor(nodes, dtype=torch.int32, device="cuda")
    res = mpv.mpv_verify_chains(tokens, p, q, u, num_nodes=num) if res is None else res
    torch.cuda.synchronize()
    P, Q, U, T = p.double().cpu().numpy(), None if q is None else q.double().cpu().numpy(), u.double().cpu().numpy(), tokens.cpu().numpy()
    zeros = bads = 0
    for b in range(B):
        n = N if nodes is None else min(max(nodes[b], 1), N)
        a, bonus, zero, bad, gap = so.verify_chain(T[b, :n], P[b, :n], None if Q is None else Q[b, :n], U[b, :n])
        assert gap > V * 2.0 ** -53 or U[b, 0] == 0.0
        zeros, bads = zeros + zero, bads + bad
        assert int(res.accept_len[b]) == a, b
        assert int(res.bonus_token[b]) == bonus, b
        deep = res.path_nodes.shape[1]
        assert res.path_nodes[b].tolist() == list(range(1, a + 1)) + [-1] * (deep - a)
        assert res.path_tokens[b].tolist() == T[b, 1:a + 1].tolist() + [-1] * (deep - a)
    counters = res.counters.tolist()
    assert counters[mpv.MPV_COUNTER_ZERO_MASS] == zeros and counters[mpv.MPV_COUNTER_BAD_TOKEN] == bads
    assert sum(counters) == zeros + bads
    return res


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("B,N,V", [(1, 1, 1), (1, 2, 2), (3, 4, 7), (5, 1, 1000), (40, 5, 63), (33, 6, 1024), (7, 64, 257), (17, 3, 8191),
                                   (4, 5, 32000), (3, 9, 50001), (2, 3, 262144)])
def test_sizes(B, N, V, draft, dtype):
    print("[case] chains", B, N, V, draft, dtype, flush=True)
    check(*make(B, N, V, dtype, draft, seed=B + N + V))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("pad", [1, 3, 8, 101])
def test_rows_apart_and_ragged_chains(draft, pad, dtype):
    print("[case] ragged", pad, draft, dtype, flush=True)
    tokens, p, q, u = make(9, 6, 1003, dtype, draft, seed=pad, pad=pad)
    check(tokens, p, q, u, nodes=[6, 1, 2, 5, 3, 0, 9, -4, 4])


@pytest.mark.parametrize("dtype", TYPES)
def test_uniforms_at_the_ends(dtype):
    print("[case] ends", dtype, flush=True)
    tokens, p, q, u = make(8, 4, 500, dtype, True, seed=3)
    u[:4] = 0.0
    u[4:] = 1.0 - 2.0 ** -24
    p[:, :, :3] = 0.0                              # the first tokens and the last have no mass
    p[:, :, -2:] = 0.0
    res = mpv.mpv_verify_chains(tokens, p, q, u)
    torch.cuda.synchronize()
    for b in range(8):
        a, bonus, *_ = so.verify_chain(tokens[b].tolist(), p[b].double().cpu().numpy(), q[b].double().cpu().numpy(), u[b].double().cpu().numpy())
        assert (int(res.accept_len[b]), int(res.bonus_token[b])) == (a, bonus)


@pytest.mark.parametrize("draft", [True, False])
def test_tokens_out_of_range_and_rows_without_mass(draft):
    print("[case] bad rows", draft, flush=True)
    tokens, p, q, u = make(6, 4, 300, torch.float32, draft, seed=4)
    tokens[0, 1], tokens[1, 2], tokens[2, 1] = -1, 300, 2 ** 31 - 1
    p[3] = 0.0                                     # nothing to draw from
    if draft:
        p[4] = q[4] * 0.5                          # p - q has no mass
        u[4, 1] = 0.9
    p[5, :, 7] = float("nan")
    p[5, :, 8] = -1.0
    check(tokens, p, q, u)


def test_the_row_after_the_last_token_of_a_draft_is_not_read():
    print("[case] last draft row", flush=True)
    tokens, p, q, u = make(5, 4, 600, torch.float32, True, seed=5)
    u[:, 1:] = 0.0
    q[:, 3] = float("inf")
    res = check(tokens, p, q, u)
    assert res.accept_len.tolist() == [3] * 5


def test_many_draws_follow_the_target():
    """Emitted first tokens over many chains with the same rows: frequencies of the target's first row (5 standard deviations)."""
    print("[case] frequencies", flush=True)
    B, V = 20000, 6
    gen = torch.Generator(device="cuda")
    gen.manual_seed(6)
    pt = torch.tensor([0.05, 0.3, 0.2, 0.25, 0.15, 0.05], device="cuda")
    qd = torch.tensor([0.3, 0.1, 0.2, 0.05, 0.05, 0.3], device="cuda")
    p, q = pt.expand(B, 2, V).contiguous(), qd.expand(B, 2, V).contiguous()
    tokens = torch.zeros(B, 2, dtype=torch.int32, device="cuda")
    tokens[:, 1] = torch.multinomial(qd.expand(B, V), 1, generator=gen).squeeze(1).to(torch.int32)
    res = mpv.mpv_verify_chains(tokens, p, q, torch.rand(B, 2, generator=gen, device="cuda"))
    first = torch.where(res.accept_len > 0, res.path_tokens[:, 0], res.bonus_token).long()
    freq = torch.bincount(first, minlength=V).double() / B
    assert ((freq - pt.double()).abs() < 5 * (pt.double() * (1 - pt.double()) / B).sqrt()).all()


def test_captured_and_replayed():
    print("[case] graph", flush=True)
    tokens, p, q, u = make(24, 5, 4001, torch.float32, True, seed=7)
    kept = mpv.mpv_verify_chains(tokens, p, q, u)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mpv.mpv_verify_chains(tokens, p, q, u, out=kept)
    for seed in (8, 9, 10):
        t2, p2, q2, u2 = make(24, 5, 4001, torch.float32, True, seed=seed)
        tokens.copy_(t2); p.copy_(p2); q.copy_(q2); u.copy_(u2)
        eager = mpv.mpv_verify_chains(tokens, p, q, u)
        graph.replay()
        torch.cuda.synchronize()
        for name in ("accept_len", "path_nodes", "path_tokens", "bonus_token", "counters"):
            assert torch.equal(getattr(kept, name), getattr(eager, name)), name
        check(tokens, p, q, u, res=kept)


def test_what_is_used_on_another_stream_is_not_given_away_before_it_is_done():
    print("[case] another stream", flush=True)
    tokens, p, q, u = make(4, 5, 32000, torch.float32)
    want = check(tokens, p, q, u)
    side = torch.cuda.Stream()
    busy = torch.zeros(64 << 20, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(600):                       # some 60 ms, in which the allocator has to wait
            busy += 1.0
    res = mpv.mpv_verify_chains(tokens, p, q, u, stream=side)
    places = {t.data_ptr() for t in (res.workspace, res.path_nodes, res.bonus_token)}
    sizes = res.workspace.numel()
    assert len(places) == 3 and not side.query()
    held = res.bonus_token
    del res
    new = [torch.empty(sizes, dtype=torch.uint8, device="cuda") for _ in range(8)] + [torch.empty_like(want.path_nodes) for _ in range(8)]
    assert not side.query() and not places & {t.data_ptr() for t in new}
    torch.cuda.synchronize()
    assert torch.equal(held, want.bonus_token)
