"""mpv_token_logprobs against the definition in 64 bits (needs an MI355X).

With e = 2^-24, c = log2(e) / T and R the largest |c (z - max z)| of a token whose probability is above 2^-40 (the others add nothing of note):
  a log probability: the exponent's rounding (the product's factor c, the reference, the difference), and the sum's relative error,
  of V terms added by lane, wave and part, an exponential each:      (8 (|log2 p| + R) + 4 |c max z| 2 + V / 256 + 64) e
(the reference's rounding falls out of differences of exponents, but an exponent c z - m is rounded by its own size, and c z by none: fma.)
  the entropy: the logarithm of the sum as above, and the weighted sum, each of whose terms has a relative error of the same kind;
  its terms add up to at most R plus the entropy:                    twice that, times (1 + R)
Whole numbers are exact.
"""

import numpy as np
import pytest
import torch

import paper_2602_16994_amd as mpv
from oracle import logprobs_oracle as lo

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16, torch.float32]


def check_row(z, token, T, top, got, i):
    """got: numpy arrays of a LogprobsResult, flattened to rows."""
    logprob, entropy, rank, tokens, logprobs = lo.row(z, token, T, top)
    e, V = 2.0 ** -24, len(z)
    finite = z[np.isfinite(z)]
    big = float(np.abs(finite).max()) / T * 1.4427 if finite.size else 0.0
    R = 40.0
    tol = lambda lp: (8 * (abs(lp) * 1.4427 + R) + 8 * big + V / 256 + 64) * e  # noqa: E731
    assert got["rank"][i] == rank
    assert list(got["top_tokens"][i]) == list(tokens)
    for mine, want in [(got["logprob"][i], logprob), *zip(got["top_logprobs"][i], logprobs)]:
        assert (np.isnan(mine) and np.isnan(want)) or mine == want or abs(mine - want) <= tol(want), (mine, want)
    mine = got["entropy"][i]
    assert (np.isnan(mine) and np.isnan(entropy)) or abs(mine - entropy) <= 2 * tol(entropy) * (1 + R), (mine, entropy)


def numbers(r):
    flat = {k: getattr(r, k).cpu().numpy() for k in ("logprob", "entropy", "rank", "top_tokens", "top_logprobs")}
    return {k: v.reshape(v.shape[0] * v.shape[1], v.shape[2]) if k.startswith("top") else v.reshape(-1) for k, v in flat.items()}


def missing(got, i):
    assert got["logprob"][i] == 0.0 and got["entropy"][i] == 0.0 and got["rank"][i] == -1
    assert (got["top_tokens"][i] == -1).all() and (got["top_logprobs"][i] == -np.inf).all()


def check_rows(logits, tokens, T=1.0, top=0, nodes=None, **kw):
    r = mpv.mpv_token_logprobs(logits, tokens, temperature=T, top=top, num_nodes=nodes, **kw)
    got, z, t = numbers(r), logits.double().cpu().numpy(), tokens.cpu().numpy()
    B, N = t.shape
    for b in range(B):
        for n in range(N):
            if nodes is not None and n >= int(nodes[b]):
                missing(got, b * N + n)
            else:
                check_row(z[b, n], int(t[b, n]), T, top, got, b * N + n)
    return r


def random(B, N, V, dtype, seed, sigma=2.5):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    logits = (torch.randn(B, N, V, generator=gen, device="cuda") * sigma).to(dtype)
    tokens = torch.randint(0, V, (B, N), generator=gen, device="cuda").to(torch.int32)
    best = logits.argmax(dim=-1).to(torch.int32)
    return logits, torch.where(torch.rand(B, N, generator=gen, device="cuda") < 0.5, best, tokens)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,N,V,top,T", [
    (1, 1, 1, 1, 1.0), (1, 1, 2, 5, 1.0), (2, 3, 7, 3, 0.5), (1, 2, 63, 64, 1.0), (3, 1, 64, 1, 2.0), (1, 3, 65, 20, 1.0), (2, 2, 1000, 0, 0.7),
    (1, 1, 8193, 8, 1.0), (4, 5, 32000, 5, 1.0), (1, 2, 50257, 64, 1.3), (2, 1, 151936, 20, 0.1), (1, 1, 262147, 7, 1.0), (700, 2, 515, 4, 1.0),
    (2, 2, 1969, 64, 1.0), (1, 2, 4096, 63, 1.0), (1, 1, 300, 2, 1.0), (1, 1, 161, 64, 1.0), (1, 1, 160, 64, 1.0),
])
def test_rows(B, N, V, top, T, dtype):
    print("[case] logprobs rows", B, N, V, top, T, dtype, flush=True)
    logits, tokens = random(B, N, V, dtype, V + top)
    check_rows(logits, tokens, T, top)


def test_the_largest_vocabulary():
    print("[case] logprobs 2^21", flush=True)
    logits, tokens = random(1, 1, 1 << 21, torch.bfloat16, 5)
    check_rows(logits, tokens, 1.0, 33)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("levels", [1, 2, 5])
def test_equal_logits(levels, dtype):
    """Whole rows of few values: of equal ones the lowest index comes first."""
    print("[case] logprobs ties", levels, dtype, flush=True)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(levels)
    logits = torch.randint(0, levels, (3, 2, 5001), generator=gen, device="cuda").to(dtype)
    tokens = torch.tensor([[0, 5000], [2500, 64], [1, 4999]], dtype=torch.int32, device="cuda")
    check_rows(logits, tokens, 1.0, 64)
    check_rows(logits, tokens, 1.0, 1)


@pytest.mark.parametrize("dtype", TYPES)
def test_masked_tokens(dtype):
    """-inf almost everywhere, in whole parts of a row, and everywhere."""
    print("[case] logprobs masks", dtype, flush=True)
    logits, tokens = random(4, 2, 70001, dtype, 6)
    logits[0, 0, 40:] = -float("inf")
    logits[0, 1, :70000] = -float("inf")
    logits[1, 0] = -float("inf")
    logits[1, 1, 100:60000] = -float("inf")
    logits[2, 0, ::2] = -float("inf")
    logits[2, 1] = torch.finfo(dtype).min
    logits[3, 0, 5:] = -float("inf")
    tokens[3, 0] = 70000
    tokens[0, 0] = 3
    check_rows(logits, tokens, 1.0, 50)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("seen,top", [(1300, 64), (1300, 20), (1025, 17), (4000, 63)])
def test_few_segments_with_many_tokens(seen, top, dtype):
    """Fewer segments of 64 tokens than alternatives, but more tokens than are put in order at once; equal ones among them."""
    print("[case] logprobs few segments", seen, top, dtype, flush=True)
    logits, tokens = random(2, 1, 70001, dtype, seen)
    logits[:, :, seen:] = -float("inf")
    logits[1, :, :seen] = 1.5
    check_rows(logits, tokens, 1.0, top)


@pytest.mark.parametrize("dtype", TYPES)
def test_values_that_are_no_numbers(dtype):
    print("[case] logprobs nan", dtype, flush=True)
    logits, tokens = random(2, 2, 20000, dtype, 7)
    logits[0, 0, 19999] = float("nan")
    logits[0, 1, 7] = float("inf")
    logits[1, 0, 123] = -float("nan")
    check_rows(logits, tokens, 1.0, 3)


def test_tokens_that_are_none_and_rows_that_are_not_there():
    print("[case] logprobs missing", flush=True)
    logits, tokens = random(3, 4, 999, torch.bfloat16, 8)
    tokens[0, 0], tokens[1, 1], tokens[2, 0] = -1, 999, 1 << 30
    check_rows(logits, tokens, 1.0, 2, nodes=torch.tensor([4, 2, 0], dtype=torch.int32, device="cuda"))


def test_zeros_of_both_signs_are_equal():
    print("[case] logprobs zeros", flush=True)
    logits = torch.zeros(1, 1, 300, device="cuda")
    logits[0, 0, ::3] = -0.0
    check_rows(logits, torch.tensor([[7]], dtype=torch.int32, device="cuda"), 1.0, 10)


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_further_apart_and_at_odd_addresses(dtype):
    print("[case] logprobs strides", dtype, flush=True)
    wide, tokens = random(2, 3, 1237, dtype, 9)
    check_rows(wide[:, :, 1:1102], tokens.clamp(max=1100), 1.0, 5)


@pytest.mark.parametrize("dtype", TYPES)
def test_paths(dtype):
    print("[case] logprobs paths", dtype, flush=True)
    B, N, V, deep, top = 5, 9, 3001, 4, 6
    logits, _ = random(B, N, V, dtype, 10)
    accept = torch.tensor([0, 4, 2, 3, 9], dtype=torch.int32, device="cuda")       # (9: taken as 4)
    path = torch.tensor([[-1] * 4, [1, 3, 5, 8], [2, 7, -1, -1], [1, 9, 3, -1], [1, 2, 3, 4]], dtype=torch.int32, device="cuda")
    tokens = torch.randint(0, V, (B, deep), device="cuda").to(torch.int32)
    bonus = torch.randint(0, V, (B,), device="cuda").to(torch.int32)
    r = mpv.mpv_token_logprobs(logits, tokens, top=top, accept_len=accept, path_nodes=path, bonus_token=bonus)
    got, z = numbers(r), logits.double().cpu().numpy()
    for b in range(B):
        a = min(int(accept[b]), deep)
        for i in range(deep + 1):
            node = 0 if i == 0 else int(path[b, i - 1])
            if i > a or not 0 <= node < N:
                missing(got, b * (deep + 1) + i)
            else:
                check_row(z[b, node], int(bonus[b] if i == a else tokens[b, i]), 1.0, top, got, b * (deep + 1) + i)


def test_after_a_verification():
    """The emitted tokens of mpv_verify, eagerly and replayed from a graph with other inputs."""
    print("[case] logprobs after a verification", flush=True)
    import workloads
    cfg = workloads.Config("logprobs", B=6, V=2003, K=3, L1=1, L2=2, dtype="bf16", T=0.8, methods=[1], draft_sigma=2.0, target_sigma=1.0, seed=3)
    x = workloads.make_inputs(cfg, "cuda")

    def step(res=None, out=None):
        res = mpv.mpv_verify(x["parent"], x["tokens"], x["target"], x["draft"], cfg.T, x["uniforms"], mpv.MPV_METHOD_TRAVERSAL, out=res)
        return res, mpv.mpv_token_logprobs(x["target"], res.path_tokens, temperature=cfg.T, top=4, accept_len=res.accept_len,
                                           path_nodes=res.path_nodes, bonus_token=res.bonus_token, out=out)

    res, out = step()
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        step(res, out)
    for seed in range(3):
        x["uniforms"].copy_(torch.rand(x["uniforms"].shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)))
        x["target"].copy_(x["target"].roll(1, dims=2))
        want_res, want = step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got, z = numbers(out), x["target"].double().cpu().numpy()
        for k, v in numbers(want).items():
            assert np.array_equal(v, got[k]), k
        a = want_res.accept_len.tolist()
        for b in range(cfg.B):
            assert (got["rank"].reshape(cfg.B, -1)[b, :a[b] + 1] > 0).all()
            row = 0 if a[b] == 0 else int(want_res.path_nodes[b, a[b] - 1])
            width = want_res.path_nodes.shape[1] + 1
            check_row(z[b, row], int(want_res.bonus_token[b]), cfg.T, 4, got, b * width + a[b])


def test_an_empty_batch():
    print("[case] logprobs empty", flush=True)
    r = mpv.mpv_token_logprobs(torch.zeros(0, 3, 10, device="cuda"), torch.zeros(0, 3, dtype=torch.int32, device="cuda"), top=2)
    assert r.top_tokens.shape == (0, 3, 2)
