"""mpv_token_logprobs where logits are large, against the definition in 64 bits (needs an MI355X).

What counts are differences z - max z, so no bound contains the size of the logits.  With e = 2^-24, y = (max z - z) / T of a token, p its
probability, and terms of a sum that are added up by lane, wave and part:
  an exponent c (z - m): the difference, the factor c, their product (or one fma): 3 e relative; an exponential 2 e; references that a term passes on
  its way add up to its distance from the maximum, each with an exponential and two more roundings: the sum's relative error is at most
      (3 E[y] + V / 256 + 64) e,   E[y] = sum p y <= entropy;
  a log probability: difference, factor, product, the sum's logarithm (|ln S| <= ln V, 4 e), the last difference; |y| <= |ln p| + ln V:
      (4 |ln p| + 8 ln V + 3 E[y] + V / 256 + 64) e;
  the entropy: that of ln S, and the quotient E[y], whose terms have one sign and relative errors of 3 e y + 3 e and the sum's:
      (8 ln V + 4 H + 4 E[y^2] + (V / 256 + 64) (2 + E[y])) e.
Whole numbers are exact.
"""

import numpy as np
import pytest
import torch

import paper_2602_16994_amd as mpv
from oracle import logprobs_oracle as lo

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16, torch.float32]


def near(mine, want, tol):
    with np.errstate(over="ignore"):
        want32 = np.float32(want)                  # (what lies beyond float32 is infinite there)
    return mine == want32 or (np.isnan(mine) and np.isnan(want32)) or abs(float(mine) - want) <= tol


def check(logits, tokens, T=1.0, top=0):
    r = mpv.mpv_token_logprobs(logits, tokens, temperature=T, top=top)
    z, t = logits.double().cpu().numpy(), tokens.cpu().numpy()
    V, e, worst = z.shape[2], 2.0 ** -24, 0.0
    lnV = np.log(V)
    for b in range(t.shape[0]):
        for n in range(t.shape[1]):
            logprob, entropy, rank, best, best_logprobs = lo.row(z[b, n], int(t[b, n]), T, top)
            y = (z[b, n].max() - z[b, n]) / T
            p = np.exp(-y)
            p /= p.sum()
            y = np.where(p > 0, y, 0.0)
            first, second, sums = float((p * y).sum()), float((p * y * y).sum()), V / 256 + 64
            assert int(r.rank[b, n]) == rank
            assert r.top_tokens[b, n].tolist() == list(best)
            for mine, want in [(float(r.logprob[b, n]), logprob), *zip(r.top_logprobs[b, n].tolist(), best_logprobs)]:
                tol = (4 * abs(want) + 8 * lnV + 3 * first + sums) * e
                assert near(mine, want, tol), (b, n, mine, want, tol)
                if np.isfinite(want) and np.isfinite(mine):
                    worst = max(worst, abs(mine - want) / tol)
            tol = (8 * lnV + 4 * entropy + 4 * second + sums * (2 + first)) * e
            assert near(float(r.entropy[b, n]), entropy, tol), (b, n, float(r.entropy[b, n]), entropy, tol)
            worst = max(worst, abs(float(r.entropy[b, n]) - entropy) / tol)
    print("[largest error over its bound] %.3f" % worst, flush=True)
    return r


def random(B, N, V, seed, sigma=2.5):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return torch.randn(B, N, V, generator=gen, device="cuda") * sigma, torch.randint(0, V, (B, N), generator=gen, device="cuda").to(torch.int32)


SIZES = [1e3, 5e3, 6e4, 1e6, 1e9, 1e12, 3e15]


def sizes_of(dtype):
    return [x for x in SIZES if x <= torch.finfo(dtype).max]


@pytest.mark.parametrize("T", [0.1, 1.0])
@pytest.mark.parametrize("dtype", TYPES)
def test_a_forced_token(dtype, T):
    """One logit far above the others: its log probability is 0, those of the others are their distances."""
    print("[case] logprobs forced", dtype, T, flush=True)
    for i, size in enumerate(sizes_of(dtype)):
        logits, tokens = random(2, 2, 9001, i)
        tokens[0, 0], tokens[1, 0] = 77, 8999
        logits[:, 0, 77] = size
        logits[:, 1, 8999] = size
        check(logits.to(dtype), tokens, T, 5)


@pytest.mark.parametrize("T", [0.1, 1.0])
@pytest.mark.parametrize("dtype", TYPES)
def test_rows_of_one_large_number(dtype, T):
    """A row that a mask of -1e9 covers whole is uniform, and so is one of +1e9."""
    print("[case] logprobs masked with a number", dtype, T, flush=True)
    for size in sizes_of(dtype):
        for V in (100, 32768):
            logits = torch.full((1, 2, V), size, device="cuda")
            logits[0, 0] = -size
            r = check(logits.to(dtype), torch.tensor([[3, V - 1]], dtype=torch.int32, device="cuda"), T, 3)
            assert torch.allclose(r.logprob.double().cpu(), torch.full((1, 2), -np.log(V), dtype=torch.float64), rtol=0, atol=1e-4)


@pytest.mark.parametrize("T", [0.1, 1.0])
@pytest.mark.parametrize("dtype", TYPES)
def test_one_offset_for_all(dtype, T):
    """Rows a long way from zero, with the differences that their type has there."""
    print("[case] logprobs offset", dtype, T, flush=True)
    for i, size in enumerate(sizes_of(dtype)):
        logits, tokens = random(1, 2, 32768, 20 + i, sigma=2.5 + 3 * size * torch.finfo(dtype).eps)
        logits[0, 0] += 0.9 * size
        logits[0, 1] -= 0.9 * size
        check(logits.to(dtype), tokens, T, 9)


@pytest.mark.parametrize("T", [0.1, 1.0])
def test_the_same_row_elsewhere(T):
    """Multiples of 1/4 with an offset that float32 holds with them: the same results."""
    print("[case] logprobs shifted", T, flush=True)
    logits, tokens = random(1, 3, 40000, 40)
    logits = (logits * 4).round() / 4
    here = check(logits, tokens, T, 6)
    for offset in (1024.0, -4096.0, 65536.0, -1048576.0):
        there = check(logits + offset, tokens, T, 6)
        assert torch.equal(here.rank, there.rank) and torch.equal(here.top_tokens, there.top_tokens)
        for a, b in ((here.logprob, there.logprob), (here.top_logprobs, there.top_logprobs), (here.entropy, there.entropy)):
            assert torch.allclose(a, b, rtol=0, atol=1e-4)


@pytest.mark.parametrize("dtype", TYPES)
def test_large_and_small_numbers_in_turn(dtype):
    """References move from far below to far above, in lanes, waves and parts of a row."""
    print("[case] logprobs moving references", dtype, flush=True)
    logits, tokens = random(2, 3, 70001, 50)
    size = min(1e9, 0.9 * torch.finfo(dtype).max)
    logits[0, 0, ::2] = -size
    logits[0, 1, 64:60000] = -size
    logits[0, 2, :69990] = -size
    logits[1, 0] += 0.01 * size * torch.arange(70001, device="cuda") / 70001
    logits[1, 1, 30000:] += 5000.0
    logits[1, 2, :30000] += 5000.0
    tokens[0, 2] = 69995
    check(logits.to(dtype), tokens, 1.0, 7)


@pytest.mark.parametrize("T", [0.5, 1.0, 3.0])
@pytest.mark.parametrize("dtype", TYPES)
def test_masks_of_the_lowest_number(dtype, T):
    """The lowest number of the type as a mask, with logits of ordinary size beside it: in the same lane, round, wave and part, and in others."""
    print("[case] logprobs lowest number", dtype, T, flush=True)
    low = torch.finfo(dtype).min
    for V in (9, 100, 2048, 8192, 70001):
        logits, tokens = random(8, 2, V, V)
        seen = torch.zeros(8, 2, V, dtype=torch.bool, device="cuda")
        at = torch.arange(V, device="cuda")
        seen[0, 0, -8:] = True                     # the last tokens
        seen[0, 1, :8] = True                      # the first
        seen[1, 0] = at % 997 == 5                 # few, far apart
        seen[1, 1] = at % 2 == 1
        seen[2, 0] = at >= V // 2
        seen[2, 1] = at < V // 2
        seen[3, 0] = at // 64 % 3 == 2             # segments
        seen[3, 1] = at // 8 % 2 == 1              # a lane's loads
        seen[4, 0] = at // 2048 % 2 == 1           # rounds of a lane
        seen[4, 1] = at // 512 % 5 == 3            # waves
        seen[5, 0] = at // 32768 % 2 == 1          # parts
        seen[5, 1] = at // 8192 % 2 == 1
        seen[6, 0, V // 3] = True                  # one alone
        seen[6, 1] = at % 64 == 63
        seen[7, 0] = at != V // 2                  # all but one
        seen[7, 1] = at >= V - 1
        seen[:, :, 5] |= ~seen.any(dim=2)
        logits = torch.where(seen, logits, low).to(dtype)
        check(logits, seen.int().argmax(dim=2).to(torch.int32), T, 1)


@pytest.mark.parametrize("T", [0.5, 1.0, 3.0, 1e30, 3e38])
@pytest.mark.parametrize("dtype", TYPES)
def test_log_probabilities_of_masked_tokens(dtype, T):
    """A token with the lowest number has a log probability, as long as float32 holds it; with a high temperature it is not small."""
    print("[case] logprobs of masked tokens", dtype, T, flush=True)
    low, high = torch.finfo(dtype).min, torch.finfo(dtype).max
    logits, tokens = random(2, 3, 5000, 60)
    logits[0, 0, 20:] = low
    logits[0, 1, :4990] = low
    logits[0, 2] = low
    logits[1, 0, ::2] = low
    logits[1, 1, ::3], logits[1, 1, 1::3] = low, high
    logits[1, 2, 17], logits[1, 2, 18] = low, high
    tokens[0, 0], tokens[0, 1], tokens[0, 2], tokens[1, 0], tokens[1, 1], tokens[1, 2] = 30, 7, 4999, 2, 3, 17
    check(logits.to(dtype), tokens, T, 40)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_the_lowest_temperature(dtype):
    print("[case] logprobs lowest temperature", dtype, flush=True)
    logits, tokens = random(2, 2, 3000, 61)
    logits[0] *= 1e-37
    tokens[1, 0] = int(logits[1, 0].argmax())
    check(logits.to(dtype), tokens, 2.0 ** -126, 5)
