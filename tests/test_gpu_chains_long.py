"""mpv_verify_chains on the rows and batches of a server (needs an MI355X): one workgroup a chain on rows of many rounds, parts of a
row that are several rounds long, and the draw from a row whose parts have no mass.  Tolerances as in test_gpu_chains.py: none."""

import pytest
import torch

import paper_2602_16994_amd as mpv
from tests.test_gpu_chains import TYPES, check, make

pytestmark = pytest.mark.gpu

# One workgroup a chain (without a draft from 144 chains on, with one from 192, or 240 of long rows): a wave's share of a row takes several
# rounds of four loads a lane (20 011: some lanes one, most two), and the share that is drawn from several groups of 16 bytes a lane (from
# 65 536 tokens of 4 bytes, 131 072 of 2 on).  Several a chain: parts of 8016 and of 10 856 tokens, of which the same holds.
SIZES = [(192, 3, 20011), (192, 2, 151937), (128, 2, 128256), (150, 2, 151937), (240, 3, 20011), (241, 2, 151937)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("B,N,V", SIZES)
def test_long_rows(B, N, V, draft, dtype):
    print("[case] long rows", B, N, V, draft, dtype, flush=True)
    check(*make(B, N, V, dtype, draft, seed=B + N + V))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("B", [9, 143, 144, 195, 239, 240])
def test_long_rows_apart_and_ragged_chains(B, draft, dtype):
    print("[case] long and ragged", B, draft, dtype, flush=True)
    tokens, p, q, u = make(B, 4, 9001, dtype, draft, seed=B, pad=5)
    check(tokens, p, q, u, nodes=[(4, 1, 2, 0, 9, -4, 3)[b % 7] for b in range(B)])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("B,V", [(6, 8191), (6, 32001), (192, 9001), (250, 9001)])
def test_tokens_out_of_range_and_long_rows_without_mass(B, V, draft, dtype):
    print("[case] long bad rows", B, V, draft, dtype, flush=True)
    tokens, p, q, u = make(B, 4, V, dtype, draft, seed=4)
    tokens[0, 1], tokens[1, 2], tokens[2, 1] = -1, V, 2 ** 31 - 1
    p[3] = 0.0                                     # nothing to draw from
    if draft:
        p[4] = q[4] * 0.5                          # p - q has no mass
        u[4, 1] = 0.9
    p[5, :, 7] = float("nan")
    p[5, :, 8] = -1.0
    check(tokens, p, q, u)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("u0", [0.0, 1.0 - 2.0 ** -24])
@pytest.mark.parametrize("B,V", [(6, 8191), (6, 32001), (192, 9001), (250, 9001)])
def test_long_rows_and_uniforms_at_the_ends(B, V, u0, dtype):
    print("[case] long ends", B, V, u0, dtype, flush=True)
    tokens, p, q, u = make(B, 3, V, dtype, True, seed=3)
    u[:, 0] = u0
    p[:, :, :2100] = 0.0                           # the first tokens and the last have no mass: a whole part of them
    p[:, :, -2100:] = 0.0
    check(tokens, p, q, u)


@pytest.mark.parametrize("B,V", [(6, 32001), (192, 9001), (250, 9001)])
def test_a_row_whose_mass_is_one_token(B, V):
    print("[case] one token", B, V, flush=True)
    tokens, p, q, u = make(B, 2, V, torch.float32, False, seed=5)
    where = [(b * 7919) % V for b in range(B)]
    where[0], where[1] = 0, V - 1
    p.zero_()
    for b in range(B):
        p[b, :, where[b]] = 1e-30 if b % 2 else 1.0
    u[:, 1] = 1.0 - 2.0 ** -24
    tokens[:, 1] = torch.tensor([(w + 1) % V for w in where], dtype=torch.int32, device="cuda")
    res = check(tokens, p, None, u)
    assert res.bonus_token.tolist() == where and res.accept_len.tolist() == [0] * B
