"""As test_gpu_serving_streams.py, for the verification and the calls that belong to it (needs an MI355X)."""

import pytest
import torch

import paper_2602_16994_amd as mpv
from tests.test_gpu_serving_streams import keep_busy

pytestmark = pytest.mark.gpu

PARENT = mpv.delayed_tree(3, 1, 2)


def calls():
    """Each returns (results, workspace or None)."""
    B, N, V = 6, len(PARENT), 2000
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    target, draft = (torch.randn(B, N, V, generator=gen, device="cuda") for _ in range(2))
    tokens = torch.randint(0, V, (B, N), generator=gen, device="cuda", dtype=torch.int32)
    u = torch.rand(B, N, generator=gen, device="cuda")

    def verify(**kw):
        r = mpv.mpv_verify(PARENT, tokens, target, draft, 1.0, u, mpv.MPV_METHOD_TRAVERSAL, **kw)
        return (r.accept_len, r.path_nodes, r.path_tokens, r.bonus_token), r.workspace

    def efficiency(**kw):
        r = mpv.mpv_block_efficiency(PARENT, tokens, target, draft, 1.0, mpv.MPV_METHOD_SPECINFER, **kw)
        return (r.expected, r.reach_prob), r.workspace

    return {
        "verify": verify,
        "efficiency": efficiency,
        "rates": lambda **kw: (mpv.mpv_acceptance_rates(PARENT, target, draft, 1.0, mpv.MPV_METHOD_SPECINFER, **kw)[:1], None),
        "nucleus": lambda **kw: (mpv.mpv_nucleus_mask(target, 1.0, 0.9, **kw), None),
        "stats": lambda **kw: ((mpv.mpv_row_stats(target.view(-1, V), 1.0, **kw),), None),
        "uniforms": lambda **kw: ((mpv.mpv_fill_uniforms(5, 3000, **kw),), None),
    }


KINDS = ["verify", "efficiency", "rates", "nucleus", "stats", "uniforms"]


@pytest.mark.parametrize("kind", KINDS)
def test_what_is_allocated_is_not_still_in_use_on_the_current_stream(kind):
    print("[case] allocated for another stream", kind, flush=True)
    call = calls()[kind]
    want, workspace = call()
    side, here = torch.cuda.Stream(), torch.cuda.current_stream()
    busy = torch.zeros(64 << 20, device="cuda")
    torch.cuda.synchronize()
    keep_busy(here, busy)
    given_back = [torch.empty_like(t) for t in (*want, workspace) if t is not None for _ in range(64)]
    for t in given_back:
        t.zero_()                                  # waits for the busy stream; the allocator has the memory back before that
    taken = {t.data_ptr() for t in given_back}
    del given_back, t
    got, own = call(stream=side)
    assert not here.query() and not taken & {t.data_ptr() for t in (*got, own) if t is not None}
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("kind", KINDS)
def test_what_was_returned_is_not_given_away_while_the_current_stream_reads_it(kind):
    print("[case] returned from another stream", kind, flush=True)
    call = calls()[kind]
    side, here = torch.cuda.Stream(), torch.cuda.current_stream()
    busy = torch.zeros(64 << 20, device="cuda")
    torch.cuda.synchronize()
    got, _ = call(stream=side)
    here.wait_stream(side)
    keep_busy(here, busy)
    copies = [t.clone() for t in got]
    first = {t.data_ptr() for t in got}
    del got, _
    others = [call(stream=side) for _ in range(4)]
    assert not here.query()
    for other, _ in others:
        assert not first & {t.data_ptr() for t in other}
    torch.cuda.synchronize()
    for a, b in zip(copies, others[0][0]):
        assert torch.equal(a, b)
