"""Memory of calls that run on another stream than the current one (needs an MI355X): what such a call allocates is not in use by
earlier work of the current stream, and what it returned is not given away while the current stream still reads it.  Told from the
addresses, while the stream in question is kept busy."""

import pytest
import torch

import paper_2602_16994_amd as mpv
from tests.test_gpu_chains import make as make_chains
from tests.test_gpu_tree_attention import DELAYED15, Case

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def tables():
    """Two requests, 3 and 16 cached tokens in pages of 16, four free pages."""
    return dict(block_table=i32([[4, -1, -1], [5, -1, -1]]), context_len=i32([3, 16]), new_len=i32([2, 1]), free_pages=i32([0, 1, 2, 3, -1, -1]),
                free_count=i32([4]), page_size=16, slot_map=torch.full((2, 4), -7, dtype=torch.int64, device="cuda"))


def calls():
    tokens, p, q, u = make_chains(4, 5, 32000, torch.float32)
    case = Case(4, DELAYED15, 8, 2, 128, torch.bfloat16, [3000, 5, 900, 64], 16, seed=1)
    rows = tables()

    def extend(**kw):                              # (the tables themselves are changed by the call: each has its own, made beforehand)
        return mpv.mpv_extend_tables(**(rows if "stream" in kw else tables()), **kw)

    return {
        "attention": (lambda **kw: case.run(**kw), ("out",)),
        "chains": (lambda **kw: mpv.mpv_verify_chains(tokens, p, q, u, **kw), ("accept_len", "path_nodes", "path_tokens", "bonus_token", "counters")),
        "tables": (extend, ("context_len", "free_count", "granted", "offsets")),
    }


def keep_busy(stream, buffer):
    with torch.cuda.stream(stream):
        for _ in range(1500):                      # some 160 ms
            buffer += 1.0


def places(res, names):
    return {getattr(res, n).data_ptr() for n in names}


@pytest.mark.parametrize("kind", ["attention", "chains", "tables"])
def test_what_is_allocated_is_not_still_in_use_on_the_current_stream(kind):
    print("[case] allocated for another stream", kind, flush=True)
    call, names = calls()[kind]
    want = call()
    side, here = torch.cuda.Stream(), torch.cuda.current_stream()
    busy = torch.zeros(64 << 20, device="cuda")
    torch.cuda.synchronize()
    keep_busy(here, busy)
    given_back = [torch.empty_like(getattr(want, n)) for n in (*names, "workspace") for _ in range(64)]
    for t in given_back:
        t.zero_()                                  # waits for the busy stream; the allocator has the memory back before that
    taken = {t.data_ptr() for t in given_back}
    del given_back, t
    res = call(stream=side)
    assert not here.query() and not taken & places(res, (*names, "workspace"))
    torch.cuda.synchronize()
    for n in names:
        assert torch.equal(getattr(res, n), getattr(want, n)), n


@pytest.mark.parametrize("kind", ["attention", "chains"])
def test_what_was_returned_is_not_given_away_while_the_current_stream_reads_it(kind):
    print("[case] returned from another stream", kind, flush=True)
    call, names = calls()[kind]
    side, here = torch.cuda.Stream(), torch.cuda.current_stream()
    busy = torch.zeros(64 << 20, device="cuda")
    torch.cuda.synchronize()
    res = call(stream=side)
    here.wait_stream(side)
    keep_busy(here, busy)
    copies = [getattr(res, n).clone() for n in names]
    first = places(res, names)
    del res
    others = [call(stream=side) for _ in range(4)]
    assert not here.query()
    for other in others:
        assert not first & places(other, names)
    torch.cuda.synchronize()
    for n, c in zip(names, copies):
        assert torch.equal(c, getattr(others[0], n)), n


def test_a_workspace_that_is_used_on_another_stream_than_its_own():
    print("[case] a workspace on two streams", flush=True)
    call, names = calls()["chains"]
    side, here = torch.cuda.Stream(), torch.cuda.current_stream()
    busy = torch.zeros(64 << 20, device="cuda")
    torch.cuda.synchronize()
    want = call()
    res = call(stream=side)
    here.wait_stream(side)
    keep_busy(here, busy)
    res = call(out=res)                            # the same buffers, on the current stream
    ws = res.workspace.data_ptr()
    del res
    with torch.cuda.stream(side):
        new = [torch.empty_like(want.workspace) for _ in range(4)]
    assert not here.query() and ws not in {t.data_ptr() for t in new}
    torch.cuda.synchronize()
