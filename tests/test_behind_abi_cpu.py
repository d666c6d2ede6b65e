"""What attention behind prefixes, log probabilities, scores and eviction refuse, before anything is launched (no GPU needed)."""

import ctypes

import pytest
import torch

import paper_2602_16994_amd as mpv
from paper_2602_16994_amd import binding as bd
from tests.test_abi_cpu import code
from tests.test_serving_abi_cpu import FAKE, attention, filled

WITHOUT_WORKSPACE = ("mpv_score_positions",)


@pytest.fixture(scope="module")
def lib():
    return mpv.load_library()


def refusals(lib, name, shape, buffers, cases):
    """cases: (fields of the shape, fields of the buffers, error)."""
    call = getattr(lib, name)
    for fields, bufs, error in cases:
        s, b = shape(**fields), buffers(**bufs)
        rest = (None,) if name in WITHOUT_WORKSPACE else (FAKE, 1 << 40, None)
        got = call(ctypes.byref(s), ctypes.byref(b), *rest)
        assert got == (code(error) if error else 0), (fields, bufs, error, got)


def workspaces(lib, name, s, b):
    call = getattr(lib, name)
    assert call(ctypes.byref(s), ctypes.byref(b), None, 1 << 40, None) == code("MPV_ERR_WORKSPACE")
    assert call(ctypes.byref(s), ctypes.byref(b), FAKE + 8, 1 << 40, None) == code("MPV_ERR_WORKSPACE")
    assert call(ctypes.byref(s), ctypes.byref(b), FAKE, 16, None) == code("MPV_ERR_WORKSPACE")
    assert call(ctypes.byref(s), None, FAKE, 1 << 40, None) == code("MPV_ERR_NULL")
    assert call(None, ctypes.byref(b), FAKE, 1 << 40, None) == code("MPV_ERR_NULL")
    assert getattr(lib, name + "_workspace_bytes")(ctypes.byref(s), None) == code("MPV_ERR_NULL")


def test_prefix_attention(lib):
    def shape(prefixes=2, prefix_width=3, **over):
        a = attention(**over)
        s = bd._Prefixed(a, prefixes, prefix_width)
        s._keepalive = a
        return s

    def bufs(prefix_of=FAKE, prefix_table=FAKE, prefix_len=FAKE, lse=FAKE, **over):
        return bd._PrefixedBuffers(filled(bd._AttentionBuffers, **{"num_nodes": None, "tree_parent": None, **over}), prefix_of, prefix_table,
                                   prefix_len, lse)

    refusals(lib, "mpv_prefix_attention", shape, bufs, [
        ({"B": -1}, {}, "MPV_ERR_BAD_SHAPE"), ({"prefixes": -1}, {}, "MPV_ERR_BAD_SHAPE"), ({"prefix_width": -1}, {}, "MPV_ERR_BAD_SHAPE"),
        ({"heads": 3}, {}, "MPV_ERR_BAD_SHAPE"), ({"dtype": 3}, {}, "MPV_ERR_BAD_DTYPE"), ({"scale": float("nan")}, {}, "MPV_ERR_BAD_TEMPERATURE"),
        ({"prefix_width": 1 << 28}, {}, "MPV_ERR_UNSUPPORTED"), ({"N": 65}, {}, "MPV_ERR_UNSUPPORTED"), ({"head_dim": 60}, {}, "MPV_ERR_ALIGNMENT"),
        ({}, {"prefix_table": None}, "MPV_ERR_NULL"), ({}, {"prefix_len": None}, "MPV_ERR_NULL"), ({}, {"q": None}, "MPV_ERR_NULL"),
        ({"table_width": 0}, {"cache_k": None}, "MPV_ERR_NULL"), ({"table_width": 0}, {"cache_v": None}, "MPV_ERR_NULL"),
        ({}, {"out": None}, "MPV_ERR_NULL"), ({}, {"out": FAKE + 4}, "MPV_ERR_ALIGNMENT"), ({"parent": (0, 0, 0)}, {}, "MPV_ERR_BAD_TREE"),
        ({"parent": None}, {}, "MPV_ERR_NULL"), ({"B": 0}, {}, None),
    ])
    workspaces(lib, "mpv_prefix_attention", shape(), bufs())
    # sizes of every kernel and both ways of reading a prefix: each is at least what its rows' states take
    need = ctypes.c_size_t()
    for dtype in (0, 1, 2):
        for D in (64, 128, 256):
            for N in (1, 3, 20, 64):
                for B, width in ((1, 4), (2, 4), (64, 100000), (300, 100000)):
                    s = shape(prefix_width=width, B=B, N=N, parent=tuple(range(-1, N - 1)), dtype=dtype, head_dim=D, q_stride=4 * D, kv_stride=2 * D,
                              out_stride=4 * D, slot_stride=2 * D, page_stride=32 * D)
                    assert lib.mpv_prefix_attention_workspace_bytes(ctypes.byref(s), ctypes.byref(need)) == 0
                    assert 0 < need.value < 1 << 32 and need.value % 256 == 0
                    if N == 1 and B >= 64:
                        assert need.value >= B * 4 * (D + 2) * 4


def test_scores(lib):
    def shape(**over):
        f = dict(layers=2, B=2, N=3, heads=4, kv_heads=2, score_heads=2, head_dim=64, dtype=1, max_depth=2, num_pages=8, page_size=16, table_width=4,
                 scale=0.125, decay=1.0, score_width=64, q_layer_stride=1536, q_stride=256, tree_layer_stride=768, tree_stride=128,
                 cache_layer_stride=16384, page_stride=2048, slot_stride=128)
        return bd._Scores(**{**f, **over})

    def bufs(**over):
        return filled(bd._ScoreBuffers, **over)

    refusals(lib, "mpv_score_positions", shape, bufs, [
        ({"layers": -1}, {}, "MPV_ERR_BAD_SHAPE"), ({"B": -1}, {}, "MPV_ERR_BAD_SHAPE"), ({"N": 0}, {}, "MPV_ERR_BAD_SHAPE"),
        ({"heads": 3}, {}, "MPV_ERR_BAD_SHAPE"), ({"score_heads": 4}, {}, "MPV_ERR_BAD_SHAPE"), ({"score_width": 63}, {}, "MPV_ERR_BAD_SHAPE"),
        ({"page_size": 0}, {}, "MPV_ERR_BAD_SHAPE"), ({"max_depth": -1}, {}, "MPV_ERR_BAD_SHAPE"), ({"q_stride": 128}, {}, "MPV_ERR_BAD_SHAPE"),
        ({"tree_stride": 64}, {}, "MPV_ERR_BAD_SHAPE"), ({"slot_stride": 64}, {}, "MPV_ERR_BAD_SHAPE"), ({"cache_layer_stride": -8}, {}, "MPV_ERR_BAD_SHAPE"),
        ({"dtype": 3}, {}, "MPV_ERR_BAD_DTYPE"), ({"scale": float("inf")}, {}, "MPV_ERR_BAD_TEMPERATURE"),
        ({"decay": float("nan")}, {}, "MPV_ERR_BAD_TEMPERATURE"), ({"N": 65}, {}, "MPV_ERR_UNSUPPORTED"),
        ({"score_width": 1 << 30}, {}, "MPV_ERR_UNSUPPORTED"), ({"q_stride": 1 << 60}, {}, "MPV_ERR_UNSUPPORTED"),
        ({"cache_layer_stride": 1 << 61}, {}, "MPV_ERR_UNSUPPORTED"), ({"layers": 1 << 20, "B": 1 << 20}, {}, "MPV_ERR_UNSUPPORTED"), ({"layers": 1 << 12, "B": 1 << 12}, {}, "MPV_ERR_UNSUPPORTED"),
        ({"head_dim": 60}, {}, "MPV_ERR_ALIGNMENT"), ({"q_layer_stride": 1540}, {}, "MPV_ERR_ALIGNMENT"), ({"page_stride": 2050}, {}, "MPV_ERR_ALIGNMENT"),
        ({}, {"q": FAKE + 8}, "MPV_ERR_ALIGNMENT"), ({}, {"cache_k": FAKE + 2}, "MPV_ERR_ALIGNMENT"),
        ({}, {"q": None}, "MPV_ERR_NULL"), ({}, {"tree_k": None}, "MPV_ERR_NULL"), ({}, {"lse": None}, "MPV_ERR_NULL"), ({}, {"scores": None}, "MPV_ERR_NULL"),
        ({}, {"context_len": None}, "MPV_ERR_NULL"), ({}, {"block_table": None}, "MPV_ERR_NULL"), ({}, {"cache_k": None}, "MPV_ERR_NULL"),
        ({"B": 0}, {}, None), ({"layers": 0}, {}, None),
    ])
    s = shape()
    assert lib.mpv_score_positions(ctypes.byref(s), None, None) == code("MPV_ERR_NULL")
    assert lib.mpv_score_positions(None, ctypes.byref(bufs()), None) == code("MPV_ERR_NULL")


def test_eviction(lib):
    def shape(**over):
        f = dict(layers=2, B=2, kv_heads=2, score_heads=2, head_dim=64, dtype=1, num_pages=8, page_size=16, table_width=4, budget=20, trigger=30, sinks=2,
                 recent=4, score_width=64, cache_layer_stride=16384, page_stride=2048, slot_stride=128)
        return bd._Eviction(**{**f, **over})

    def bufs(**over):
        return filled(bd._EvictionBuffers, **over)

    refusals(lib, "mpv_evict_positions", shape, bufs, [
        ({"layers": -1}, {}, "MPV_ERR_BAD_SHAPE"), ({"B": -1}, {}, "MPV_ERR_BAD_SHAPE"), ({"budget": 0}, {}, "MPV_ERR_BAD_SHAPE"),
        ({"trigger": 19}, {}, "MPV_ERR_BAD_SHAPE"), ({"sinks": -1}, {}, "MPV_ERR_BAD_SHAPE"), ({"recent": -1}, {}, "MPV_ERR_BAD_SHAPE"),
        ({"sinks": 10, "recent": 11}, {}, "MPV_ERR_BAD_SHAPE"), ({"sinks": 2 ** 31 - 1, "recent": 2 ** 31 - 1}, {}, "MPV_ERR_BAD_SHAPE"),
        ({"score_heads": 3}, {}, "MPV_ERR_BAD_SHAPE"), ({"score_width": 63}, {}, "MPV_ERR_BAD_SHAPE"), ({"slot_stride": 64}, {}, "MPV_ERR_BAD_SHAPE"),
        ({"dtype": 5}, {}, "MPV_ERR_BAD_DTYPE"), ({"head_dim": 264, "slot_stride": 1024}, {}, "MPV_ERR_UNSUPPORTED"),
        ({"num_pages": 1 << 30}, {}, "MPV_ERR_UNSUPPORTED"), ({"page_stride": 1 << 61}, {}, "MPV_ERR_UNSUPPORTED"), ({"B": (1 << 24) + 1}, {}, "MPV_ERR_UNSUPPORTED"),
        ({"layers": 1 << 20}, {}, "MPV_ERR_UNSUPPORTED"), ({"layers": 1 << 16, "kv_heads": 1024, "score_heads": 1, "slot_stride": 65536, "page_stride": 1 << 20}, {}, "MPV_ERR_UNSUPPORTED"),
        ({"head_dim": 60}, {}, "MPV_ERR_ALIGNMENT"), ({"cache_layer_stride": 16388}, {}, "MPV_ERR_ALIGNMENT"),
        ({}, {"cache_k": FAKE + 8}, "MPV_ERR_ALIGNMENT"), ({}, {"kept": None}, "MPV_ERR_NULL"), ({}, {"scores": None}, "MPV_ERR_NULL"),
        ({}, {"scores_out": None}, "MPV_ERR_NULL"), ({}, {"free_pages": None}, "MPV_ERR_NULL"), ({}, {"free_count_out": None}, "MPV_ERR_NULL"),
        ({}, {"context_len": None}, "MPV_ERR_NULL"), ({}, {"block_table": None}, "MPV_ERR_NULL"), ({}, {"cache_v": None}, "MPV_ERR_NULL"),
        ({"B": 0}, {}, None),
    ])
    workspaces(lib, "mpv_evict_positions", shape(), bufs())


def test_logprobs(lib):
    def shape(**over):
        return bd._Logprobs(**{**dict(B=2, N=4, V=100, dtype=1, top=3, paths=1, max_depth=3, temperature=1.0, stride=100), **over})

    def bufs(**over):
        return filled(bd._LogprobBuffers, **over)

    refusals(lib, "mpv_token_logprobs", shape, bufs, [
        ({"B": -1}, {}, "MPV_ERR_BAD_SHAPE"), ({"N": 0}, {}, "MPV_ERR_BAD_SHAPE"), ({"V": 0}, {}, "MPV_ERR_BAD_SHAPE"), ({"top": -1}, {}, "MPV_ERR_BAD_SHAPE"),
        ({"stride": 99}, {}, "MPV_ERR_BAD_SHAPE"), ({"paths": 2}, {}, "MPV_ERR_BAD_SHAPE"), ({"max_depth": 0}, {}, "MPV_ERR_BAD_SHAPE"),
        ({"dtype": 3}, {}, "MPV_ERR_BAD_DTYPE"), ({"temperature": 0.0}, {}, "MPV_ERR_BAD_TEMPERATURE"), ({"temperature": float("inf")}, {}, "MPV_ERR_BAD_TEMPERATURE"),
        ({"temperature": -1.0}, {}, "MPV_ERR_BAD_TEMPERATURE"), ({"temperature": float("nan")}, {}, "MPV_ERR_BAD_TEMPERATURE"),
        ({"V": (1 << 21) + 1, "stride": 1 << 22}, {}, "MPV_ERR_UNSUPPORTED"), ({"top": 65}, {}, "MPV_ERR_UNSUPPORTED"), ({"stride": 1 << 61}, {}, "MPV_ERR_UNSUPPORTED"),
        ({"B": 1 << 24}, {}, "MPV_ERR_UNSUPPORTED"), ({"B": 1 << 20}, {}, "MPV_ERR_UNSUPPORTED"),
        ({"B": 1 << 19, "V": 1 << 21, "stride": 1 << 21}, {}, "MPV_ERR_UNSUPPORTED"),
        ({}, {"logits": None}, "MPV_ERR_NULL"), ({}, {"tokens": None}, "MPV_ERR_NULL"), ({}, {"accept_len": None}, "MPV_ERR_NULL"),
        ({}, {"path_nodes": None}, "MPV_ERR_NULL"), ({}, {"bonus_token": None}, "MPV_ERR_NULL"), ({}, {"rank": None}, "MPV_ERR_NULL"),
        ({}, {"top_tokens": None}, "MPV_ERR_NULL"), ({}, {"top_logprobs": None}, "MPV_ERR_NULL"), ({}, {"logits": FAKE + 1}, "MPV_ERR_ALIGNMENT"),
        ({"dtype": 0}, {"logits": FAKE + 2}, "MPV_ERR_ALIGNMENT"), ({"B": 0}, {}, None),
    ])
    workspaces(lib, "mpv_token_logprobs", shape(), bufs())


def test_the_binding_refuses():
    """Tensors on the CPU, and shapes, types and strides that do not fit, without a GPU."""
    bf = dict(dtype=torch.bfloat16)
    q, k = torch.zeros(2, 3, 4, 64, **bf), torch.zeros(2, 3, 2, 64, **bf)
    cache, table, context = torch.zeros(8, 16, 2, 64, **bf), torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        mpv.mpv_prefix_attention([-1, 0, 0], q, k, k, cache, cache, table, context)
    with pytest.raises(ValueError, match="layers"):
        mpv.mpv_score_positions(q, k.unsqueeze(0), cache, table, context, torch.zeros(2, 3, 4), torch.zeros(2, 2, 64))
    with pytest.raises(ValueError, match="CUDA"):
        mpv.mpv_score_positions(q, k, cache, table, context, torch.zeros(2, 3, 4), torch.zeros(2, 2, 64))
    with pytest.raises(ValueError, match="layers"):
        mpv.mpv_evict_positions(cache, cache, table, context, torch.zeros(1, 2, 2, 64), torch.zeros(8, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), 4)
    with pytest.raises(ValueError, match="32 bits"):
        mpv.mpv_evict_positions(cache, cache, table, context, torch.zeros(2, 2, 64), torch.zeros(8, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), 1 << 40)
    with pytest.raises(ValueError, match="CUDA"):
        mpv.mpv_evict_positions(cache, cache, table, context, torch.zeros(2, 2, 64), torch.zeros(8, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), 4)
    with pytest.raises(ValueError, match="CUDA"):
        mpv.mpv_token_logprobs(torch.zeros(1, 2, 10), torch.zeros(1, 2, dtype=torch.int32))
    with pytest.raises(ValueError, match="B,N,V"):
        mpv.mpv_token_logprobs(torch.zeros(2, 10), torch.zeros(2, dtype=torch.int32))
