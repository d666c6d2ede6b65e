"""What the calls around a verification refuse, before anything is launched (no GPU needed)."""

import ctypes

import pytest
import torch

import paper_2602_16994_amd as mpv
from paper_2602_16994_amd import binding as bd
from tests.test_abi_cpu import code

FAKE = 1 << 20                                     # an aligned address that is never read


@pytest.fixture(scope="module")
def lib():
    return mpv.load_library()


def filled(cls, **over):
    b = cls()
    for name, _ in cls._fields_:
        setattr(b, name, FAKE)
    for name, value in over.items():
        setattr(b, name, value)
    return b


def refusals(lib, name, shape, buffers, cases):
    """cases: (fields of the shape, fields of the buffers, error)."""
    call = getattr(lib, name)
    for fields, bufs, error in cases:
        s, b = shape(**fields), buffers(**bufs)
        got = call(ctypes.byref(s), ctypes.byref(b), FAKE, 1 << 30, None) if name != "mpv_append_paths" else call(ctypes.byref(s), ctypes.byref(b), None)
        assert got == (code(error) if error else 0), (fields, bufs, error, got)


def attention(parent=(-1, 0, 0), **over):
    f = dict(B=2, N=3, heads=4, kv_heads=2, head_dim=64, dtype=1, num_pages=8, page_size=16, table_width=4, window=0, sinks=0, scale=0.125,
             q_stride=256, kv_stride=128, out_stride=256, page_stride=2048, slot_stride=128)
    f.update(over)
    arr = (ctypes.c_int32 * len(parent))(*parent) if parent is not None else None
    s = bd._Attention(**f)
    s.parent = arr
    s._keepalive = arr
    return s


def test_attention(lib):
    def bufs(**over):
        return filled(bd._AttentionBuffers, **{"num_nodes": None, "tree_parent": None, **over})

    none = dict(B=0)
    refusals(lib, "mpv_tree_attention", attention, bufs, [
        ({"B": -1}, {}, "MPV_ERR_BAD_SHAPE"), ({"N": 0}, {}, "MPV_ERR_BAD_SHAPE"), ({"heads": 3}, {}, "MPV_ERR_BAD_SHAPE"),
        ({"heads": 0}, {}, "MPV_ERR_BAD_SHAPE"), ({"kv_heads": 0}, {}, "MPV_ERR_BAD_SHAPE"), ({"head_dim": 0}, {}, "MPV_ERR_BAD_SHAPE"),
        ({"page_size": 0}, {}, "MPV_ERR_BAD_SHAPE"), ({"num_pages": -1}, {}, "MPV_ERR_BAD_SHAPE"), ({"table_width": -1}, {}, "MPV_ERR_BAD_SHAPE"),
        ({"q_stride": 248}, {}, "MPV_ERR_BAD_SHAPE"), ({"kv_stride": 64}, {}, "MPV_ERR_BAD_SHAPE"), ({"out_stride": 0}, {}, "MPV_ERR_BAD_SHAPE"),
        ({"slot_stride": 64}, {}, "MPV_ERR_BAD_SHAPE"), ({"page_stride": -128}, {}, "MPV_ERR_BAD_SHAPE"),
        ({"dtype": 3}, {}, "MPV_ERR_BAD_DTYPE"), ({"dtype": -1}, {}, "MPV_ERR_BAD_DTYPE"),
        ({"scale": float("nan")}, {}, "MPV_ERR_BAD_TEMPERATURE"), ({"scale": float("inf")}, {}, "MPV_ERR_BAD_TEMPERATURE"),
        ({"N": 65}, {}, "MPV_ERR_UNSUPPORTED"), ({"head_dim": 264, "q_stride": 2048, "out_stride": 2048, "kv_stride": 1024, "slot_stride": 1024}, {}, "MPV_ERR_UNSUPPORTED"),
        ({"table_width": 1 << 20, "page_size": 1 << 12}, {}, "MPV_ERR_UNSUPPORTED"), ({"q_stride": 1 << 60}, {}, "MPV_ERR_UNSUPPORTED"),
        ({"page_stride": 1 << 61}, {}, "MPV_ERR_UNSUPPORTED"), ({"B": (1 << 24) + 1}, {}, "MPV_ERR_UNSUPPORTED"),
        ({"head_dim": 60}, {}, "MPV_ERR_ALIGNMENT"), ({"q_stride": 260}, {}, "MPV_ERR_ALIGNMENT"), ({"kv_stride": 132}, {}, "MPV_ERR_ALIGNMENT"),
        ({"page_stride": 2050}, {}, "MPV_ERR_ALIGNMENT"),
        ({}, {"q": FAKE + 8}, "MPV_ERR_ALIGNMENT"), ({}, {"cache_v": FAKE + 2}, "MPV_ERR_ALIGNMENT"), ({}, {"out": FAKE + 4}, "MPV_ERR_ALIGNMENT"),
        ({}, {"q": None}, "MPV_ERR_NULL"), ({}, {"tree_k": None}, "MPV_ERR_NULL"), ({}, {"cache_k": None}, "MPV_ERR_NULL"),
        ({}, {"block_table": None}, "MPV_ERR_NULL"), ({}, {"context_len": None}, "MPV_ERR_NULL"), ({}, {"out": None}, "MPV_ERR_NULL"),
        ({"parent": None}, {}, "MPV_ERR_NULL"), ({"parent": (0, 0, 0)}, {}, "MPV_ERR_BAD_TREE"), ({"parent": (-1, 1, 0)}, {}, "MPV_ERR_BAD_TREE"),
        ({"parent": (-1, 0, 2)}, {}, "MPV_ERR_BAD_TREE"),
        (none, {}, None), ({**none, "parent": None}, {}, "MPV_ERR_NULL"),
    ])
    s, b = attention(), bufs()
    assert lib.mpv_tree_attention(ctypes.byref(s), ctypes.byref(b), None, 1 << 30, None) == code("MPV_ERR_WORKSPACE")
    assert lib.mpv_tree_attention(ctypes.byref(s), ctypes.byref(b), FAKE + 8, 1 << 30, None) == code("MPV_ERR_WORKSPACE")
    assert lib.mpv_tree_attention(ctypes.byref(s), ctypes.byref(b), FAKE, 16, None) == code("MPV_ERR_WORKSPACE")
    assert lib.mpv_tree_attention(None, ctypes.byref(b), FAKE, 1 << 30, None) == code("MPV_ERR_NULL")
    assert lib.mpv_tree_attention(ctypes.byref(s), None, FAKE, 1 << 30, None) == code("MPV_ERR_NULL")
    assert lib.mpv_tree_attention_workspace_bytes(ctypes.byref(s), None) == code("MPV_ERR_NULL")


def test_chains(lib):
    def shape(**over):
        return bd._Chains(**{**dict(B=2, N=4, V=100, dtype=0, max_depth=3, target_stride=100, draft_stride=100), **over})

    def bufs(**over):
        return filled(bd._ChainBuffers, **{"num_nodes": None, **over})

    refusals(lib, "mpv_verify_chains", shape, bufs, [
        ({"B": -1}, {}, "MPV_ERR_BAD_SHAPE"), ({"N": 0}, {}, "MPV_ERR_BAD_SHAPE"), ({"V": 0}, {}, "MPV_ERR_BAD_SHAPE"),
        ({"max_depth": 2}, {}, "MPV_ERR_BAD_SHAPE"), ({"N": 1, "max_depth": 0}, {}, "MPV_ERR_BAD_SHAPE"),
        ({"target_stride": 99}, {}, "MPV_ERR_BAD_SHAPE"), ({"draft_stride": 99}, {}, "MPV_ERR_BAD_SHAPE"),
        ({"dtype": 7}, {}, "MPV_ERR_BAD_DTYPE"), ({"N": 65, "max_depth": 64}, {}, "MPV_ERR_UNSUPPORTED"),
        ({"V": (1 << 21) + 1, "target_stride": 1 << 22, "draft_stride": 1 << 22}, {}, "MPV_ERR_UNSUPPORTED"),
        ({"target_stride": 1 << 61}, {}, "MPV_ERR_UNSUPPORTED"),
        ({}, {"target_probs": None}, "MPV_ERR_NULL"), ({}, {"tokens": None}, "MPV_ERR_NULL"), ({}, {"uniforms": None}, "MPV_ERR_NULL"),
        ({}, {"accept_len": None}, "MPV_ERR_NULL"), ({}, {"path_nodes": None}, "MPV_ERR_NULL"), ({}, {"path_tokens": None}, "MPV_ERR_NULL"),
        ({}, {"bonus_token": None}, "MPV_ERR_NULL"), ({}, {"counters": None}, "MPV_ERR_NULL"),
        ({}, {"target_probs": FAKE + 2}, "MPV_ERR_ALIGNMENT"), ({"dtype": 1}, {"draft_probs": FAKE + 1}, "MPV_ERR_ALIGNMENT"),
        ({"B": 0}, {}, None),
    ])
    s, b = shape(), bufs()
    assert lib.mpv_verify_chains(ctypes.byref(s), ctypes.byref(b), None, 1 << 30, None) == code("MPV_ERR_WORKSPACE")
    assert lib.mpv_verify_chains(ctypes.byref(s), ctypes.byref(b), FAKE, 8, None) == code("MPV_ERR_WORKSPACE")
    assert lib.mpv_verify_chains(ctypes.byref(s), None, FAKE, 1 << 30, None) == code("MPV_ERR_NULL")


def test_tables(lib):
    def shape(**over):
        return bd._Tables(**{**dict(B=2, page_size=16, table_width=4, num_pages=8, extra=1, packed=0, slot_width=5), **over})

    def bufs(**over):
        return filled(bd._TableBuffers, **over)

    refusals(lib, "mpv_extend_tables", shape, bufs, [
        ({"B": -1}, {}, "MPV_ERR_BAD_SHAPE"), ({"page_size": 0}, {}, "MPV_ERR_BAD_SHAPE"), ({"table_width": -1}, {}, "MPV_ERR_BAD_SHAPE"),
        ({"num_pages": -1}, {}, "MPV_ERR_BAD_SHAPE"), ({"extra": -1}, {}, "MPV_ERR_BAD_SHAPE"), ({"packed": 2}, {}, "MPV_ERR_BAD_SHAPE"),
        ({"slot_width": -1}, {}, "MPV_ERR_BAD_SHAPE"),
        ({"slot_width": 1 << 31, "packed": 1}, {}, "MPV_ERR_UNSUPPORTED"), ({"slot_width": 1 << 30}, {}, "MPV_ERR_UNSUPPORTED"),
        ({"table_width": 1 << 20, "page_size": 1 << 11}, {}, "MPV_ERR_UNSUPPORTED"),
        ({}, {"new_len": None}, "MPV_ERR_NULL"), ({}, {"context_len": None}, "MPV_ERR_NULL"), ({}, {"block_table": None}, "MPV_ERR_NULL"),
        ({}, {"free_pages": None}, "MPV_ERR_NULL"), ({}, {"free_count": None}, "MPV_ERR_NULL"), ({}, {"context_len_out": None}, "MPV_ERR_NULL"),
        ({}, {"free_count_out": None}, "MPV_ERR_NULL"), ({}, {"slot_map": None}, "MPV_ERR_NULL"), ({}, {"granted": None}, "MPV_ERR_NULL"),
        ({"packed": 1}, {"offsets": None}, "MPV_ERR_NULL"), ({"B": 0}, {}, None),
    ])
    s, b = shape(), bufs()
    assert lib.mpv_extend_tables(ctypes.byref(s), ctypes.byref(b), None, 1 << 30, None) == code("MPV_ERR_WORKSPACE")
    assert lib.mpv_extend_tables(ctypes.byref(s), ctypes.byref(b), FAKE, 16, None) == code("MPV_ERR_WORKSPACE")


def test_append(lib):
    def shape(**over):
        return bd._Append(**{**dict(layers=2, B=2, N=4, dtype=1, row=128, max_depth=3, slot_width=4, num_pages=8, page_size=16,
                                    tree_layer_stride=1024, tree_stride=128, cache_layer_stride=16384, page_stride=2048, slot_stride=128), **over})

    def bufs(**over):
        return filled(bd._AppendBuffers, **over)

    refusals(lib, "mpv_append_paths", shape, bufs, [
        ({"layers": -1}, {}, "MPV_ERR_BAD_SHAPE"), ({"N": 0}, {}, "MPV_ERR_BAD_SHAPE"), ({"row": 0}, {}, "MPV_ERR_BAD_SHAPE"),
        ({"page_size": 0}, {}, "MPV_ERR_BAD_SHAPE"), ({"max_depth": -1}, {}, "MPV_ERR_BAD_SHAPE"), ({"tree_stride": 120}, {}, "MPV_ERR_BAD_SHAPE"),
        ({"slot_stride": 64}, {}, "MPV_ERR_BAD_SHAPE"), ({"cache_layer_stride": -8}, {}, "MPV_ERR_BAD_SHAPE"),
        ({"dtype": 9}, {}, "MPV_ERR_BAD_DTYPE"), ({"N": 65}, {}, "MPV_ERR_UNSUPPORTED"), ({"page_stride": 1 << 61}, {}, "MPV_ERR_UNSUPPORTED"),
        ({"tree_layer_stride": 1 << 62}, {}, "MPV_ERR_UNSUPPORTED"), ({"layers": 1 << 20}, {}, "MPV_ERR_UNSUPPORTED"),
        ({}, {"tree_k": None}, "MPV_ERR_NULL"), ({}, {"cache_v": None}, "MPV_ERR_NULL"), ({}, {"slot_map": None}, "MPV_ERR_NULL"),
        ({}, {"accept_len": None}, "MPV_ERR_NULL"), ({}, {"tree_v": FAKE + 8}, "MPV_ERR_ALIGNMENT"), ({"row": 124}, {}, "MPV_ERR_ALIGNMENT"),
        ({"page_stride": 2052}, {}, "MPV_ERR_ALIGNMENT"),
        ({"B": 0}, {}, None), ({"layers": 0}, {}, None), ({"slot_width": 0}, {}, None),
    ])


def test_the_binding_refuses_host_tensors_and_other_layouts():
    i = torch.zeros(2, dtype=torch.int32)
    q, k, c = torch.zeros(2, 3, 4, 64), torch.zeros(2, 3, 2, 64), torch.zeros(8, 16, 2, 64)
    with pytest.raises(ValueError):
        mpv.mpv_tree_attention([-1, 0, 0], q, k, k, c, c, torch.zeros(2, 4, dtype=torch.int32), i)
    with pytest.raises(ValueError):
        mpv.mpv_verify_chains(torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, 3, 9), None, torch.zeros(2, 3))
    with pytest.raises(ValueError):
        mpv.mpv_extend_tables(torch.zeros(2, 4, dtype=torch.int32), i, i, torch.zeros(8, dtype=torch.int32), i[:1], 16, torch.zeros(2, 3, dtype=torch.int64))
    with pytest.raises(ValueError):
        mpv.mpv_append_paths(k, k, c, c, torch.zeros(2, 3, dtype=torch.int64), i)


def test_row_strides():
    x = torch.zeros(4, 5, 6, 8)
    assert bd._row_stride("x", x, (4, 5), (6, 8)) == 48
    assert bd._row_stride("x", x[:, :, :2], (4, 5), (2, 8)) == 48
    assert bd._row_stride("x", x[:1, :, 2:3], (1, 5), (1, 8)) == 48
    assert bd._row_stride("x", x[:, :1], (4, 1), (6, 8)) == 240
    assert bd._row_stride("x", x[:1, :1], (1, 1), (6, 8)) == 48
    for bad, lead, inner in ((x[:, :4], (4, 4), (6, 8)), (x[:, :, :, :4], (4, 5), (6, 4)), (x.transpose(0, 1), (5, 4), (6, 8)),
                             (x, (4, 5), (6, 7)), (x[:, :, ::2], (4, 5), (3, 8))):
        with pytest.raises(ValueError):
            bd._row_stride("x", bad, lead, inner)
    k = torch.zeros(9, 2, 16, 3, 8)
    assert bd._cache_strides(k[:, 0], k[:, 1], (9, 16, 3, 8)) == (768, 24)
    with pytest.raises(ValueError):
        bd._cache_strides(k[:, 0], k[:, 1].contiguous(), (9, 16, 3, 8))
    with pytest.raises(ValueError):
        bd._cache_strides(k[:, 0, :, :, ::2], k[:, 1, :, :, ::2], (9, 16, 3, 4))
