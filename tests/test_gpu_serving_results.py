"""Whose memory the calls around a verification write (needs an MI355X)."""

import pytest
import torch

import paper_2602_16994_amd as mpv
from tests.test_gpu_chains import make as make_chains
from tests.test_gpu_serving_streams import i32, tables

pytestmark = pytest.mark.gpu


def test_a_result_of_a_call_in_place_is_used_again_by_one_that_is_not():
    print("[case] in place, then not", flush=True)
    a = tables()
    res = mpv.mpv_extend_tables(**a, inplace=True)
    assert a["context_len"].tolist() == [5, 17] and a["free_count"].tolist() == [3]
    res = mpv.mpv_extend_tables(**a, out=res)
    assert res.context_len.tolist() == [7, 18] and res.free_count.tolist() == [3]
    assert a["context_len"].tolist() == [5, 17] and a["free_count"].tolist() == [3]
    # nor does it write to the tensors of the earlier call when it is given others
    b = tables()
    res = mpv.mpv_extend_tables(**b, inplace=True)
    c = tables()
    c["context_len"] += 1
    again = mpv.mpv_extend_tables(**c, out=res)
    assert b["context_len"].tolist() == [5, 17] and b["free_count"].tolist() == [3]
    assert again.context_len.tolist() == [6, 18] and c["context_len"].tolist() == [4, 17]


def test_lengths_of_a_result_are_the_next_call_s_input():
    print("[case] lengths from a result", flush=True)
    a = tables()
    res = mpv.mpv_extend_tables(**a)
    given, left = res.context_len, res.free_count
    a["context_len"], a["free_count"] = given, left
    res = mpv.mpv_extend_tables(**a, out=res)
    assert given.tolist() == [5, 17] and left.tolist() == [3]
    assert res.context_len.tolist() == [7, 18] and res.free_count.tolist() == [3]
    kept = res.context_len.data_ptr(), res.free_count.data_ptr()
    a["context_len"], a["free_count"] = i32([5, 17]), i32([3])
    res = mpv.mpv_extend_tables(**a, out=res)      # otherwise the buffers are reused
    assert (res.context_len.data_ptr(), res.free_count.data_ptr()) == kept


def test_a_refused_call_leaves_the_result_as_it_was():
    print("[case] refused", flush=True)
    a = tables()
    res = mpv.mpv_extend_tables(**a)
    kept = res.context_len, res.free_count
    b = tables()
    b["new_len"] = b["new_len"].long()
    with pytest.raises(TypeError):
        mpv.mpv_extend_tables(**b, inplace=True, out=res)
    assert res.context_len is kept[0] and res.free_count is kept[1]


@pytest.mark.parametrize("packed", [False, True])
def test_no_requests(packed):
    print("[case] no requests", packed, flush=True)
    a = tables()
    for name in ("block_table", "context_len", "new_len"):
        a[name] = a[name][:0]
    a["slot_map"] = torch.full((4,), -7, dtype=torch.int64, device="cuda") if packed else a["slot_map"][:0]
    old = mpv.TablesResult(context_len=i32([]), free_count=i32([99]), granted=i32([]), slot_map=a["slot_map"], offsets=i32([99]))
    res = mpv.mpv_extend_tables(**a, out=old)
    assert res.free_count.tolist() == [4] and res.offsets.tolist() == [0] and res.context_len.numel() == 0
    assert a["free_count"].tolist() == [4] and a["free_pages"].tolist() == [0, 1, 2, 3, -1, -1] and (a["slot_map"] == -7).all()
    a["free_count"] = i32([10 ** 6])               # taken within [0, num_pages]
    res = mpv.mpv_extend_tables(**a, inplace=True)
    assert a["free_count"].tolist() == [6] and res.free_count is a["free_count"]


def test_no_chains():
    print("[case] no chains", flush=True)
    tokens, p, q, u = make_chains(2, 3, 10, torch.float32)
    old = mpv.mpv_verify_chains(tokens, p, q, u)
    for name in ("accept_len", "path_nodes", "path_tokens", "bonus_token"):
        setattr(old, name, getattr(old, name)[:0])
    old.counters.fill_(5)
    res = mpv.mpv_verify_chains(tokens[:0], p[:0], q[:0], u[:0], out=old)
    assert res.counters.tolist() == [0] * 8 and res.accept_len.numel() == 0
