"""Whose memory the calls around a verification write (needs an MI355X)."""

import pytest
import torch

import paper_2602_16994_amd as mpv
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
