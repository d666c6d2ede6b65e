"""Temperatures that mpv_token_logprobs takes (no GPU)."""

import ctypes

import pytest

import paper_2602_16994_amd as mpv
from paper_2602_16994_amd import binding as bd
from tests.test_abi_cpu import code


@pytest.mark.parametrize("temperature,fine", [(1.0, True), (3.4e38, True), (2.0 ** -126, True), (2.0 ** -127, False), (1e-44, False), (0.0, False)])
def test_temperatures(temperature, fine):
    """1 / T and log2(e) / T are float32: of numbers below the smallest normal one they would be infinite, and every result no number."""
    lib = mpv.load_library()
    shape = bd._Logprobs(B=1, N=1, V=10, dtype=0, top=1, paths=0, max_depth=0, temperature=temperature, stride=10)
    need = ctypes.c_size_t()
    assert lib.mpv_token_logprobs_workspace_bytes(ctypes.byref(shape), ctypes.byref(need)) == (0 if fine else code("MPV_ERR_BAD_TEMPERATURE"))
