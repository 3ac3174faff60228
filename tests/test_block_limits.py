"""Calls of more work than a launch has threads for are refused on the host (CPU;
no call here reaches a kernel launch)."""
import ctypes

import pytest
import torch

import paper_2407_00066_amd as cts
from paper_2407_00066_amd import _binding as B

from test_block_abi import INVALID, UNSUPPORTED, _attend, _cache, _problem, _write

GROUPS = 2 ** 24 - 1                  # workgroups of 256 threads that a launch can have


@pytest.mark.parametrize("dtype,read,tokens", [(B.CTS_BF16, False, 32), (B.CTS_F32, False, 32), (B.CTS_BF16, True, 32),
                                               (B.CTS_F32, True, 16)])
def test_kv_calls_past_a_launch(dtype, read, tokens):
    """tokens: of a workgroup, for two heads of 64."""
    assert _write(T=GROUPS * tokens + 1, dtype=dtype, read=read) == UNSUPPORTED
    assert _write(T=2 ** 31 - 1, dtype=dtype, read=read) == UNSUPPORTED


@pytest.mark.parametrize("kw", [
    dict(T=2 ** 22, B=2 ** 22),                                         # 2^23 tiles of 512 threads
    dict(T=2 ** 22, B=2 ** 21, max_q=2, n_q_heads=32),                  # two tiles a sequence
    dict(T=2 ** 29 - 1, B=1, max_q=1000),                               # prompts of 128 rows a workgroup
    dict(T=2 ** 27, B=1, max_q=1000, dtype=B.CTS_F32)])                 # 16 rows a workgroup
def test_attention_past_a_launch(kw):
    p, c = _problem(**kw), _cache()
    assert cts.lib().cts_kv_attention_workspace_size(ctypes.byref(p), ctypes.byref(c)) == 0
    assert _attend(p) == UNSUPPORTED


def test_scale_past_the_exponent():
    """The kernels' exponentials are of base 2: scale log2(e) has to be a float too."""
    assert _attend(_problem(scale=3e38)) == INVALID
    p, c = _problem(scale=2.0 ** 127), _cache()
    assert cts.lib().cts_kv_attention_workspace_size(ctypes.byref(p), ctypes.byref(c)) > 0


def test_workspace_size_of_sizes_past_32_bits():
    cache, q = cts.kv_cache(2, 16, 2, 64, device="cpu"), torch.zeros(3, 4, 64)
    assert cts.kv_attention_workspace_size(q, cache, 3, 1, 40) > 0
    for kw in (dict(B=2 ** 32 + 3), dict(max_q=2 ** 32 + 1), dict(max_kv=2 ** 32 + 40), dict(window=2 ** 32 + 5)):
        assert cts.kv_attention_workspace_size(q, cache, **{**dict(B=3, max_q=1, max_kv=40), **kw}) == 0, kw


def test_attention_plan():
    def plan(B_, max_q=1, max_kv=4000, kvh=8, heads=32, window=0, dtype=torch.bfloat16, cols=1 << 14):
        cache = cts.kv_cache(1, 16, kvh, 128, device="cpu")
        return cts.kv_attention_plan(torch.zeros(B_ * max_q, heads, 128, dtype=dtype), cache, torch.zeros(B_, cols), max_q,
                                     max_kv, window)
    assert plan(1, max_kv=700) == ("whole", 0, 0) and plan(1) == ("runs", 64, 0)
    assert plan(64) == ("by length", 0, 0) and plan(65) == ("whole", 0, 0) and plan(64, max_kv=1000) == ("whole", 0, 0)
    assert plan(64, max_kv=10000)[0] == "runs" and plan(64, max_kv=10000, cols=64)[0] == "by length"
    assert plan(4, max_q=100, max_kv=300) == ("whole", 0, 1) and plan(1, max_q=100, max_kv=9000)[2] > 1
    assert plan(4, max_q=100, max_kv=300, dtype=torch.float32)[2] == 0
    assert plan(1, max_kv=9000, window=500)[0] == "whole"
    p, c, out = _problem(), _cache(), (ctypes.c_int32 * 3)()
    f = cts.lib().cts_kv_attention_plan
    assert f(ctypes.byref(p), ctypes.byref(c), None) == INVALID and f(None, ctypes.byref(c), out) == INVALID
    assert f(ctypes.byref(_problem(dtype=5)), ctypes.byref(c), out) == UNSUPPORTED


@pytest.mark.parametrize("kw", [dict(T=2 ** 22 - 1, B=2 ** 22 - 1), dict(T=2 ** 28, B=1, max_q=1000),
                                dict(T=2 ** 26 - 64, B=1, max_q=1000, dtype=B.CTS_F32)])
def test_attention_of_a_whole_launch_is_taken(kw):
    p, c = _problem(**kw), _cache()
    assert cts.lib().cts_kv_attention_workspace_size(ctypes.byref(p), ctypes.byref(c)) > 0
