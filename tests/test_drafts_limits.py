"""How much work cts_kv_tree_attention takes in a call (CPU; no call here reaches a kernel launch)."""
import ctypes

import pytest
import torch

import paper_2407_00066_amd as cts

from test_block_abi import UNSUPPORTED, _cache, _problem
from test_drafts_abi import _tree


def _need(B, max_q, max_kv, window=0, heads=32, kvh=8, d=128, tree=True):
    p = _problem(T=B * min(max_q, 8), B=B, n_q_heads=heads, max_q=max_q, max_kv=max_kv, window=window, max_pages=1 << 16)
    f = cts.lib().cts_kv_tree_attention_workspace_size if tree else cts.lib().cts_kv_attention_workspace_size
    return f(ctypes.byref(p), ctypes.byref(_cache(n_heads=kvh, head_dim=d, n_pages=1 << 20)))


@pytest.mark.parametrize("B,max_q,max_kv,window", [
    (64, 64, 2 ** 20, 0), (256, 16, 2 ** 20, 0), (256, 128, 131072, 0), (64, 64, 2 ** 20, 4096), (200, 512, 2 ** 20, 0),
    (5, 512, 2 ** 20, 0), (2000, 32, 2 ** 20, 0), (8192, 512, 2 ** 20, 4096), (20000, 8, 2 ** 20, 0)])
def test_loose_bounds_are_taken(B, max_q, max_kv, window):
    """Bounds say what could be, not what is: batches that a launch has the workgroups for are taken, whatever their bounds
    multiply to."""
    assert 0 < _need(B, max_q, max_kv, window) <= 8 << 30


def test_past_a_launch():
    """2^23 workgroups of 512 threads."""
    for kw in (dict(T=2 ** 20, B=2 ** 20, max_q=1, n_q_heads=32), dict(T=2 ** 19, B=2 ** 18, max_q=512, n_q_heads=32)):
        for window in (0, 100):
            p, c = _problem(**kw, window=window, max_kv=40), _cache(n_heads=8)
            assert cts.lib().cts_kv_tree_attention_workspace_size(ctypes.byref(p), ctypes.byref(c)) == 0
            assert _tree(p, c, ldq=1 << 13, ldo=1 << 13) == UNSUPPORTED
    p, c = _problem(T=2 ** 20 - 512, B=2 ** 20 - 512, n_q_heads=32, max_kv=40), _cache(n_heads=8)
    assert cts.lib().cts_kv_tree_attention_workspace_size(ctypes.byref(p), ctypes.byref(c)) > 0


@pytest.mark.parametrize("kvh,heads,d", [(8, 32, 128), (1, 8, 256), (2, 2, 64)])
def test_workspace_does_not_fall_with_much_work(kvh, heads, d):
    """A workspace for the largest batch serves every smaller one, where tiles are no longer cut too."""
    batches, lengths = [1, 3, 60, 64, 65, 500, 1023, 1025, 4095, 4097, 9000, 33000], [0, 2000, 8192, 8224, 9000, 131072, 2 ** 20]
    for max_q in (1, 7, 64, 512):
        need = [[_need(b, max_q, n, 0, heads, kvh, d) for n in lengths] for b in batches]
        if max_q < 512:
            assert all(min(r) > 0 for r in need)
        need = [r for r in need if min(r) > 0]
        assert all(r == sorted(r) for r in need) and all(list(col) == sorted(col) for col in zip(*need))
    for b in batches:
        rows = [_need(b, q, 131072, 0, heads, kvh, d) for q in (1, 2, 3, 8, 17, 64)]
        assert rows == sorted(rows)
        for window in (1, 700, 9000, 2 ** 19):
            assert _need(b, 33, 2 ** 20, window, heads, kvh, d) <= _need(b, 33, 2 ** 20, 0, heads, kvh, d)


def test_plan_of_much_work():
    """Many tiles are taken whole however long they may be, fewer are cut."""
    def how(B, max_q, cols):
        cache = cts.kv_cache(1, 16, 8, 128, device="cpu")
        q = torch.zeros(1, 32, 128, dtype=torch.bfloat16).expand(B * 2, -1, -1)
        return cts.kv_tree_attention_plan(q, cache, torch.zeros(1, 1).expand(B, cols), max_q, cols * 16)[1]
    assert how(64, 64, 65536) == "cut" and how(1024, 8, 65536) == "cut" and how(2048, 8, 65536) == "cut"
    assert how(2049, 8, 65536) == "whole" and how(1025, 31, 65536) == "whole"


@pytest.mark.parametrize("rows,words", [(33, 1), (40, 1), (65, 2), (513, 20)])
def test_max_q_is_asked_for(rows, words):
    """(CPU tensors: refused before the device is.)"""
    cache = cts.kv_cache(2, 16, 2, 64, device="cpu")
    i32 = lambda *shape: torch.zeros(*shape, dtype=torch.int32)
    args = [torch.zeros(rows, 2, 64), cache, i32(2, 2), i32(2), i32(rows, words)]
    with pytest.raises(ValueError, match="max_q"):
        cts.kv_tree_attention(*args, q_start=i32(3))
    for kw in (dict(q_start=i32(3), max_q=32), dict()):
        with pytest.raises(ValueError, match="GPU"):
            cts.kv_tree_attention(*args, **kw)
