"""Sizes at which the decoder block's memory-bound operators take other kernels or
launches than in the small tests: streaming stores (outputs of 4 MB and more),
angles shared by several heads, several tokens a workgroup, and more rows than one
launch has threads for."""
import numpy as np
import pytest
import torch

import paper_2407_00066_amd as cts

from _gpu_helpers import say

pytestmark = pytest.mark.gpu


def test_norm_of_more_rows_than_a_launch():
    """2^32 threads is what a launch cannot have: short rows reach it with 134 MB."""
    T = 2 ** 26 + 5
    x = torch.randn(T, 1, device="cuda").bfloat16()
    w = torch.full((1,), 3.0, dtype=torch.bfloat16, device="cuda")
    say("block_norm T=%d d=1" % T)
    n = torch.full_like(x, float("nan"))
    cts.block_norm(x, w, eps=1e-3, n_out=n)
    torch.cuda.synchronize()
    for at in range(0, T, 2 ** 24):
        a = x[at:at + 2 ** 24].float()
        want = 3 * a / (a * a + 1e-3).sqrt()
        # one rounding to bf16, and a few of fp32 on either side
        assert bool(((n[at:at + 2 ** 24].float() - want).abs() <= 1.001 * 2.0 ** -8 * want.abs()).all())


def test_block_norm_of_more_rows_than_a_launch():
    """With the residual, a gate for every token and outputs in place."""
    T, d = 2 ** 22 + 9, 2
    x, y, gate = (torch.randn(T, d, device="cuda") for _ in range(3))
    w, post = torch.tensor([3.0, -1.0], device="cuda"), torch.tensor([0.5, 2.0], device="cuda")

    def unit(a):
        return a / ((a * a).mean(1, keepdim=True) + 1e-3).sqrt()
    h = x.double() + 0.7 * gate.double() * unit(y.double()) * post.double()
    n = unit(h) * w.double()
    # h of two terms of a few roundings each; n's mean follows h's error
    mag = 8 * 2.0 ** -24 * (x.double().abs() + (0.7 * gate * post).double().abs() * 2)
    say("block_norm T=%d d=%d" % (T, d))
    got = cts.block_norm(x, w, y=y, post_weight=post, gate=gate, scale=0.7, eps=1e-3, h_out=x, n_out=y)
    assert got[0].data_ptr() == x.data_ptr()
    assert bool(((got[0].double() - h).abs() <= mag).all())
    rs = 1 / ((h * h).mean(1, keepdim=True) + 1e-3).sqrt()
    assert bool(((got[1].double() - n).abs() <= 3 * rs * (mag + mag.amax(1, keepdim=True) * n.abs()) + 2.0 ** -20 * n.abs()).all())
