"""Helpers of the decoder-block GPU tests: bf16 values on the host, caches on
both sides, and the comparison against a bound for every element."""
import numpy as np
import torch

import paper_2407_00066_amd as cts

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
# half a step of the output type, relative: outputs are rounded once
ROUND = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def values(rng, shape, dtype, scale=1.0):
    """Normal values that dtype holds, as (float64 array, device tensor)."""
    t = torch.from_numpy((rng.standard_normal(shape) * scale).astype(np.float32)).to(TORCH[dtype])
    return t.double().numpy(), t.cuda()


def to_device(cache) -> cts.KVCache:
    return cts.KVCache(*(torch.from_numpy(a.copy()).cuda() for a in cache))


def to_host(cache: cts.KVCache):
    return tuple(t.cpu().numpy() for t in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales))


def f64(t):
    return t.detach().double().cpu().numpy()


def assert_within(got, want, bound, what=""):
    got = f64(got) if isinstance(got, torch.Tensor) else got
    assert got.shape == want.shape
    assert np.array_equal(np.isnan(got), np.isnan(want)), "%s: NaN in different places" % what
    with np.errstate(invalid="ignore"):
        over = np.abs(got - want) - bound
    worst = np.nanmax(over) if over.size else -1.0
    assert not worst > 0, "%s: off by up to %.3g past its bound (largest error %.3g)" % (
        what, worst, np.nanmax(np.abs(got - want)))
