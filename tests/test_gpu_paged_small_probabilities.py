"""Outputs that are made of small probabilities alone, beside tokens that have nearly all of the weight and no value in some
channels."""
import numpy as np
import pytest
import torch

from tests import gpu_util_paged as U

pytestmark = pytest.mark.gpu


def _floor(p, V, dtype):
    """What the operands of an fp16 cache's probabilities may lose beyond 2^-22 of each: fp16 numbers are 2^-24 apart or more, so
    that the second operand is off by 2^-25; the largest probability of a wavefront stands at 2^10 or more when it is done, and
    what was added before is scaled down with it: 2^-35 of the largest probability for every token.  (bf16 has fp32's range.)"""
    return 2.0 ** -35 * p.max(-1, keepdims=True) * np.abs(V).sum(0) if dtype == "f16" else 0.0


@pytest.mark.parametrize("below", [8, 16, 20, 24, 28, 32, 40])
@pytest.mark.parametrize("n", [64, 3000, 20000])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_many_small_probabilities(dtype, n, below):
    """Every unit of 32 tokens has one that is 2^below times as heavy as its others and is zero in the first channels."""
    Hq, d, page, gain = 2, 64, 32, 1000.0
    cache = U.make(1, Hq, 1, d, page, dtype, -(-n // page))
    cache.reserve([n])
    K, V = U.rows(1, 1, 1, n, d, dtype=dtype, gain=0.02), U.rows(2, 1, 1, n, d, dtype=dtype, gain=gain) + gain
    q = U.rows(3, 1, Hq, d, dtype=dtype, gain=0.5)
    heavy = torch.arange(n) % 32 == 7
    q[..., 0] = 8
    K[..., 0] = torch.where(heavy, below * np.log(2) / 8, 0.0).to(K.dtype)
    V[..., :d // 2] = torch.where(heavy[:, None], torch.zeros((), dtype=V.dtype), V[..., :d // 2])
    cache.append(K.to(U.DEVICE), V.to(U.DEVICE))
    out = U.f64(cache.decode_attn(q.to(U.DEVICE), softmax_scale=1.0))[0]
    k, v = U.f64(K)[0, 0], U.f64(V)[0, 0]
    want, p, bound, _ = U.attention_and_bounds(U.f64(q)[0], k, v, 1.0, dtype)
    bound = bound + (1 + U.HALF_STEP[dtype]) * _floor(p, v, dtype)
    off = np.abs(out - want)
    assert (off <= bound).all(), (off.max(), (off / bound).max())
