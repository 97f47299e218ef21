"""Rotary positions on the GPU against the oracle."""
import numpy as np
import pytest
import torch

from oracle import paged
from paper_2503_19950_amd import binding
from tests import gpu_util_paged as U

pytestmark = pytest.mark.gpu

CASES = [  # B, L, Hq, Hkv, d, dims, interleaved, dtype
    (3, 1, 32, 8, 128, 128, False, "f16"), (1, 33, 4, 2, 128, 128, False, "bf16"), (2, 17, 3, 1, 96, 96, False, "f16"),
    (2, 5, 2, 2, 64, 64, True, "bf16"), (1, 16, 1, 1, 128, 64, True, "f16"), (1, 100, 8, 2, 64, 32, False, "bf16"),
    # rotated channels that are no whole pieces of 16 bytes
    (2, 9, 2, 1, 96, 24, False, "f16"), (1, 20, 3, 3, 64, 2, False, "bf16"), (1, 3, 2, 1, 128, 126, False, "f16"),
    (2, 7, 2, 1, 64, 6, True, "f16"), (1, 31, 5, 5, 96, 90, True, "bf16"), (1, 2, 1, 1, 96, 8, True, "f16"),
    # many workgroups that share no heads, and many tokens
    (1, 4099, 2, 1, 64, 64, False, "f16"), (70, 1, 71, 1, 64, 64, False, "bf16"),
]


def _positions(seed, B, L):
    r = np.random.RandomState(seed)
    return torch.from_numpy(r.choice([0, 1, 7, 4095, 131071, 10 ** 6, 2 ** 31 - 1, -1, -5000, -2 ** 31], (B, L)).astype(np.int32))


def _check(got, x, positions, freq, interleaved, factor, dtype):
    for b in range(x.shape[0]):
        want, bound = U.rotated_and_bound(U.f64(x[b]), positions[b], freq, interleaved, factor, dtype)
        off = np.abs(U.f64(got[b]) - want)
        assert (off <= bound).all(), (b, off.max(), np.argwhere(~(off <= bound))[:3])


@pytest.mark.parametrize("case", CASES, ids=str)
def test_rotate(case):
    B, L, Hq, Hkv, d, dims, interleaved, dtype = case
    q, k = U.rows(1, B, Hq, L, d, dtype=dtype), U.rows(2, B, Hkv, L, d, dtype=dtype, gain=3.0)
    at = _positions(3, B, L)
    freq = binding.logquant_rope_frequencies(dims, stretch=8.0, original=8192.0, slow=1.0, fast=4.0)
    rope = binding.Rope(freq, interleaved, 1.25, U.DEVICE)
    Q, K, P = q.to(U.DEVICE), k.to(U.DEVICE), at.to(U.DEVICE)
    q_out, k_out = binding.rotate(rope, P, Q, K)
    assert torch.equal(Q.cpu(), q) and torch.equal(K.cpu(), k)
    _check(q_out, q, at.numpy(), freq, interleaved, 1.25, dtype)
    _check(k_out, k, at.numpy(), freq, interleaved, 1.25, dtype)
    one, _ = binding.rotate(rope, P, q=Q)
    _, two = binding.rotate(rope, P, k=K)
    assert torch.equal(one, q_out) and torch.equal(two, k_out)
    again = binding.rotate(rope, P, Q, K, Q, K)                # in place
    assert again[0] is Q and again[1] is K and torch.equal(Q, q_out) and torch.equal(K, k_out)


def test_positions_by_default_and_queries_of_one_token():
    rope = binding.Rope(binding.logquant_rope_frequencies(64), device=U.DEVICE)
    k = U.rows(1, 2, 3, 40, 64, dtype="bf16").to(U.DEVICE)
    at = torch.arange(40, dtype=torch.int32, device=U.DEVICE).repeat(2, 1)
    assert torch.equal(binding.rotate(rope, None, k=k)[1], binding.rotate(rope, at, k=k)[1])
    q, at = U.rows(2, 5, 3, 64, dtype="bf16").to(U.DEVICE), torch.arange(5, dtype=torch.int32, device=U.DEVICE)
    assert torch.equal(binding.rotate(rope, at, q)[0], binding.rotate(rope, at[:, None].contiguous(), q[:, :, None].contiguous())[0][:, :, 0])


def test_position_nothing_and_back():
    """Position 0 changes no bit; a position and its negative leave what two roundings do."""
    rope = binding.Rope(binding.logquant_rope_frequencies(96), device=U.DEVICE)
    x = U.rows(1, 1, 2, 50, 96, dtype="f16").to(U.DEVICE)
    zero = torch.zeros((1, 50), dtype=torch.int32, device=U.DEVICE)
    assert torch.equal(binding.rotate(rope, zero, x)[0], x)
    there = binding.rotate(rope, zero + 12345, x)[0]
    back = binding.rotate(rope, zero - 12345, there)[0]
    one, two = paged.partners(96, False)
    size = U.f64(x)
    size = np.hypot(size[..., one], size[..., two])
    size = np.concatenate([size, size], -1)
    # a rounding of either channel of a pair, each within half a step of the pair's length, turned back, and the last one
    assert (np.abs(U.f64(back) - U.f64(x)) <= (2 * 2 ** 0.5 + 0.1) * 2.0 ** -11 * size + 4 * U.TINY["f16"]).all()


def test_refusals():
    rope = binding.Rope(binding.logquant_rope_frequencies(64), device=U.DEVICE)
    q = U.rows(1, 2, 3, 4, 64, dtype="f16").to(U.DEVICE)
    at = torch.zeros((2, 4), dtype=torch.int32, device=U.DEVICE)
    for kw in (dict(), dict(q=q.float()), dict(q=q.transpose(1, 2)), dict(q=q.cpu()), dict(q=q, q_out=q[:, :2].contiguous()),
               dict(q=q, k=q.bfloat16()), dict(q=q, k=q[:1].contiguous()), dict(q=q, k_out=q), dict(q=q, positions=at.long()),
               dict(q=q, positions=at[:, :3].contiguous()), dict(q=q, positions=at.cpu()), dict(q=q[0, 0])):
        with pytest.raises(ValueError):
            binding.rotate(rope, **kw)
    with pytest.raises(binding.LogQuantError):
        binding.rotate(binding.Rope([1.0] * 33, device=U.DEVICE), at, q)
    with pytest.raises(binding.LogQuantError):
        binding.rotate(rope, q=torch.zeros((1, 1, 1, 80), dtype=torch.float16, device=U.DEVICE))
