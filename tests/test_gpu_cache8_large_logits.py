"""Attention over the 8-bit cache where logits are so large that fp32 no longer tells them from ten more: outputs are finite, a single
token gives its value, equal keys give the mean, and any keys give something between the values."""
import numpy as np
import pytest
import torch

from tests import gpu_util8 as U

pytestmark = pytest.mark.gpu
# With d = 128 the exponent of two is 16.3 q k: 2^24, 2^27 and 2^28, 2^31, 2^34, below 2^24 and negative ones
GAINS = [(1000.0, 1024.0), (3000.0, 2048.0), (4095.0, 4096.0), (12000.0, 8192.0), (30000.0, 32768.0), (100.0, 64.0), (-3000.0, 4096.0)]


def check_mean(out, held, dtype, n_weights):
    """Outputs of equal logits against the mean of the values held: probabilities are equal up to exp2's 2^-22, sums of n terms
    in fp32 are off by at most n 2^-24 of the mean magnitude, two operands by 2^-22; and the output is rounded."""
    want, A = held.mean(0), np.abs(held).mean(0)
    inner = A * (2.0 ** -20 + (n_weights + 64) * 2.0 ** -23)
    bound = inner + U.HALF_STEP[dtype] * (np.abs(want) + inner) + 2.0 ** -25
    off = np.abs(U.f64(out) - want)
    assert (off <= bound).all(), "off by %.3g" % np.nanmax(off) if np.isfinite(off).any() else "not finite"


def equal_keys(seed, lengths, Hq, Hkv, d, G, dtype, k_gain):
    cache = U.make(len(lengths), Hq, Hkv, d, G, dtype, (max(lengths) // G + 2) * G)
    oracle = U.Oracle(cache, dtype)
    V = U.rows(seed, len(lengths), Hkv, max(lengths), d, dtype, outliers=False)
    K = torch.full_like(V, k_gain)
    oracle.append(K, V, lengths)
    cache.append(K.to(U.DEVICE), V.to(U.DEVICE), lengths)
    return cache, oracle


def query(B, Hq, d, dtype, gain):
    return torch.full((B, Hq, d), gain).to(U.TYPES[dtype]).to(U.DEVICE)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("q_gain,k_gain", GAINS)
def test_one_token_gives_its_value(q_gain, k_gain, dtype):
    for n in (1, 32):                                                  # in the tail; 32 equal tokens as a block of codes
        cache = U.make(2, 4, 2, 128, 32, dtype, 64)
        V = U.rows(601, 2, 2, 1, 128, dtype, outliers=False)
        V = torch.exp2(torch.round(torch.log2(V.float().abs() + 0.25))).to(V.dtype) * torch.sign(V)      # exact as codes
        cache.append(*(x.expand(2, 2, n, 128).contiguous().to(U.DEVICE) for x in (torch.full_like(V, k_gain), V)))
        out = cache.decode_attn(query(2, 4, 128, dtype, q_gain)).cpu()
        assert torch.equal(out.view(2, 2, 2, 128), V.expand(2, 2, 2, 128)), n


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("q_gain,k_gain", GAINS)
def test_equal_keys_give_the_mean(q_gain, k_gain, dtype):
    """Rows of the tail, of codes, of both, and one shared by many workgroups."""
    for lengths in ([31, 32, 77, 5, 200], [6000]):
        cache, oracle = equal_keys(611, lengths, 6, 2, 128, 32, dtype, k_gain)
        out = cache.decode_attn(query(len(lengths), 6, 128, dtype, q_gain))
        for b, n in enumerate(lengths):
            for h in range(6):
                check_mean(out[b, h], oracle.v[b][h // 3].held(), dtype, n)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("q_gain,k_gain", GAINS)
def test_steps_across_the_end_of_a_block(q_gain, k_gain, dtype):
    cache, oracle = equal_keys(621, [62, 30, 7], 6, 2, 128, 32, dtype, k_gain)
    for step in range(3):
        v = U.rows(630 + step, 3, 2, 1, 128, dtype, outliers=False)
        k = torch.full_like(v, k_gain)
        out = cache.decode_step(k.to(U.DEVICE), v.to(U.DEVICE), query(3, 6, 128, dtype, q_gain))
        oracle.append(k, v)
        for b in range(3):
            for h in range(6):
                check_mean(out[b, h], oracle.v[b][h // 3].held(), dtype, len(oracle.v[b][0].rows))


@pytest.mark.parametrize("d,Hq,dtype", [(64, 4, "f16"), (96, 8, "bf16"), (128, 4, "f16"), (128, 4, "bf16"), (128, 20, "f16")])
def test_outputs_of_any_keys_lie_between_the_values(d, Hq, dtype):
    """Queries and keys of normal values, with and without common signs, 1e4 and more large; values between 1 and 2."""
    G, lengths = 32, [700, 32, 95, 1, 31, 64]
    for sigma in (1e3, 1e4, 6e4 / 5):
        for common in (False, True):
            cache = U.make(len(lengths), Hq, 1, d, G, dtype, 768)
            q = U.rows(641, len(lengths), Hq, 1, d, dtype, sigma, outliers=False)[:, :, 0].contiguous()
            K = U.rows(642, len(lengths), 1, 700, d, dtype, sigma, outliers=False)
            if common:
                K = K.abs() * torch.sign(q[:, :1, None])
            V = 1 + torch.rand(K.shape, generator=torch.Generator().manual_seed(643))
            cache.append(K.to(U.DEVICE), V.to(K.dtype).to(U.DEVICE), lengths)
            out = cache.decode_attn(q.to(U.DEVICE)).float()
            assert torch.isfinite(out).all() and (out >= 1 - 2 ** -7).all() and (out <= 2 + 2 ** -6).all(), (sigma, common)


def test_far_logits_of_bf16():
    """Exponents of 2^84: still within fp32."""
    cache, oracle = equal_keys(651, [77, 5, 1500], 2, 1, 128, 64, "bf16", 2.0 ** 40)
    for gain in (2.0 ** 40, 3.0 * 2.0 ** 39, -(2.0 ** 40)):
        out = cache.decode_attn(query(3, 2, 128, "bf16", gain))
        for b in range(3):
            for h in range(2):
                check_mean(out[b, h], oracle.v[b][0].held(), "bf16", len(oracle.v[b][0].rows))
