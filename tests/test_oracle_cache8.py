"""Pins of oracle/cache8.py: the e4m3 rounding against torch's, scales against their definition, layouts as permutations."""
import numpy as np
import pytest
import torch

from oracle import cache8


def test_rounding_is_torch_s_for_every_16_bit_value_within_range():
    for dt in (torch.float16, torch.bfloat16):
        x = torch.arange(-2 ** 15, 2 ** 15, dtype=torch.int32).to(torch.int16).view(dt).float()
        x = x[torch.isfinite(x) & (x.abs() <= 448)]
        assert np.array_equal(cache8.to_bytes(x.double().numpy()), x.to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    u = np.array([i for i in range(256) if i & 127 != 127], np.uint8)
    assert np.array_equal(cache8.from_bytes(u), torch.from_numpy(u).view(torch.float8_e4m3fn).double().numpy())
    assert np.array_equal(cache8.to_bytes(cache8.from_bytes(u)), u)


def test_rounding_picks_the_nearest_and_the_even_of_two():
    v = cache8.VALUES
    mid = (v[1:] + v[:-1]) / 2
    even = np.where(np.arange(126) % 2 == 0, np.arange(126), np.arange(126) + 1)
    assert np.array_equal(cache8.to_bytes(mid), even.astype(np.uint8))
    assert np.array_equal(cache8.to_bytes(mid * (1 - 1e-12)), np.arange(126).astype(np.uint8))
    assert np.array_equal(cache8.to_bytes(mid * (1 + 1e-12)), np.arange(1, 127).astype(np.uint8))


@pytest.mark.parametrize("top,want", [(448.0, 1.0), (448.0001, 2.0), (224.0, 0.5), (0.0, 2.0 ** -126), (1.75, 2.0 ** -8), (1.7500001, 2.0 ** -7),
                                      (cache8.cut("f16"), 2.0 ** 8), (cache8.cut("bf16"), 2.0 ** 120)])
def test_scales(top, want):
    assert cache8.scale_of(top) == want


@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("which", ["k", "v"])
def test_layouts_are_permutations_unit_by_unit(which, d):
    t, c = np.arange(128)[:, None], np.arange(d)[None]
    i = cache8.code_index(which, t, c, d)
    assert np.array_equal(np.sort(i.ravel()), np.arange(128 * d))
    assert np.array_equal(i // (32 * d), np.broadcast_to(t // 32, i.shape))
    i = cache8.tail_index(which, t, c, d)
    assert np.array_equal(np.sort(i.ravel()), np.arange(128 * d))


def test_values_read_back_stay_in_the_type_and_within_half_a_step():
    rng = np.random.default_rng(5)
    for dtype, dt in (("f16", torch.float16), ("bf16", torch.bfloat16)):
        for gain in (1.0, 1e-6, 3e4):
            x = torch.from_numpy(rng.standard_normal((96, 64)) * gain).to(dt)
            if dtype == "f16":
                x = x.clamp(-65504, 65504)
            c = cache8.Cache8(32, 64, dtype)
            c.append(x.double().numpy())
            held = c.held()
            assert np.array_equal(torch.from_numpy(held).to(dt).double().numpy(), held)
            x = np.clip(x.double().numpy(), -cache8.cut(dtype), cache8.cut(dtype))
            s = np.repeat([cache8.scale_of(np.abs(b).max()) for b in x.reshape(3, 32, 64)], 32)[:, None]
            # half a step: 2^-4 of a normal code's value, 2^-10 of the scale below
            assert (np.abs(held - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * s)).all()
