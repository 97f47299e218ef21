"""Counts set back into a block that has just become full: its rows are in the tail, whichever call filled it up, as long as the
block had rows there before and the call ended with it."""
import numpy as np
import pytest
import torch

from tests import gpu_util8 as U

pytestmark = pytest.mark.gpu
CASES = [(d, G, dtype) for d in (64, 96, 128) for G in (32, 64, 128) for dtype in ("f16", "bf16")]


def check_reading(cache, oracle):
    k, v = cache.read(0, max(cache.counts()))
    for b, n in enumerate(cache.counts()):
        for h in range(cache.cfg.Hkv):
            assert np.array_equal(U.f64(k[b, h, :n]), oracle.k[b][h].held()), (b, h)
            assert np.array_equal(U.f64(v[b, h, :n]), oracle.v[b][h].held()), (b, h)


@pytest.mark.parametrize("way", ["append", "step"])
@pytest.mark.parametrize("d,G,dtype", CASES)
def test_into_a_block_that_a_call_has_filled_up(d, G, dtype, way):
    """Rows whose tails hold 1, some or all but one of a block's rows, in the first block or behind two; one call (or one step)
    fills them up; the counts go back to anywhere in the block, and other tokens follow."""
    helds = [1, 2, 17, G // 2 + 3, G - 2, G - 1, 2 * G + 5, 3 * G - 1] if way == "append" else [G - 1, 2 * G - 1, 3 * G - 1]
    B, Hkv, Hq = len(helds), 2, 4
    fill = [-n % G for n in helds]
    for keep in (0, 1, G // 2, G - 1):                   # rows of the filled block that stay
        cache = U.make(B, Hq, Hkv, d, G, dtype, 5 * G)
        oracle = U.Oracle(cache, dtype)
        K, V = (U.rows(701 + j, B, Hkv, max(helds), d, dtype) for j in range(2))
        cache.append(K.to(U.DEVICE), V.to(U.DEVICE), helds)
        oracle.append(K, V, helds)
        K, V = (U.rows(711 + j, B, Hkv, max(fill), d, dtype) for j in range(2))
        q = U.rows(720, B, Hq, 1, d, dtype, outliers=False)[:, :, 0].contiguous()
        if way == "append":
            cache.append(K.to(U.DEVICE), V.to(U.DEVICE), fill)
        else:
            cache.decode_step(K.to(U.DEVICE), V.to(U.DEVICE), q.to(U.DEVICE))
        oracle.append(K, V, fill)
        oracle.check(cache)
        back = [n - G + keep for n in cache.counts()]
        cache.set_counts(back)
        for b in range(B):
            for h in range(Hkv):
                for o in (oracle.k[b][h], oracle.v[b][h]):
                    o.rows = o.rows[:back[b]]
        oracle.check(cache)
        check_reading(cache, oracle)
        U.check_output(cache.decode_attn(q.to(U.DEVICE)), q, oracle, dtype)
        K, V = (U.rows(731 + j, B, Hkv, G + 9, d, dtype) for j in range(2))
        take = [1, G - keep, G + 9, G - keep, G - keep - 1 if keep < G - 1 else 1, 3, 0, G + 8][:B]
        cache.append(K.to(U.DEVICE), V.to(U.DEVICE), take)
        oracle.append(K, V, take)
        oracle.check(cache)
        check_reading(cache, oracle)


@pytest.mark.parametrize("d,G,dtype", CASES[::5])
def test_steps_again_from_a_count_set_back(d, G, dtype):
    """A draft that was rejected: three steps fill a block up and go back, three others take their place."""
    B, Hkv, Hq = 2, 2, 4
    cache = U.make(B, Hq, Hkv, d, G, dtype, 4 * G)
    oracle = U.Oracle(cache, dtype)
    start = [G - 3, 2 * G - 3]
    K, V = (U.rows(741 + j, B, Hkv, max(start), d, dtype) for j in range(2))
    cache.append(K.to(U.DEVICE), V.to(U.DEVICE), start)
    oracle.append(K, V, start)
    for draft in range(3):
        for step in range(3):
            k, v = (U.rows(750 + 10 * draft + 3 * j + step, B, Hkv, 1, d, dtype) for j in range(2))
            q = U.rows(790 + step, B, Hq, 1, d, dtype, outliers=False)[:, :, 0].contiguous()
            out = cache.decode_step(k.to(U.DEVICE), v.to(U.DEVICE), q.to(U.DEVICE))
            oracle.append(k, v)
            U.check_output(out, q, oracle, dtype)
        oracle.check(cache)
        cache.set_counts(start)
        for b in range(B):
            for h in range(Hkv):
                for o in (oracle.k[b][h], oracle.v[b][h]):
                    o.rows = o.rows[:start[b]]
        oracle.check(cache)
