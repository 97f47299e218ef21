"""Attention over the 8-bit cache to what two operands for the probabilities give: bounds without room for a rounding of the
probabilities themselves, over short rows of small logits, where nothing else hides it."""
import numpy as np
import pytest
import torch

from tests import gpu_util8 as U
from tests.test_gpu_cache8_state import build

CASES = [(d, G, dtype) for d, G in ((64, 32), (96, 64), (128, 32), (128, 128)) for dtype in ("f16", "bf16")]


def attention_and_tight_bound(q, K, V, dtype):
    """fp64 attention of q [g][d] over K, V [n][d], and how far a kernel's output may be from it.  With A = sum p |v|:
      a probability is the sum of fp16 operands, the second one of what the first one's rounding left: off by at most 2^-22
        of itself, and by 2^-25 where it falls below fp16's normal numbers; the largest of a wavefront's is 2^10 at least, so
        that is 2^-35 of the largest (the tail's three bf16 operands are off by 2^-27);
      logits: fp32 sums of d exact products, each addition off by at most 2^-23 of the products' magnitudes (an addition
        inside a matrix instruction may cut off), three roundings of the logit, its factor and its reference, 2^-22 of
        the power of two; a relative error e of every weight moves the output by at most 2 e A;
      the sums of 32 products for each of two or three operands, 2^-23 an addition; of n/32 units and of up to 16 wavefronts'
        or 128 parts' results, 2^-24 each; of the probabilities themselves, n/4 a lane, 2^-24 each;
      the rounding of the output to T: half a step, or half of T's smallest number."""
    q, K, V = U.f64(q), np.asarray(K), np.asarray(V)
    d, n = q.shape[-1], len(K)
    s = d ** -0.5 * (q @ K.T)
    p = np.exp(s - s.max(-1, keepdims=True))
    total = p.sum(-1, keepdims=True)
    o, A = p @ V / total, p @ np.abs(V) / total
    lost = 2.0 ** -35 * np.abs(V).sum(0) / total                       # (the largest p is 1)
    spread = d ** -0.5 * (np.abs(q) @ np.abs(K).T).max(-1, keepdims=True)
    e = d * 2.0 ** -23 * spread + 3 * 2.0 ** -23 * np.abs(s).max(-1, keepdims=True) + 2.0 ** -22
    inner = A * (2.0 ** -22 + 2 * e + 96 * 2.0 ** -23 + (n / 32 + 144 + n / 4) * 2.0 ** -24) + lost
    return o, inner + U.HALF_STEP[dtype] * (np.abs(o) + inner) + (2.0 ** -25 if dtype == "f16" else 0)


def small_logits(seed, lengths, Hq, d, G, dtype):
    """A cache of kv heads with eight query heads each whose keys and queries give logits so small that their own rounding stays below that of a probability to fp16."""
    B, Hkv, top = len(lengths), Hq // 8, max(lengths)
    cache = U.make(B, Hq, Hkv, d, G, dtype, (top // G + 2) * G)
    oracle = U.Oracle(cache, dtype)
    K, V = (U.rows(seed + i, B, Hkv, top, d, dtype, outliers=False) for i in range(2))
    q = U.rows(seed + 2, B, Hq, 1, d, dtype, 0.03, outliers=False)[:, :, 0].contiguous()
    oracle.append(K, V, lengths)
    cache.append(K.to(U.DEVICE), V.to(U.DEVICE), lengths)
    return cache, oracle, q


def check(out, q, oracle, dtype):
    cfg = oracle.cfg
    gh, got = cfg.Hq // cfg.Hkv, U.f64(out)
    for b in range(cfg.B):
        for h in range(cfg.Hkv):
            at = slice(h * gh, (h + 1) * gh)
            want, bound = attention_and_tight_bound(q[b, at], oracle.k[b][h].held(), oracle.v[b][h].held(), dtype)
            over = np.abs(got[b, at] - want) / bound
            assert (over <= 1).all(), "row %d kv head %d: %.2f bounds, %d of %d outside" % (b, h, over.max(), (over > 1).sum(), over.size)


@pytest.mark.parametrize("terms", [1, 2])
def test_the_bound_tells_one_operand_from_two(terms):
    """The rounding planted into the 64-bit form: probabilities as one fp16 number break the bound, as two they keep it."""
    rng = np.random.default_rng(1)
    d, n, broken = 128, 64, 0
    for dtype in ("f16", "bf16"):
        q, K, V = (torch.from_numpy(rng.standard_normal((m, d)) * gain).to(U.TYPES[dtype]) for m, gain in ((8, 0.03), (n, 1), (n, 1)))
        s = d ** -0.5 * (U.f64(q) @ U.f64(K).T)
        p = np.exp(s - s.max(-1, keepdims=True)) * 2.0 ** 10
        used = np.zeros_like(p)
        for _ in range(terms):
            used += (p - used).astype(np.float16).astype(np.float64)
        got = torch.from_numpy(used @ U.f64(V) / p.sum(-1, keepdims=True)).to(U.TYPES[dtype])
        want, bound = attention_and_tight_bound(q, U.f64(K), U.f64(V), dtype)
        broken += (np.abs(U.f64(got) - want) > bound).sum() > 0
    assert broken == (2 if terms == 1 else 0)


@pytest.mark.gpu
@pytest.mark.parametrize("d,G,dtype", CASES)
def test_rows_of_codes_and_of_the_tail(d, G, dtype):
    lengths = [G, G - 1, 4 * G, 3, 2 * G + G // 2, 32, 4 * G - 1]
    cache, oracle, q = small_logits(501, lengths, 16, d, G, dtype)
    check(cache.decode_attn(q.to(U.DEVICE)), q, oracle, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("d,G,dtype", CASES)
def test_steps_across_the_end_of_a_block(d, G, dtype):
    cache, oracle, q = small_logits(511, [2 * G - 2, G - 1, 7], 16, d, G, dtype)
    for step in range(3):
        k, v = (U.rows(520 + 10 * i + step, 3, 2, 1, d, dtype, outliers=False) for i in range(2))
        out = cache.decode_step(k.to(U.DEVICE), v.to(U.DEVICE), q.to(U.DEVICE))
        oracle.append(k, v)
        check(out, q, oracle, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_many_parts_and_two_sets_of_heads(dtype):
    """Rows shared by many workgroups (the bound of the sums has room for 144 of them), and more than 16 heads a kv head in one."""
    cache, oracle = build(531, 1, 8, 1, 128, 64, dtype, [1500])
    q = U.rows(533, 1, 8, 1, 128, dtype, 0.03, outliers=False)[:, :, 0].contiguous()
    check(cache.decode_attn(q.to(U.DEVICE)), q, oracle, dtype)
    lengths = [1200 - b for b in range(80)]                            # 24 MB: two sets of heads a workgroup
    cache, oracle = build(541, 80, 24, 1, 128, 32, dtype, lengths)
    q = U.rows(543, 80, 24, 1, 128, dtype, 0.03, outliers=False)[:, :, 0].contiguous()
    check(cache.decode_attn(q.to(U.DEVICE)), q, oracle, dtype)
