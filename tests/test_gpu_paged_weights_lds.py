"""Weighted caches whose logits stay in LDS: all rows against the oracle, with one and two sets of query heads, every kind of score,
entries that are no pages, and steps."""
import numpy as np
import pytest
import torch

from paper_2503_19950_amd import binding
from tests import gpu_util_paged as U

pytestmark = pytest.mark.gpu

CASES = [  # lengths, Hq, Hkv, d, page, dtype: more items than are split, logits that fit
    ([500] * 33, 192, 8, 64, 32, "f16"), ([300 - 7 * b % 290 for b in range(40)], 136, 8, 96, 64, "bf16"), ([400] * 17, 512, 16, 128, 128, "f16"),
    ([33 + 13 * b % 200 for b in range(70)], 16, 4, 128, 32, "bf16"), ([64] * 300, 2, 1, 64, 64, "f16"),
]
SCORES = [dict(), dict(softcap=20.0, slopes=True, window=45)]


@pytest.mark.parametrize("how", SCORES, ids=str)
@pytest.mark.parametrize("case", CASES, ids=lambda c: "%d_rows_to_%d_%s" % (len(c[0]), max(c[0]), "_".join(str(x) for x in c[1:])))
def test_all_rows(case, how):
    lengths, Hq, Hkv, d, page, dtype = case
    B, n = len(lengths), max(lengths)
    cache = U.make(B, Hq, Hkv, d, page, dtype, -(-(n + 1) // page), weighted=True)
    cache.reserve([x + 1 for x in lengths])
    K, V = U.rows(1, B, Hkv, n, d, dtype=dtype, outliers=True), U.rows(2, B, Hkv, n, d, dtype=dtype)
    cache.append(K.to(U.DEVICE), V.to(U.DEVICE), lengths)
    model = U.Model(cache, dtype)
    model.append(K, V, lengths)
    how = dict(how)
    if how.pop("slopes", None):
        how["slopes"] = torch.exp2(-8.0 * torch.arange(1, Hq + 1) / Hq)
    on_gpu = {k: v.to(U.DEVICE) if k == "slopes" else v for k, v in how.items()}
    untouched = cache.weights.view(torch.int32).clone()
    q = U.rows(3, B, Hq, d, dtype=dtype)
    out = cache.decode_attn(q.to(U.DEVICE), **on_gpu)
    model.check_output(out, q, weights=U.live_weights(cache), **how)
    K, V, q = U.rows(4, B, Hkv, 1, d, dtype=dtype), U.rows(5, B, Hkv, 1, d, dtype=dtype), U.rows(6, B, Hq, d, dtype=dtype)
    rope = binding.Rope(binding.logquant_rope_frequencies(d), device=U.DEVICE)
    at = torch.tensor(lengths, dtype=torch.int32, device=U.DEVICE)
    tq, tk = (x.cpu() for x in binding.rotate(rope, at, q[:, :, None].contiguous().to(U.DEVICE), K.to(U.DEVICE)))
    out = cache.decode_step(K.to(U.DEVICE), V.to(U.DEVICE), q.to(U.DEVICE), rope=rope, **on_gpu)
    model.append(tk, V)
    model.check_output(out, tq[:, :, 0], weights=U.live_weights(cache), **how)
    now = cache.weights.view(torch.int32)
    assert torch.equal(now[1], untouched[1])
    for b, x in enumerate(cache.counts()):
        assert torch.equal(now[0, b, :, x:], untouched[0, b, :, x:])


def test_entries_that_are_no_pages():
    B, Hq, Hkv, d, page, dtype = 34, 48, 8, 64, 32, "f16"
    cache = U.make(B, Hq, Hkv, d, page, dtype, 5, weighted=True)
    lengths = [90 + b for b in range(B)]
    cache.reserve(lengths)
    K, V = U.rows(1, B, Hkv, max(lengths), d, dtype=dtype), U.rows(2, B, Hkv, max(lengths), d, dtype=dtype)
    cache.append(K.to(U.DEVICE), V.to(U.DEVICE), lengths)
    model = U.Model(cache, dtype)
    model.append(K, V, lengths)
    cache.table[0, 1, :4] = -1                                           # no page at all
    cache.table[0, 5, 1] = cache.cfg.n_pages                             # tokens 32 .. 63 have none
    q = U.rows(3, B, Hq, d, dtype=dtype)
    out = cache.decode_attn(q.to(U.DEVICE))
    w = U.live_weights(cache)
    assert (out[1] == 0).all() and (w[1, :, :lengths[1]] == 0).all() and (w[5, :, 32:64] == 0).all()
    model.K[5], model.V[5], model.w[5] = (np.delete(x[5], np.s_[32:64], 1) for x in (model.K, model.V, model.w))
    w[5, :, 32:lengths[5] - 32] = w[5, :, 64:lengths[5]].copy()
    model.check_output(out, q, weights=w, skip=(1,))
