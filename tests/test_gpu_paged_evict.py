"""Eviction by accumulated weight on the GPU, and the operators of the paged cache one after the other."""
import numpy as np
import pytest
import torch

from paper_2503_19950_amd import binding
from tests import gpu_util_paged as U

pytestmark = pytest.mark.gpu


def _filled(seed, lengths, Hkv, d, page, dtype, values, n_pages=None):
    """A weighted cache whose weights are drawn from `values`."""
    B = len(lengths)
    cache = U.make(B, Hkv, Hkv, d, page, dtype, -(-max(lengths) // page) + 2, weighted=True, seed=seed, n_pages=n_pages)
    cache.reserve(lengths)
    K, V = U.rows(seed, B, Hkv, max(lengths), d, dtype=dtype), U.rows(seed + 1, B, Hkv, max(lengths), d, dtype=dtype)
    cache.append(K.to(U.DEVICE), V.to(U.DEVICE), lengths)
    model = U.Model(cache, dtype)
    model.append(K, V, lengths)
    r = np.random.RandomState(seed)
    for b, n in enumerate(lengths):
        w = values(r, (Hkv, n)).astype(np.float32)
        cache.weights[0, b, :, :n] = torch.from_numpy(w).to(U.DEVICE)
        model.w[b] = w.astype(np.float64)
    return cache, model


def _check(cache, model, before):
    U.check_rows(cache, model, before)
    w = U.live_weights(cache)
    for b in range(cache.cfg.B):
        assert np.array_equal(w[b, :, :cache.n[b]], model.w[b])


VALUES = {"spread": lambda r, s: np.exp(4 * r.randn(*s)), "few": lambda r, s: r.randint(0, 4, s) / 4, "none": lambda r, s: np.zeros(s),
          "close": lambda r, s: 1 + r.randint(0, 3, s) * 2.0 ** -23,
          "signs": lambda r, s: r.choice([-2.0, -0.0, 0.0, 1e-42, -1e-42, 3e38, np.inf], s)}

CASES = [  # lengths, Hkv, d, page, keep, recent
    ([40, 200, 0], 2, 64, 32, 33, 5), ([100, 64, 65, 63], 3, 96, 64, 64, 64), ([300], 1, 128, 128, 1, 0), ([300, 299], 1, 128, 32, 299, 298),
    ([3000, 17], 2, 64, 128, 1000, 1), ([70, 30, 31], 2, 64, 32, [69, 0, 31], 0), ([5000, 4097], 1, 64, 32, [4096, 1025], 100),
    ([1 + b * 41 % 300 for b in range(140)], 1, 64, 32, 100, 10),
]


@pytest.mark.parametrize("values", VALUES)
@pytest.mark.parametrize("case", CASES, ids=lambda c: "%d_rows_to_%d_%s" % (len(c[0]), max(c[0]), "_".join(str(x) for x in c[1:])))
def test_evict(case, values):
    lengths, Hkv, d, page, keep, recent = case
    dtype = "f16" if d == 64 else "bf16"
    cache, model = _filled(len(lengths) + d, lengths, Hkv, d, page, dtype, VALUES[values])
    before = U.pools(cache)
    free = len(cache.free)
    other = cache.weights.view(torch.int32).clone()
    cache.evict(keep, recent)
    model.evict(keep, recent)
    limit = [keep] * len(lengths) if isinstance(keep, int) else keep
    assert cache.counts() == [min(n, k) for n, k in zip(lengths, limit)]
    assert list(cache.cur) == [int(n > k) for n, k in zip(lengths, limit)]
    assert free - len(cache.free) == sum(-(-k // page) for n, k in zip(lengths, limit) if n > k)
    # the rows as they were are where they were: only new pages are written
    held = U.Model(cache, dtype)
    held.K, held.V, held.w = model.K, model.V, model.w
    _check(cache, held, before)
    now = cache.weights.view(torch.int32)
    assert torch.equal(now[0], other[0])
    for b, (n, k) in enumerate(zip(lengths, limit)):
        tail = k if n > k else 0
        assert torch.equal(now[1, b, :, tail:], other[1, b, :, tail:])


@pytest.mark.parametrize("values", VALUES)
@pytest.mark.parametrize("lengths,keep,recent,d", [([70001], 33333, 4096, 64), ([16385, 16384, 40, 20001], [300, 9000, 40, 20000], 0, 128),
                                                   ([18500, 100], [2048, 50], 50, 96)])
def test_long_rows(lengths, keep, recent, d, values):
    cache, model = _filled(3, lengths, 1, d, 128, "bf16", VALUES[values])
    before = U.pools(cache)
    cache.evict(keep, recent)
    model.evict(keep, recent)
    _check(cache, model, before)


@pytest.mark.parametrize("lengths,keep,recent,d,page", [([6000, 3000], 200, 7, 96, 64), ([9000], 500, 3, 128, 32), ([4000, 4100], [64, 600], 0, 64, 128)])
def test_few_stay_of_many(lengths, keep, recent, d, page):
    """Tokens of a unit that come from many others."""
    cache, model = _filled(5, lengths, 2, d, page, "f16", VALUES["spread"])
    before = U.pools(cache)
    cache.evict(keep, recent)
    model.evict(keep, recent)
    _check(cache, model, before)


def test_replays_of_a_recorded_eviction():
    """Replayed, it moves the same tokens' places again, by the weights as they are then."""
    lengths, keep, recent = [17000, 300, 90], 200, 20
    cache, model = _filled(13, lengths, 1, 64, 32, "f16", VALUES["spread"])
    cache.reserve([200, 200, 0], spare=True)
    before = U.pools(cache)
    K, V = [x.copy() for x in model.K], [x.copy() for x in model.V]
    halves = list(cache.cur)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        cache.evict(keep, recent)                                        # (code is loaded before the recording)
    stream.synchronize()
    cache.set_counts(lengths, halves)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        cache.evict(keep, recent)
    for i in range(3):
        r = np.random.RandomState(50 + i)
        model.K, model.V = [x.copy() for x in K], [x.copy() for x in V]
        for b, n in enumerate(lengths):
            w = VALUES["few" if i else "spread"](r, (1, n)).astype(np.float32)
            cache.weights[0, b, :, :n] = torch.from_numpy(w).to(U.DEVICE)
            model.w[b] = w.astype(np.float64)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        model.evict(keep, recent)
        _check(cache, model, before)
        q = U.rows(i, 3, 1, 64, dtype="f16")
        model.check_output(cache.decode_attn(q.to(U.DEVICE)), q)         # (adds to the weights of the evicted rows' halves)
        model.w = [x.copy() for x in model.w]


def test_a_page_that_a_row_names_twice():
    cache, model = _filled(9, [64], 1, 64, 32, "f16", VALUES["spread"])
    cache.set_pages(0, cache.ids[0][0] + cache.ids[0][0])
    cache.n[0] = 128
    model.K[0], model.V[0] = (np.concatenate([x[0], x[0]], 1) for x in (model.K, model.V))
    w = np.float32(np.random.RandomState(1).rand(1, 128))
    cache.weights[0, 0, :, :128] = torch.from_numpy(w).to(U.DEVICE)
    for keep, recent in ((100, 50), (70, 0)):
        model.w[0] = w.astype(np.float64)
        one, two = cache.clone(), U.Model(cache, "f16")
        two.K, two.V, two.w = [x.copy() for x in model.K], [x.copy() for x in model.V], [x.copy() for x in model.w]
        before = U.pools(one)
        one.evict(keep, recent)
        two.evict(keep, recent)
        _check(one, two, before)


def test_tokens_without_a_page_become_zeros():
    cache, model = _filled(5, [96], 1, 64, 32, "f16", VALUES["spread"])
    before = U.pools(cache)
    cache.table[0, 0, 1] = -1
    model.K[0][:, 32:64] = model.V[0][:, 32:64] = 0
    cache.evict(80, 40)
    model.evict(80, 40)
    _check(cache, model, before)


def test_an_eviction_without_new_pages_stores_nothing():
    cache, _ = _filled(7, [96], 1, 64, 32, "f16", VALUES["spread"])
    cache.reserve([64], spare=True)
    cache.table[1, 0] = cache.cfg.n_pages
    before = U.pools(cache)
    cache.evict(64, 8)
    now = U.pools(cache)
    assert all(np.array_equal(now[w], before[w]) for w in "kv") and cache.counts() == [64]


def test_evictions_of_one_row_after_the_other():
    """Both halves of the table take their turns; pages go back to the pool."""
    Hkv, d, page, dtype = 2, 96, 32, "f16"
    cache, model = _filled(11, [150, 90], Hkv, d, page, dtype, VALUES["few"], n_pages=17)
    for i, (keep, recent) in enumerate([([100, 90], 10), ([64, 50], 0), ([40, 50], 40), ([39, 1], 1)]):
        before = U.pools(cache)
        cache.evict(keep, recent)
        model.evict(keep, recent)
        _check(cache, model, before)
        for b in range(2):
            cache.release(b, spare=True)
        K, V = U.rows(50 + i, 2, Hkv, 7, d, dtype=dtype), U.rows(60 + i, 2, Hkv, 7, d, dtype=dtype)
        cache.reserve([n + 7 for n in cache.counts()])
        before = U.pools(cache)
        cache.append(K.to(U.DEVICE), V.to(U.DEVICE))
        model.append(K, V)
        _check(cache, model, before)
    assert len(cache.free) == 17 - sum(len(x) for half in cache.ids for x in half)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_the_life_of_a_batch(dtype):
    """Prompts rotated on their way, steps, attention, eviction, and on."""
    B, Hq, Hkv, d, page = 3, 8, 2, 128, 64
    lengths = [200, 77, 0]
    cache = U.make(B, Hq, Hkv, d, page, dtype, 6, n_pages=18, weighted=True)
    model = U.Model(cache, dtype)
    rope = binding.Rope(binding.logquant_rope_frequencies(64, stretch=4.0), True, device=U.DEVICE)
    slopes = torch.exp2(-torch.arange(1.0, Hq + 1))
    how, on_gpu = dict(softcap=20.0, slopes=slopes), dict(softcap=20.0, slopes=slopes.to(U.DEVICE))
    K, V = U.rows(1, B, Hkv, 200, d, dtype=dtype, outliers=True), U.rows(2, B, Hkv, 200, d, dtype=dtype)
    cache.reserve([n + 40 for n in lengths])
    cache.append(K.to(U.DEVICE), V.to(U.DEVICE), lengths, rope=rope)
    model.append(binding.rotate(rope, None, k=K.to(U.DEVICE))[1].cpu(), V, lengths)
    places = torch.tensor(lengths, dtype=torch.int32, device=U.DEVICE)
    for i in range(30):
        K, V, q = U.rows(100 + i, B, Hkv, 1, d, dtype=dtype), U.rows(200 + i, B, Hkv, 1, d, dtype=dtype), U.rows(300 + i, B, Hq, d, dtype=dtype)
        tq, tk = (x.cpu() for x in binding.rotate(rope, places, q[:, :, None].contiguous().to(U.DEVICE), K.to(U.DEVICE)))
        out = cache.decode_step(K.to(U.DEVICE), V.to(U.DEVICE), q.to(U.DEVICE), rope=rope, positions=places, **on_gpu)
        model.append(tk, V)
        model.check_output(out, tq[:, :, 0], weights=U.live_weights(cache), **how)
        places += 1
        if i in (9, 19):
            before = U.pools(cache)
            cache.evict(64 + i, 16)
            model.evict(64 + i, 16)
            _check(cache, model, before)
            for b in range(B):
                cache.release(b, spare=True)
            cache.reserve([n + 20 for n in cache.counts()])
    assert cache.counts() == [93, 93, 30]
