"""Attention over the paged cache on the GPU against the oracle."""
import numpy as np
import pytest
import torch

from paper_2503_19950_amd import binding
from tests import gpu_util_paged as U

pytestmark = pytest.mark.gpu


def _filled(seed, lengths, Hq, Hkv, d, page, dtype, weighted=False, more=1, gain=1.0):
    B = len(lengths)
    cache = U.make(B, Hq, Hkv, d, page, dtype, -(-(max(lengths) + more) // page), weighted=weighted, seed=seed)
    cache.reserve([n + more for n in lengths])
    model = U.Model(cache, dtype)
    n = max(max(lengths), 1)
    K, V = U.rows(seed, B, Hkv, n, d, dtype=dtype, gain=gain, outliers=True), U.rows(seed + 1, B, Hkv, n, d, dtype=dtype)
    cache.append(K.to(U.DEVICE), V.to(U.DEVICE), lengths)
    model.append(K, V, lengths)
    return cache, model


CASES = [  # lengths, Hq, Hkv, d, page, dtype
    ([1], 1, 1, 64, 32, "f16"), ([1, 2, 31, 32, 33, 0], 4, 2, 128, 32, "bf16"), ([63, 64, 65], 8, 1, 96, 64, "f16"),
    ([127, 128, 129, 0], 3, 1, 64, 128, "bf16"), ([300, 5, 1000], 32, 8, 128, 64, "f16"), ([520], 32, 8, 128, 64, "bf16"),
    # more than 16 heads of a kv head: two groups, and two sets of one where much is read
    ([200, 40], 17, 1, 64, 32, "f16"), ([333], 40, 1, 128, 128, "bf16"), ([16, 700], 33, 1, 96, 32, "f16"), ([30000], 24, 1, 128, 64, "bf16"),
    ([9000] * 8, 48, 2, 64, 128, "f16"),
    # parts, joined at once and by sixteens; rows of different lengths in parts, in larger workgroups, and many of them
    ([20000], 4, 1, 64, 32, "f16"), ([8000, 3000], 8, 1, 128, 64, "bf16"), ([17] * 300, 1, 1, 64, 32, "bf16"),
    ([b * 37 % 400 for b in range(150)], 2, 1, 96, 32, "f16"), ([1 + b * 997 % 2000 for b in range(40)], 16, 8, 64, 64, "f16"),
    ([1 + b * 997 % 2000 for b in range(40)], 4, 4, 128, 128, "bf16"), ([700] * 33, 8, 8, 64, 32, "f16"),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "%d_rows_to_%d_%s" % (len(c[0]), max(c[0]), "_".join(str(x) for x in c[1:])))
def test_attention(case):
    lengths, Hq, Hkv, d, page, dtype = case
    cache, model = _filled(len(lengths) + d, *case)
    q = U.rows(7, len(lengths), Hq, d, dtype=dtype)
    out = cache.decode_attn(q.to(U.DEVICE))
    model.check_output(out, q)
    assert torch.equal(cache.decode_attn(q.to(U.DEVICE)), out)           # the same bits again
    model.check_output(cache.decode_attn(q.to(U.DEVICE), softmax_scale=0.25), q, scale=0.25)


SCORES = [dict(softcap=30.0), dict(softcap=0.5), dict(softcap=1000.0), dict(window=1), dict(window=32), dict(window=33), dict(window=100),
          dict(window=5000), dict(slopes=True), dict(softcap=5.0, slopes=True, window=70)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("how", SCORES, ids=str)
def test_scores(how, dtype):
    lengths, Hq, Hkv, d, page = [1, 32, 40, 101, 513, 0, 3000], 6, 2, 96, 32
    cache, model = _filled(3, lengths, Hq, Hkv, d, page, dtype, gain=2.0)
    q = U.rows(8, len(lengths), Hq, d, dtype=dtype)
    how = dict(how)
    if how.get("slopes"):
        how["slopes"] = torch.tensor([0.5, 0.25, 0.0625, 0.0, -0.001, 4.0])
    on_gpu = dict(how, slopes=how["slopes"].to(U.DEVICE)) if "slopes" in how else how
    model.check_output(cache.decode_attn(q.to(U.DEVICE), **on_gpu), q, **how)


@pytest.mark.parametrize("heads", [(20, 1), (6, 3)])
def test_what_is_masked_may_be_anything(heads):
    """Slots behind a row's length, and tokens before its window, hold NaN and infinities."""
    Hq, Hkv = heads
    dtype, d, page = "f16", 64, 64
    cache, model = _filled(5, [100, 77, 200], Hq, Hkv, d, page, dtype)
    for w in "kv":
        pool = getattr(cache, w + "_pages").view(torch.float16)
        for b in range(3):
            seen = [U.addresses(cache, w, b, h, cache.n[b])[max(0, cache.n[b] - 50):] for h in range(Hkv)]
            rest = np.concatenate([U.addresses(cache, w, b, h, cache.n[b]).ravel() for h in range(Hkv)])
            rest = np.setdiff1d(rest, np.concatenate([x.ravel() for x in seen]))
            pool[torch.from_numpy(rest[::2].copy()).to(U.DEVICE)] = float("inf")
            pool[torch.from_numpy(rest[1::2].copy()).to(U.DEVICE)] = float("nan")
    q = U.rows(9, 3, Hq, d, dtype=dtype)
    model.check_output(cache.decode_attn(q.to(U.DEVICE), window=50), q, window=50)


@pytest.mark.parametrize("dims,interleaved,positions", [(0, False, False), (96, False, False), (96, False, True), (30, True, True)])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_step_is_rotate_append_attend(dims, interleaved, positions, dtype):
    lengths, Hq, Hkv, d, page = [0, 1, 31, 32, 63, 64, 500], 6, 2, 96, 64
    cache, model = _filled(11, lengths, Hq, Hkv, d, page, dtype, more=70)
    B = len(lengths)
    rope = binding.Rope(binding.logquant_rope_frequencies(dims), interleaved, 1.5, U.DEVICE) if dims else None
    before = U.pools(cache)
    for i in range(4):
        K, V, q = (U.rows(20 + 3 * i + x, B, *((Hkv, 1) if x < 2 else (Hq,)), d, dtype=dtype) for x in range(3))
        at = torch.randint(0, 1 << 17, (B,), generator=torch.Generator().manual_seed(i), dtype=torch.int32).to(U.DEVICE) if positions else None
        places = at if positions else torch.tensor(cache.counts(), dtype=torch.int32, device=U.DEVICE)
        tq, tk = (x.cpu() for x in binding.rotate(rope, places, q[:, :, None].contiguous().to(U.DEVICE), K.to(U.DEVICE))) if dims else (q[:, :, None], K)
        out = cache.decode_step(K.to(U.DEVICE), V.to(U.DEVICE), q.to(U.DEVICE), rope=rope, positions=at, window=i * 20)
        model.append(tk, V)
        U.check_rows(cache, model, before)
        model.check_output(out, tq[:, :, 0], window=i * 20)


@pytest.mark.parametrize("heads,lengths", [((24, 1), [40, 3000]), ((17, 1), [9000]), ((16, 16), [100] * 3), ((32, 8), [4000] * 9), ((4, 4), [1 + 97 * b % 900 for b in range(70)]),
                                           ((2, 1), [37 * b % 200 for b in range(260)])])
def test_steps_of_other_shapes(heads, lengths):
    Hq, Hkv = heads
    dtype, d, page, B = "bf16", 128, 32, len(lengths)
    cache, model = _filled(13, lengths, Hq, Hkv, d, page, dtype)
    rope = binding.Rope(binding.logquant_rope_frequencies(d), device=U.DEVICE)
    K, V, q = U.rows(1, B, Hkv, 1, d, dtype=dtype), U.rows(2, B, Hkv, 1, d, dtype=dtype), U.rows(3, B, Hq, d, dtype=dtype)
    before = U.pools(cache)
    places = torch.tensor(cache.counts(), dtype=torch.int32, device=U.DEVICE)
    tq, tk = (x.cpu() for x in binding.rotate(rope, places, q[:, :, None].contiguous().to(U.DEVICE), K.to(U.DEVICE)))
    out = cache.decode_step(K.to(U.DEVICE), V.to(U.DEVICE), q.to(U.DEVICE), rope=rope)
    model.append(tk, V)
    U.check_rows(cache, model, before)
    model.check_output(out, tq[:, :, 0])


@pytest.mark.parametrize("how", [dict(), dict(softcap=8.0, window=60)], ids=str)
@pytest.mark.parametrize("heads", [(1, 1), (6, 2), (17, 1)])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_weights_add_up(how, heads, dtype):
    Hq, Hkv = heads
    lengths, d, page = [0, 1, 30, 64, 1100, 5000], 64, 32
    cache, model = _filled(17, lengths, Hq, Hkv, d, page, dtype, weighted=True, more=10)
    B = len(lengths)
    untouched = cache.weights.view(torch.int32).clone()
    for i in range(3):
        q = U.rows(30 + i, B, Hq, d, dtype=dtype)
        out = cache.decode_attn(q.to(U.DEVICE), **how)
        model.check_output(out, q, weights=U.live_weights(cache), **how)
        K, V = U.rows(40 + i, B, Hkv, 1, d, dtype=dtype), U.rows(50 + i, B, Hkv, 1, d, dtype=dtype)
        out = cache.decode_step(K.to(U.DEVICE), V.to(U.DEVICE), q.to(U.DEVICE), **how)
        model.append(K, V)
        model.check_output(out, q, weights=U.live_weights(cache), **how)
    now = cache.weights.view(torch.int32)
    assert torch.equal(now[1], untouched[1])                              # the other half
    for b in range(B):
        assert torch.equal(now[0, b, :, cache.n[b]:], untouched[0, b, :, cache.n[b]:])


# logits in LDS: rows of one length in workgroups of 4 wavefronts, of different lengths in larger ones, up to what a compute unit has;
# through memory: longer rows, shared kv heads, split items
@pytest.mark.parametrize("lengths,heads,d", [([500] * 40, (32, 8), 64), ([4096 - 61 * b % 3000 for b in range(36)], (32, 8), 128),
                                             ([1 + 37 * b % 700 for b in range(40)], (40, 8), 96), ([3000 - 90 * b for b in range(20)], (64, 16), 64),
                                             ([200] * 33, (8, 8), 96), ([700] * 9, (68, 2), 64), ([9000, 50], (4, 2), 64),
                                             ([4500] * 40, (32, 8), 64), ([8000 - 100 * b for b in range(36)], (32, 8), 64)])
@pytest.mark.parametrize("window", [0, 90])
def test_weights_by_every_route(lengths, heads, d, window):
    Hq, Hkv = heads
    B, dtype = len(lengths), "f16"
    cache, model = _filled(31, lengths, Hq, Hkv, d, 32, dtype, weighted=True)
    untouched = cache.weights.view(torch.int32).clone()
    q = U.rows(1, B, Hq, d, dtype=dtype)
    out = cache.decode_attn(q.to(U.DEVICE), window=window)
    for b in range(4, B - 2):                                            # (some rows are enough)
        model.K[b], model.V[b] = model.K[b][:, :0], model.V[b][:, :0]
    some = [b for b in range(B) if 4 <= b < B - 2]
    model.check_output(out, q, window=window, weights=U.live_weights(cache), skip=some)
    now = cache.weights.view(torch.int32)
    for b in range(B):
        assert torch.equal(now[0, b, :, cache.n[b]:], untouched[0, b, :, cache.n[b]:])
        if window and cache.n[b] > window:
            assert (now[0, b, :, :cache.n[b] - window] == 0).all()
        # all of a head's probabilities, whatever their number: each is off by less than 2^-20 of itself, as are the sums
        w = cache.weights[0, b, :, :cache.n[b]].double().sum(-1)
        assert (w - Hq / Hkv).abs().max() < 2.0 ** -18 * Hq / Hkv
    K, V = U.rows(2, B, Hkv, 1, d, dtype=dtype), U.rows(3, B, Hkv, 1, d, dtype=dtype)
    again = cache.decode_step(K.to(U.DEVICE), V.to(U.DEVICE), q.to(U.DEVICE), window=window)
    assert torch.isfinite(again).all()
    for b in range(B):
        w = cache.weights[0, b, :, :cache.n[b]].double().sum(-1)
        assert (w - 2 * Hq / Hkv).abs().max() < 2.0 ** -17 * Hq / Hkv


def test_a_step_without_a_page_for_its_token():
    """Nothing is stored, and nothing but the tokens that have a page gets weight."""
    dtype = "bf16"
    cache, model = _filled(37, [64, 70], 4, 2, 96, 32, dtype, weighted=True, more=30)
    cache.table[0, 0, 2] = -1                                            # row 0: of the new token alone
    cache.table[0, 1, 2] = cache.cfg.n_pages                             # row 1: of the six before it as well
    before = U.pools(cache)
    K, V, q = U.rows(1, 2, 2, 1, 96, dtype=dtype), U.rows(2, 2, 2, 1, 96, dtype=dtype), U.rows(3, 2, 4, 96, dtype=dtype)
    rope = binding.Rope(binding.logquant_rope_frequencies(96), device=U.DEVICE)
    out = cache.decode_step(K.to(U.DEVICE), V.to(U.DEVICE), q.to(U.DEVICE), rope=rope)
    assert cache.counts() == [65, 71] and all(np.array_equal(U.pools(cache)[w], before[w]) for w in "kv")
    w = U.live_weights(cache)
    assert (w[0, :, 64] == 0).all() and (w[1, :, 64:71] == 0).all()
    model.K, model.V, model.w = ([x[:, :64] for x in t] for t in (model.K, model.V, model.w))
    places = torch.tensor([64, 70], dtype=torch.int32, device=U.DEVICE)
    tq = binding.rotate(rope, places, q.to(U.DEVICE))[0].cpu()
    model.check_output(out, tq, weights=w)


def test_a_cache_without_pages_of_some_rows_weighs_nothing():
    cache, model = _filled(19, [70, 40], 2, 1, 64, 32, "f16", weighted=True)
    cache.table[0, 0] = -1
    q = U.rows(1, 2, 2, 64, dtype="f16")
    out = cache.decode_attn(q.to(U.DEVICE))
    assert (out[0] == 0).all()
    w = U.live_weights(cache)
    assert (w[0, :, :70] == 0).all()
    model.check_output(out, q, skip=(0,))


def test_another_stream_and_a_given_output():
    cache, model = _filled(23, [400, 90], 8, 2, 128, 64, "bf16")
    q = U.rows(2, 2, 8, 128, dtype="bf16")
    Q, out = q.to(U.DEVICE), torch.full((2, 8, 128), float("nan"), dtype=torch.bfloat16, device=U.DEVICE)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        assert cache.decode_attn(Q, out) is out
    stream.synchronize()
    model.check_output(out, q)


def test_replays_of_a_recorded_step_and_attention():
    """A recorded call keeps its counts: a replayed step writes the same places again; queries, keys and pages are read anew."""
    lengths, Hq, Hkv, d, page, dtype = [100, 33, 0], 8, 2, 64, 32, "f16"
    cache, model = _filled(29, lengths, Hq, Hkv, d, page, dtype, weighted=True, more=4)
    rope = binding.Rope(binding.logquant_rope_frequencies(d), device=U.DEVICE)
    B = len(lengths)
    K, V, q = (torch.zeros(shape, dtype=torch.float16, device=U.DEVICE) for shape in ((B, Hkv, 1, d), (B, Hkv, 1, d), (B, Hq, d)))
    out, out2 = torch.empty_like(q), torch.empty_like(q)
    stream = torch.cuda.Stream()
    counts = cache.counts()
    with torch.cuda.stream(stream):
        cache.decode_step(K, V, q, out, rope=rope)                       # (code is loaded before the recording)
        cache.decode_attn(q, out2)
    stream.synchronize()
    cache.set_counts(counts)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        cache.decode_step(K, V, q, out, rope=rope)
        cache.decode_attn(q, out2)
    assert cache.counts() == [n + 1 for n in counts]
    places = torch.tensor(counts, dtype=torch.int32, device=U.DEVICE)
    K0, V0 = [x.copy() for x in model.K], [x.copy() for x in model.V]
    for i in range(4):
        k, v, x = U.rows(60 + i, B, Hkv, 1, d, dtype=dtype), U.rows(70 + i, B, Hkv, 1, d, dtype=dtype), U.rows(80 + i, B, Hq, d, dtype=dtype)
        for to, a in ((K, k), (V, v), (q, x)):
            to.copy_(a)
        torch.cuda.synchronize()
        model.w = [np.concatenate([w[:, :n], np.zeros((Hkv, 1))], 1) for w, n in zip(np.asarray(U.live_weights(cache)), counts)]
        graph.replay()
        torch.cuda.synchronize()
        tq, tk = (y.cpu() for y in binding.rotate(rope, places, x[:, :, None].contiguous().to(U.DEVICE), k.to(U.DEVICE)))
        model.K = [np.concatenate([a, U.f64(tk[b])], 1) for b, a in enumerate(K0)]
        model.V = [np.concatenate([a, U.f64(v[b])], 1) for b, a in enumerate(V0)]
        model.check_output(out, tq[:, :, 0])
        model.check_output(out2, x)
        # both added their weights
        both = [w.copy() for w in model.w]
        gh = Hq // Hkv
        for b in range(B):
            for h in range(Hkv):
                at = slice(h * gh, (h + 1) * gh)
                for y in (U.f64(tq[b, at, 0]), U.f64(x[b, at])):
                    both[b][h] += U.attention_and_bounds(y, model.K[b][h], model.V[b][h], 0, dtype)[1].sum(0)
            assert np.allclose(U.live_weights(cache)[b][:, :counts[b] + 1], both[b], rtol=1e-5, atol=1e-6)
        eager = cache.decode_attn(q)                                     # the program's own work between the replays
        assert torch.equal(eager, out2)
