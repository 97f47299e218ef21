"""Decode attention and the decode step over the 8-bit cache against fp64 attention over what the oracle holds."""
import numpy as np
import pytest
import torch

from tests import gpu_util8 as U
from tests.test_gpu_cache8_state import build

pytestmark = pytest.mark.gpu


def queries(seed, B, Hq, d, dtype, gain=1.0):
    return U.rows(seed, B, Hq, 1, d, dtype, gain, outliers=False)[:, :, 0].contiguous()


@pytest.mark.parametrize("d,G,dtype", [(d, G, dtype) for d in (64, 96, 128) for G in (32, 64, 128) for dtype in ("f16", "bf16")])
def test_lengths_from_none_to_several_blocks(d, G, dtype):
    lengths = [0, 1, 2, G - 1, G, G + 1, 2 * G - 1, 33, 5 * G + 31, 9 * G + 32]
    cache, oracle = build(101, len(lengths), 4, 2, d, G, dtype, lengths)
    q = queries(102, len(lengths), 4, d, dtype)
    out = cache.decode_attn(q.to(U.DEVICE), torch.full_like(q, float("nan")).to(U.DEVICE))
    U.check_output(out, q, oracle, dtype)
    assert (out[0] == 0).all()


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (2, 1), (3, 1), (5, 1), (16, 1), (17, 1), (24, 1), (32, 1), (33, 1), (72, 1), (40, 2), (12, 4), (64, 8), (32, 32)])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_head_layouts(Hq, Hkv, dtype):
    cache, oracle = build(111, 2, Hq, Hkv, 64, 32, dtype, [700, 45])
    q = queries(112, 2, Hq, 64, dtype)
    U.check_output(cache.decode_attn(q.to(U.DEVICE)), q, oracle, dtype)


@pytest.mark.parametrize("B,Hq,Hkv,d,G,dtype,L", [
    (1, 8, 2, 128, 64, "bf16", 20011), (2, 24, 1, 128, 64, "f16", 12345), (1, 70, 1, 64, 32, "bf16", 9000), (1, 16, 1, 128, 32, "f16", 30001),
    (1, 5, 1, 96, 64, "bf16", 40000), (1, 2, 1, 64, 32, "f16", 70001), (3, 8, 1, 96, 128, "bf16", 9001), (1, 4, 4, 128, 32, "f16", 4096),
])
def test_long_rows_shared_by_many_workgroups(B, Hq, Hkv, d, G, dtype, L):
    cache, oracle = build(121, B, Hq, Hkv, d, G, dtype, [L] * B)
    for seed in (122, 123):
        q = queries(seed, B, Hq, d, dtype)
        U.check_output(cache.decode_attn(q.to(U.DEVICE)), q, oracle, dtype)


@pytest.mark.parametrize("seed", range(12))
def test_drawn_batches(seed):
    rng = np.random.default_rng(1000 + seed)
    B, Hkv, gh = int(rng.integers(1, 40)), int(rng.choice([1, 2, 4, 8])), int(rng.choice([1, 2, 3, 4, 6, 8]))
    d, G, dtype = int(rng.choice([64, 96, 128])), int(rng.choice([32, 64, 128])), str(rng.choice(["f16", "bf16"]))
    lengths = [int(x) for x in np.exp(rng.uniform(0, np.log(3000), B))]
    if rng.random() < 0.3:
        lengths = [lengths[0]] * B
    cache, oracle = build(2000 + seed, B, Hkv * gh, Hkv, d, G, dtype, lengths)
    q = queries(3000 + seed, B, Hkv * gh, d, dtype)
    U.check_output(cache.decode_attn(q.to(U.DEVICE)), q, oracle, dtype)


def test_more_rows_than_travel_in_a_launch():
    lengths = [(7 * i) % 150 for i in range(300)]
    cache, oracle = build(131, 300, 2, 1, 64, 32, "f16", lengths)
    q = queries(132, 300, 2, 64, "f16")
    U.check_output(cache.decode_attn(q.to(U.DEVICE)), q, oracle, "f16")
    k, v = U.rows(133, 300, 1, 1, 64, "f16"), U.rows(134, 300, 1, 1, 64, "f16")
    out = cache.decode_step(k.to(U.DEVICE), v.to(U.DEVICE), q.to(U.DEVICE))
    oracle.append(k, v)
    oracle.check(cache)
    U.check_output(out, q, oracle, "f16")


def shapes_of_plans():
    """Numbers of items around those where the workgroups' plan changes, with rows alike and not, and rows whose work
    is not in the order of their lengths (a tail of 127 tokens counts more than the block that it becomes)."""
    frac = lambda B, L: [L - int(L * (b * 0.6180339887 % 1.0)) for b in range(B)]  # noqa: E731
    return [
        ("few_alike", 3, 2, 64, [3000] * 3), ("half_alike", 33, 4, 32, [400] * 33), ("nearly_full_alike", 60, 4, 32, [300] * 60),
        ("one_more_alike", 65, 4, 32, [700] * 65), ("more_alike", 85, 4, 32, [300] * 85), ("many_alike", 130, 4, 32, [100] * 130),
        ("few", 9, 4, 64, frac(9, 6000)), ("nearly_full", 62, 4, 32, frac(62, 1500)), ("one_long", 66, 4, 32, [9000] + [65] * 65),
        ("one_long_few", 20, 4, 32, [9000] + [65] * 19), ("large", 70, 4, 64, frac(70, 2500)), ("many", 280, 4, 32, frac(280, 300)),
        ("tails", 300, 4, 128, [(i % 2) * 127 + 128 * (1 + (i + 1) % 2) for i in range(300)]),
        ("long_and_tails", 150, 2, 128, [12000, 11999, 11904] + [(i % 2) * 127 + 128 * (1 + (i + 1) % 2) for i in range(147)]),
    ]


@pytest.mark.parametrize("name,B,Hkv,G,lengths", shapes_of_plans(), ids=[x[0] for x in shapes_of_plans()])
def test_shapes_of_plans(name, B, Hkv, G, lengths):
    cache, oracle = build(301, B, 2 * Hkv, Hkv, 64, G, "f16", lengths)
    q = queries(302, B, 2 * Hkv, 64, "f16").to(U.DEVICE)
    out = cache.decode_attn(q, torch.full_like(q, float("nan")))
    U.check_output(out, q.cpu(), oracle, "f16", rows_of=sorted(set(list(range(0, B, max(1, B // 12))) + [0, 1, 2, B - 2, B - 1])))
    assert torch.isfinite(out).all()
    assert torch.equal(cache.decode_attn(q), out)


@pytest.mark.parametrize("dtype,gh,lengths", [("bf16", 16, [3000 - 37 * i for i in range(40)]), ("f16", 7, [3000 - 37 * i for i in range(40)]),
                                              ("f16", 15, [3000 - 37 * i for i in range(40)]), ("bf16", 16, [500] * 20)])
def test_many_heads_in_large_workgroups(dtype, gh, lengths):
    """Head counts at which a workgroup's merge outgrows what a launch may ask of LDS, with 8 kv heads and d = 128."""
    B = len(lengths)
    cache, oracle = build(311, B, 8 * gh, 8, 128, 32, dtype, lengths)
    q = queries(312, B, 8 * gh, 128, dtype)
    U.check_output(cache.decode_attn(q.to(U.DEVICE)), q, oracle, dtype, rows_of=[0, 1, B // 2, B - 1])


@pytest.mark.parametrize("B,gh,d,G,dtype,L", [(4, 24, 64, 32, "f16", 48030), (1, 32, 128, 64, "bf16", 95038), (2, 17, 96, 128, "f16", 65150),
                                              (3, 40, 64, 128, "bf16", 64126)])
def test_more_than_16_heads_over_a_long_context(B, gh, d, G, dtype, L):
    """Two sets of heads in a workgroup (from 24 MB on), attention and steps across the end of a block."""
    cache, oracle = build(361, B, gh, 1, d, G, dtype, [L] + [L - 1001 * b for b in range(1, B)], capacity=(L // G + 2) * G)
    q = queries(362, B, gh, d, dtype)
    U.check_output(cache.decode_attn(q.to(U.DEVICE)), q, oracle, dtype)
    for i in range(3):
        k, v, q = U.rows(370 + i, B, 1, 1, d, dtype), U.rows(380 + i, B, 1, 1, d, dtype), queries(390 + i, B, gh, d, dtype)
        out = cache.decode_step(k.to(U.DEVICE), v.to(U.DEVICE), q.to(U.DEVICE))
        oracle.append(k, v)
        U.check_output(out, q, oracle, dtype)
    oracle.check(cache)


def test_counts_set_back_within_a_block():
    """Tokens that are dropped again: within the tail, and from a block that single tokens have just filled."""
    G, d = 64, 64
    cache, oracle = build(321, 2, 2, 1, d, G, "f16", [G - 3, 2 * G - 3], capacity=4 * G)
    held = [cache.clone()]
    steps = [(U.rows(330 + i, 2, 1, 1, d, "f16").to(U.DEVICE), U.rows(340 + i, 2, 1, 1, d, "f16").to(U.DEVICE)) for i in range(3)]
    for k, v in steps:
        cache.append(k, v)
        held.append(cache.clone())
    q = queries(351, 2, 2, d, "f16").to(U.DEVICE)
    for back in (1, 2, 3):
        cache.set_counts([G - back, 2 * G - back])
        assert torch.equal(cache.decode_attn(q), held[3 - back].decode_attn(q))
    cache.set_counts([G - 3, 2 * G - 3])
    oracle.check(cache)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("scale", [0.0, 0.3, 1e-3])
def test_scales_of_the_softmax(dtype, scale):
    cache, oracle = build(141, 2, 4, 2, 96, 64, dtype, [1000, 77])
    q = queries(142, 2, 4, 96, dtype, 0.5)
    U.check_output(cache.decode_attn(q.to(U.DEVICE), softmax_scale=scale), q, oracle, dtype, scale)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_logits_that_rise_and_fall_along_a_row(dtype):
    """References that change often, one token that takes all the weight, blocks whose scales differ by 2^20."""
    G, d, L = 32, 128, 1500
    cache = U.make(3, 2, 1, d, G, dtype, 1600)
    oracle = U.Oracle(cache, dtype)
    K, V = U.rows(151, 3, 1, L, d, dtype).float(), U.rows(152, 3, 1, L, d, dtype, outliers=False).float()
    K[0] *= torch.linspace(0.01, 3, L)[:, None]
    K[1, 0, 700] *= 12
    V[2] *= torch.exp2(torch.randint(-10, 11, (L // G + 1,), generator=torch.Generator().manual_seed(3)).float()).repeat_interleave(G)[:L, None]
    K, V = K.to(cache.dtype), V.to(cache.dtype)
    oracle.append(K, V)
    cache.append(K.to(U.DEVICE), V.to(U.DEVICE))
    for gain in (1.0, 3.0):
        q = queries(153, 3, 2, d, dtype, gain)
        U.check_output(cache.decode_attn(q.to(U.DEVICE)), q, oracle, dtype)


@pytest.mark.parametrize("q_gain,k_gain,v_gain", [(2.0 ** 40, 2.0 ** -40, 2.0 ** 85), (2.0 ** -60, 2.0 ** 60, 2.0 ** -100), (2.0 ** 80, 2.0 ** -80, 2.0 ** -120)])
def test_far_magnitudes_of_bf16(q_gain, k_gain, v_gain):
    """Scales of blocks near the ends of their range: the outputs are those of ordinary magnitudes, times v's."""
    cache = U.make(2, 4, 2, 96, 32, "bf16", 1024)
    oracle = U.Oracle(cache, "bf16")
    K, V = U.rows(157, 2, 2, 1000, 96, "bf16", k_gain), U.rows(158, 2, 2, 1000, 96, "bf16", v_gain, outliers=False)
    oracle.append(K, V)
    cache.append(K.to(U.DEVICE), V.to(U.DEVICE))
    oracle.check(cache)
    q = queries(159, 2, 4, 96, "bf16", q_gain)
    U.check_output(cache.decode_attn(q.to(U.DEVICE)), q, oracle, "bf16")


def test_a_sink_ahead_of_a_long_even_context():
    """One heavy token sets the reference, tens of thousands 2^16 below it weigh as much as it does."""
    d, L = 64, 60000
    cache = U.make(1, 1, 1, d, 64, "f16", 60032)
    oracle = U.Oracle(cache, "f16")
    K, V = torch.zeros((1, 1, L, d)), U.rows(161, 1, 1, L, d, "f16", outliers=False).float() + 1
    K[0, 0, 0, 0] = 11.0
    K, V = K.half(), V.half()
    oracle.append(K, V)
    cache.append(K.to(U.DEVICE), V.to(U.DEVICE))
    q = torch.zeros((1, 1, d))
    q[..., 0] = 8.0
    q = q.half()
    U.check_output(cache.decode_attn(q.to(U.DEVICE)), q, oracle, "f16")


def test_what_lies_behind_the_counts_is_not_seen():
    """NaN, infinities and the type's lowest value where no token is."""
    for fill in (float("nan"), float("inf"), torch.finfo(torch.bfloat16).min):
        cache, oracle = build(171, 4, 4, 2, 64, 64, "bf16", [70, 64, 5, 200])
        q = queries(172, 4, 4, 64, "bf16")
        want = cache.decode_attn(q.to(U.DEVICE))
        U.check_output(want, q, oracle, "bf16")
        for which in "kv":
            tail = getattr(cache, which + "_tail").view(torch.bfloat16).view(8, -1)
            keep = tail.clone()
            tail.fill_(fill)
            from oracle import cache8
            for b, n in enumerate([70, 64, 5, 200]):
                for h in range(2):
                    at = cache8.tail_index(which, np.arange(n % 64)[:, None], np.arange(64)[None], 64).ravel()
                    tail[2 * b + h, torch.from_numpy(at).to(U.DEVICE)] = keep[2 * b + h, torch.from_numpy(at).to(U.DEVICE)]
        assert torch.equal(cache.decode_attn(q.to(U.DEVICE)), want)


@pytest.mark.parametrize("d,G,dtype,Hq,Hkv", [(128, 32, "f16", 8, 2), (96, 64, "bf16", 4, 4), (64, 128, "f16", 24, 1), (128, 64, "bf16", 4, 1)])
def test_generation(d, G, dtype, Hq, Hkv):
    """Prompt, then a step at a time across the end of a block; rows of different lengths and alike; then read back."""
    for lengths in ([2 * G - 4] * 3, [2 * G - 4, 7, 0], [31 * G - 2, 28 * G - 3, G - 1]):
        cache, oracle = build(181, 3, Hq, Hkv, d, G, dtype, lengths, capacity=32 * G)
        other = cache.clone()
        for step in range(9):
            k, v, q = U.rows(190 + step, 3, Hkv, 1, d, dtype), U.rows(210 + step, 3, Hkv, 1, d, dtype), queries(230 + step, 3, Hq, d, dtype)
            oracle.append(k, v)
            out = cache.decode_step(k.to(U.DEVICE), v.to(U.DEVICE), q.to(U.DEVICE))
            oracle.check(cache)
            U.check_output(out, q, oracle, dtype)
            other.append(k.to(U.DEVICE), v.to(U.DEVICE))
            # the results of the two calls; where a block has just become full (and is counted otherwise in the plan of the
            # whole batch), up to the order of sums
            again = other.decode_attn(q.to(U.DEVICE))
            U.check_output(again, q, oracle, dtype)
            if all(n % G for n in cache.n):
                assert torch.equal(again, out)
        assert cache.counts() == [x + 9 for x in lengths] == other.counts()
        top = max(cache.counts())
        kd, vd = cache.read(0, top)
        for b in range(3):
            for h in range(Hkv):
                assert np.array_equal(U.f64(kd[b, h, :cache.n[b]]), oracle.k[b][h].held())
                assert np.array_equal(U.f64(vd[b, h, :cache.n[b]]), oracle.v[b][h].held())


def test_calls_again_give_the_same_bits():
    cache, _ = build(241, 2, 8, 2, 128, 64, "bf16", [9000, 4001])
    q = queries(242, 2, 8, 128, "bf16").to(U.DEVICE)
    first = cache.decode_attn(q).clone()
    for _ in range(20):
        assert torch.equal(cache.decode_attn(q), first)


@pytest.mark.parametrize("lengths", [[5000], [300, 17, 0, 64, 900, 64, 63, 2]])
def test_calls_replay_from_graphs(lengths):
    """Attention with fixed counts, and appends of one token to its place, from two graphs that share a workspace, with
    eager calls in between."""
    B = len(lengths)
    cache, _ = build(251, B, 8, 2, 128, 64, "f16", lengths)
    qs = [queries(252 + i, B, 8, 128, "f16").to(U.DEVICE) for i in range(3)]
    ks, vs = ([U.rows(260 + 10 * j + i, B, 2, 1, 128, "f16").to(U.DEVICE) for i in range(3)] for j in range(2))
    counts = cache.counts()
    eager, stepped, buffers = [], [], []
    for q, k, v in zip(qs, ks, vs):
        eager.append(cache.decode_attn(q).clone())
        stepped.append(cache.decode_step(k, v, q).clone())
        buffers.append([getattr(cache, n).clone() for n in cache.BUFFERS])
        cache.set_counts(counts)
    q_in, k_in, v_in = qs[0].clone(), ks[0].clone(), vs[0].clone()
    out_a, out_s = torch.empty_like(q_in), torch.empty_like(q_in)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        cache.decode_attn(q_in, out_a)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    attn, step = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(attn, stream=side):
        cache.decode_attn(q_in, out_a)
    with torch.cuda.graph(step, stream=side):
        cache.decode_step(k_in, v_in, q_in, out_s)
    cache.set_counts(counts)
    for rep in range(3):
        for i in range(3):
            q_in.copy_(qs[i])
            k_in.copy_(ks[i])
            v_in.copy_(vs[i])
            attn.replay()
            step.replay()
            torch.cuda.synchronize()
            assert torch.equal(out_a, eager[i]) and torch.equal(out_s, stepped[i]), (rep, i)
            for n, want in zip(cache.BUFFERS, buffers[i]):
                assert torch.equal(getattr(cache, n), want), (rep, i, n)
            assert torch.equal(cache.decode_attn(qs[(i + 1) % 3]), eager[(i + 1) % 3])
            torch.cuda.synchronize()


def test_a_stream_of_its_own():
    cache, oracle = build(271, 2, 4, 2, 64, 32, "f16", [500, 90])
    q = queries(272, 2, 4, 64, "f16")
    k, v = U.rows(273, 2, 2, 1, 64, "f16"), U.rows(274, 2, 2, 1, 64, "f16")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        kd, vd, qd = k.to(U.DEVICE), v.to(U.DEVICE), q.to(U.DEVICE)
        out = cache.decode_step(kd, vd, qd)
        got = cache.read(0, 501)
    side.synchronize()
    oracle.append(k, v)
    oracle.check(cache)
    U.check_output(out, q, oracle, "f16")
    assert np.array_equal(U.f64(got[0][0, 1]), oracle.k[0][1].held())
