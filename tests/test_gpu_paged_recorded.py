"""A recorded run of all calls of the paged cache against the same calls made one by one: every replay gives the same bits, whatever
the program did with the cache in between."""
import pytest
import torch

from paper_2503_19950_amd import binding
from tests import gpu_util_paged as U

pytestmark = pytest.mark.gpu


def _life(cache, rope, x, out, n_new, keep):
    """Rotate, append, step, attend, evict, attend."""
    binding.rotate(rope, x["at"], x["q"], x["k"], x["tq"], x["tk"])
    cache.append(x["k"], x["v"], n_new, rope=rope, positions=x["at"])
    cache.decode_step(x["k1"], x["v1"], x["q1"], out[0], rope=rope, positions=x["at1"], softcap=30.0)
    cache.decode_attn(x["q1"], out[1], window=40, slopes=x["slopes"])
    cache.evict(keep, 5)
    cache.decode_attn(x["q1"], out[2])


def _inputs(seed, B, Hq, Hkv, n, d, dtype):
    rows = lambda i, *shape: U.rows(10 * seed + i, *shape, dtype=dtype)  # noqa: E731
    g = torch.Generator().manual_seed(seed)
    at = torch.randint(0, 1 << 18, (B, n), generator=g, dtype=torch.int32)
    return dict(q=rows(0, B, Hq, n, d), k=rows(1, B, Hkv, n, d), v=rows(2, B, Hkv, n, d), k1=rows(3, B, Hkv, 1, d), v1=rows(4, B, Hkv, 1, d),
                q1=rows(5, B, Hq, d), at=at, at1=at[:, -1] + 1, slopes=torch.rand(Hq, generator=g))


# few rows, which travel with a launch, and more than that; rows of one length in both halves and of many
@pytest.mark.parametrize("B,Hq,Hkv,d,page,dtype,longest", [(3, 8, 2, 128, 64, "bf16", 700), (200, 2, 1, 64, 32, "f16", 90), (140, 1, 1, 96, 32, "bf16", 0),
                                                           (2, 34, 1, 64, 128, "f16", 17500)])
def test_a_recorded_run(B, Hq, Hkv, d, page, dtype, longest):
    lengths = [60 + (b * 37 % longest if longest else 0) for b in range(B)]
    lengths[-1] = 60 + longest
    n, n_new, keep = 5, [b % 6 for b in range(B)], 64 if longest != 17500 else [64, 9000]
    cache = U.make(B, Hq, Hkv, d, page, dtype, -(-(max(lengths) + n + 1) // page), weighted=True)
    cache.reserve([x + n + 1 for x in lengths])
    cache.reserve([64 if isinstance(keep, int) else keep[b] for b in range(B)], spare=True)
    K, V = U.rows(1, B, Hkv, max(lengths), d, dtype=dtype), U.rows(2, B, Hkv, max(lengths), d, dtype=dtype)
    cache.append(K.to(U.DEVICE), V.to(U.DEVICE), lengths)
    cache.weights[0] = torch.rand(cache.weights.shape[1:], generator=torch.Generator().manual_seed(7)).to(U.DEVICE)
    rope = binding.Rope(binding.logquant_rope_frequencies(d // 2), True, device=U.DEVICE)
    x = {k: v.to(U.DEVICE) for k, v in _inputs(0, B, Hq, Hkv, n, d, dtype).items()}
    x["tq"], x["tk"] = torch.empty_like(x["q"]), torch.empty_like(x["k"])
    out = [torch.empty_like(x["q1"]) for _ in range(3)]
    start, counts, halves = cache.clone(), cache.counts(), list(cache.cur)

    def back(to):
        for name in to.BUFFERS:
            getattr(to, name).copy_(getattr(start, name))

    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        _life(cache, rope, x, out, n_new, keep)                          # (code is loaded before the recording)
    stream.synchronize()
    cache.set_counts(counts, halves)
    back(cache)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        _life(cache, rope, x, out, n_new, keep)
    behind = cache.counts()
    assert max(behind) <= 9000 and list(cache.cur) != halves
    other = start.clone()
    for i in range(4):
        for name, y in _inputs(i + 1, B, Hq, Hkv, n, d, dtype).items():
            x[name].copy_(y)
        back(cache)
        back(other)
        other.set_counts(counts, halves)
        mine = {k: torch.empty_like(v) if k in ("tq", "tk") else v for k, v in x.items()}
        expected = [torch.empty_like(y) for y in out]
        _life(other, rope, mine, expected, n_new, keep)
        assert other.counts() == behind
        for y in (*out, x["tq"], x["tk"]):
            y.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, expected)) and torch.equal(x["tq"], mine["tq"]) and torch.equal(x["tk"], mine["tk"])
        for name in cache.BUFFERS:
            a, b = (getattr(c, name).view(torch.uint8) for c in (cache, other))
            assert torch.equal(a, b), name
        # the program's own work on what the recording uses: workspace, counts on the device, weights
        cache.set_counts([max(1, n // 2) for n in counts], halves)
        cache.decode_attn(x["q1"], softcap=5.0)
        cache.set_counts(behind)
