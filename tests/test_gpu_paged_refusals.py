"""Calls of the paged cache on the GPU that are refused, and what works behind them."""
import numpy as np
import pytest
import torch

from paper_2503_19950_amd import binding
from tests import gpu_util_paged as U

pytestmark = pytest.mark.gpu


def held(cache):
    return (dict(cache.free), list(cache.uses), [[list(i) for i in half] for half in cache.ids], list(cache.pages), cache.shared,
            cache.counts(), list(cache.cur), cache.table.tolist())


def shared_prompt(d=64, dtype="f16"):
    """Rows 0 and 1 read a prompt of 64 tokens; row 0 has been evicted from."""
    cache = U.make(2, 2, 1, d, 32, dtype, 4, n_pages=9, weighted=True)
    model = U.Model(cache, dtype)
    K, V = U.rows(1, 2, 1, 64, d, dtype=dtype), U.rows(2, 2, 1, 64, d, dtype=dtype)
    K[:], V[:] = K[:1], V[:1]
    cache.reserve([64, 0])
    cache.append(K.to(U.DEVICE), V.to(U.DEVICE), [64, 0])
    cache.set_pages(1, cache.ids[0][0])
    cache.set_counts([64, 64])
    model.append(K, V)
    w = np.random.RandomState(1).rand(2, 1, 64).astype(np.float32)
    cache.weights[0, :, :, :64] = torch.from_numpy(w).to(U.DEVICE)
    model.w = [x.astype(np.float64) for x in w]
    cache.evict([50, 64], 8)
    model.evict([50, 64], 8)
    return cache, model


def test_a_refused_eviction_leaves_the_pages_of_a_shared_prompt():
    """In a recording, with too many newest tokens, without room: nothing changes, and the next call goes on from there."""
    cache, model = shared_prompt()
    q = U.rows(3, 2, 2, 64, dtype="f16")
    Q = q.to(U.DEVICE)
    before, out = held(cache), torch.zeros_like(Q)
    weights = cache.weights.clone()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        with pytest.raises(binding.LogQuantError) as e:
            cache.evict([40, 64], 8)
        assert e.value.status == binding.LQ_ERR_STATE
        cache.decode_attn(Q, out)
    assert held(cache) == before
    for kw, status in ((dict(keep=[40, 64], recent=41), binding.LQ_ERR_SHAPE), (dict(keep=[40, 64], recent=-1), binding.LQ_ERR_SHAPE)):
        with pytest.raises(binding.LogQuantError) as e:
            cache.evict(**kw)
        assert e.value.status == status and held(cache) == before
    taken = cache.free
    cache.free = {}
    with pytest.raises(binding.LogQuantError) as e:
        cache.evict([40, 64], 8)
    cache.free = taken
    assert e.value.status == binding.LQ_ERR_CAPACITY and held(cache) == before
    for _ in range(2):
        cache.weights.copy_(weights)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        model.check_output(out, q)
    cache.weights.copy_(weights)
    pools = U.pools(cache)
    cache.evict([40, 64], 8)
    model.evict([40, 64], 8)
    U.check_rows(cache, model, pools)
    w = U.live_weights(cache)
    assert all(np.array_equal(w[b, :, :cache.n[b]], model.w[b]) for b in range(2))


def test_a_prompt_is_shared_on_after_one_of_its_readers_was_evicted_from():
    cache, model = shared_prompt()
    cache.set_pages(0, cache.ids[cache.cur[0]][0])                       # its own again: nothing changes
    cache.release(0)
    cache.set_pages(0, cache.ids[0][1])                                  # joins the prompt again, which row 1 reads
    cache.set_counts([64, 64])
    model.K[0], model.V[0] = model.K[1], model.V[1]
    q = U.rows(3, 2, 2, 64, dtype="f16")
    model.check_output(cache.decode_attn(q.to(U.DEVICE)), q)


def test_tokens_behind_an_eviction_are_turned_by_positions_alone():
    cache, model = shared_prompt()
    cache.set_pages(1, cache.ids[0][1] + [cache.free.popitem()[0]])
    rope = binding.Rope(binding.logquant_rope_frequencies(64), device=U.DEVICE)
    K, V, q = U.rows(4, 2, 1, 1, 64, dtype="f16"), U.rows(5, 2, 1, 1, 64, dtype="f16"), U.rows(6, 2, 2, 64, dtype="f16")
    before, pools = held(cache), U.pools(cache)
    with pytest.raises(ValueError):
        cache.decode_step(K.to(U.DEVICE), V.to(U.DEVICE), q.to(U.DEVICE), rope=rope)
    with pytest.raises(ValueError):
        cache.append(K.to(U.DEVICE), V.to(U.DEVICE), rope=rope)
    assert held(cache) == before
    cache.append(K.to(U.DEVICE), V.to(U.DEVICE), [0, 1], rope=rope)      # the other row's places are its positions
    model.append(binding.rotate(rope, torch.full((2,), 64, dtype=torch.int32, device=U.DEVICE), k=K.to(U.DEVICE))[1].cpu(), V, [0, 1])
    U.check_rows(cache, model, pools)
    at = torch.tensor([64, 65], dtype=torch.int32, device=U.DEVICE)
    tq, tk = (x.cpu() for x in binding.rotate(rope, at, q[:, :, None].contiguous().to(U.DEVICE), K.to(U.DEVICE)))
    out = cache.decode_step(K.to(U.DEVICE), V.to(U.DEVICE), q.to(U.DEVICE), rope=rope, positions=at)
    model.append(tk, V)
    U.check_rows(cache, model, pools)
    model.check_output(out, tq[:, :, 0])


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_tokens_without_a_page_are_tokens_of_zeros_behind_an_eviction(dtype):
    """Before it they get no attention and no weight; those that stay take part in the softmax as a key and a value of zeros."""
    Hkv, d, page, lengths = 2, 64, 32, [96, 70]
    cache = U.make(2, 4, Hkv, d, page, dtype, 4, weighted=True)
    cache.reserve(lengths)
    K, V = U.rows(1, 2, Hkv, 96, d, dtype=dtype), U.rows(2, 2, Hkv, 96, d, dtype=dtype)
    cache.append(K.to(U.DEVICE), V.to(U.DEVICE), lengths)
    cache.table[0, 0, 1] = -1                                            # row 0: 32 of its 96 tokens
    q = U.rows(3, 2, 4, d, dtype=dtype)
    seen = U.Model(cache, dtype)                                         # what attends: row 0 without them
    seen.append(K, V, lengths)
    seen.K[0], seen.V[0] = (np.delete(x[0], np.s_[32:64], 1) for x in (seen.K, seen.V))
    seen.check_output(cache.decode_attn(q.to(U.DEVICE)), q)
    w = U.live_weights(cache)
    assert (w[0, :, 32:64] == 0).all() and (w[0, :, :32] > 0).all() and (w[0, :, 64:96] > 0).all()
    model = U.Model(cache, dtype)
    model.append(K, V, lengths)
    model.K[0][:, 32:64] = model.V[0][:, 32:64] = 0
    model.w = [w[b, :, :n].copy() for b, n in enumerate(lengths)]
    # 64 tokens have a page: of 60 that stay none is without one, of 70 six are
    for keep in (60, 70):
        one, two = cache.clone(), U.Model(cache, dtype)
        one.table[0, 0, 1] = -1
        two.K, two.V, two.w = ([x.copy() for x in t] for t in (model.K, model.V, model.w))
        before = U.pools(one)
        one.evict([keep, 70], 8)
        two.evict([keep, 70], 8)
        assert all((two.K[0][h] == 0).all(-1).sum() == max(0, keep - 64) for h in range(Hkv))
        U.check_rows(one, two, before)
        two.check_output(one.decode_attn(q.to(U.DEVICE)), q, weights=U.live_weights(one))
