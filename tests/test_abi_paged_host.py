"""CPU-side checks of rotary positions' and the paged cache's entry points: sizes, frequencies, and refusals before anything
touches the GPU."""
import ctypes as C
import math

import numpy as np
import pytest

from oracle import paged
from paper_2503_19950_amd import binding as B

AT = 4096                      # a stand-in for device memory


def _cfg(**kw):
    a = dict(B=2, Hq=32, Hkv=8, d=128, page=64, dtype="f16", n_pages=64, max_pages=16, weighted=True)
    a.update(kw)
    return B.make_config_paged(**a)


def _cache(n=(0, 0), cur=None, pages=None, **kw):
    arrays = [(C.c_int32 * len(x))(*x) for x in (n, cur or [0] * len(n), pages or [16] * (2 * len(n)))]
    c = B.lq_cache_paged(AT, AT, AT, AT, *(C.cast(x, B._I32P) for x in arrays), AT)
    c.keep = arrays
    for k, v in kw.items():
        setattr(c, k, v)
    return c, arrays


def _rope(dims=128, interleaved=0, factor=1.0, freq=AT):
    return B.lq_rope(dims, interleaved, factor, freq)


def _append(cfg, cache, rope=None, positions=None, k=AT, v=AT, n_new=None, n_max=1):
    return B.logquant_append_paged(cfg, cache, rope, positions, k, v, n_new, n_max)


def _attn(cfg, cache, scores=None, q=AT, scale=0.0, out=AT, ws=AT):
    return B.logquant_decode_attn_paged(cfg, cache, scores, q, scale, out, ws)


def _step(cfg, cache, rope=None, positions=None, scores=None, k=AT, v=AT, q=AT, scale=0.0, out=AT, ws=AT):
    return B.logquant_decode_step_paged(cfg, cache, rope, positions, scores, k, v, q, scale, out, ws)


def _rotate(rope=None, B_=2, L=3, Hq=4, Hkv=2, d=128, dtype=0, positions=AT, q=AT, q_out=AT, k=AT, k_out=AT):
    return B.logquant_rotate(rope or _rope(), B_, L, Hq, Hkv, d, dtype, positions, q, q_out, k, k_out)


def test_sizes_match_the_documented_layouts():
    s = B.logquant_sizes_paged(_cfg())
    assert s.pages == 64 * 8 * 64 * 128 * 2
    assert s.table == 2 * 2 * 16 * 4
    assert s.weights == 2 * 2 * 8 * 16 * 64 * 4
    assert s.seq_state >= 2 * 16
    plain = B.logquant_sizes_paged(_cfg(weighted=False))
    assert plain.weights == 0 and plain.workspace % 16 == 0
    assert s.workspace == plain.workspace + 2 * 32 * 8 + 2 * 32 * 16 * 64 * 4
    assert B.logquant_sizes_paged(_cfg(n_pages=1 << 20)).pages == (1 << 20) * 8 * 64 * 128 * 2 > 1 << 36


@pytest.mark.parametrize("kw,status", [
    (dict(B=0), B.LQ_ERR_SHAPE), (dict(Hq=0), B.LQ_ERR_SHAPE), (dict(Hq=30), B.LQ_ERR_SHAPE), (dict(Hkv=-8), B.LQ_ERR_SHAPE),
    (dict(n_pages=0), B.LQ_ERR_SHAPE), (dict(max_pages=0), B.LQ_ERR_SHAPE), (dict(max_pages=-1), B.LQ_ERR_SHAPE),
    (dict(d=80), B.LQ_ERR_UNSUPPORTED), (dict(page=16), B.LQ_ERR_UNSUPPORTED), (dict(page=256), B.LQ_ERR_UNSUPPORTED),
    (dict(page=48), B.LQ_ERR_UNSUPPORTED), (dict(B=4096, Hq=16), B.LQ_ERR_UNSUPPORTED),
    (dict(max_pages=(1 << 24) + 1), B.LQ_ERR_SHAPE), (dict(n_pages=1 << 25), B.LQ_ERR_SHAPE),
    (dict(Hkv=128, Hq=128, n_pages=1 << 24), B.LQ_ERR_SHAPE), (dict(B=2000, max_pages=1 << 16), B.LQ_ERR_SHAPE),
])
def test_bad_configs_are_rejected_by_every_call(kw, status):
    cfg = _cfg(**kw)
    assert B._lib.logquant_sizes_paged(C.byref(cfg), C.byref(B.lq_sizes_paged())) == status
    with pytest.raises(B.LogQuantError):
        B.logquant_sizes_paged(cfg)
    cache, _ = _cache([0] * max(1, kw.get("B", 2)))
    assert B.logquant_workspace_init_paged(cfg, AT) == status
    assert _append(cfg, cache) == _attn(cfg, cache) == _step(cfg, cache) == status
    assert B.logquant_evict_paged(cfg, cache, [0, 0], 0, AT) == status


def test_values_that_are_none_of_a_kind():
    for name, x in (("dtype", 2), ("weighted", 2), ("weighted", -1)):
        cfg = _cfg()
        setattr(cfg, name, x)
        assert B._lib.logquant_sizes_paged(C.byref(cfg), C.byref(B.lq_sizes_paged())) == B.LQ_ERR_SHAPE


def test_null_pointers():
    cfg, (cache, arrays) = _cfg(), _cache()
    assert B.logquant_workspace_init_paged(None, AT) == B.logquant_workspace_init_paged(cfg, None) == B.LQ_ERR_NULL
    assert B._lib.logquant_sizes_paged(C.byref(cfg), None) == B.LQ_ERR_NULL
    assert _append(None, cache) == _append(cfg, None) == _append(cfg, cache, k=None) == _append(cfg, cache, v=None) == B.LQ_ERR_NULL
    assert _attn(None, cache) == _attn(cfg, None) == B.LQ_ERR_NULL
    for name in ("q", "out", "ws"):
        assert _attn(cfg, cache, **{name: None}) == B.LQ_ERR_NULL, name
    for name in ("k", "v", "q", "out", "ws"):
        assert _step(cfg, cache, **{name: None}) == B.LQ_ERR_NULL, name
    assert B.logquant_evict_paged(cfg, cache, None, 0, AT) == B.logquant_evict_paged(cfg, cache, [0, 0], 0, None) == B.LQ_ERR_NULL
    for name in ("k_pages", "v_pages", "table", "weights", "n", "cur", "pages", "seq_state"):
        c, _ = _cache()
        setattr(c, name, B._I32P() if name in ("n", "cur", "pages") else None)
        assert _append(cfg, c) == _attn(cfg, c) == _step(cfg, c) == B.logquant_evict_paged(cfg, c, [0, 0], 0, AT) == B.LQ_ERR_NULL, name
    assert _append(cfg, cache, rope=_rope(freq=None)) == _step(cfg, cache, rope=_rope(freq=None)) == B.LQ_ERR_NULL
    assert list(arrays[0]) == [0, 0]


def test_buffers_off_their_alignment():
    cfg, (cache, _) = _cfg(), _cache((5, 5))
    assert B.logquant_workspace_init_paged(cfg, 4104) == B.LQ_ERR_SHAPE
    for name in ("k", "v"):
        assert _append(cfg, cache, **{name: 4098}) == B.LQ_ERR_SHAPE
    for name in ("q", "out", "ws"):
        assert _attn(cfg, cache, **{name: 4104}) == B.LQ_ERR_SHAPE
    for name in ("k", "v", "q", "out", "ws"):
        assert _step(cfg, cache, **{name: 4104}) == B.LQ_ERR_SHAPE
    assert B.logquant_evict_paged(cfg, cache, [3, 3], 0, 4104) == B.LQ_ERR_SHAPE
    for name in ("k_pages", "v_pages", "table", "weights", "seq_state"):
        c, _ = _cache((5, 5), **{name: 4100})
        assert _attn(cfg, c) == B.LQ_ERR_SHAPE, name
    assert _attn(cfg, cache, scores=B.lq_scores(0, 0, 4098)) == B.LQ_ERR_SHAPE
    assert _append(cfg, cache, rope=_rope(freq=4100)) == _append(cfg, cache, rope=_rope(), positions=4098) == B.LQ_ERR_SHAPE
    for name in ("q", "q_out", "k", "k_out", "positions"):
        assert _rotate(**{name: 4098}) == B.LQ_ERR_SHAPE, name


def test_counts_halves_and_pages():
    cfg = _cfg()
    for kw in (dict(n=(-1, 0)), dict(n=(0, 1025)), dict(n=(0, 65), pages=[16, 1, 16, 16]), dict(cur=[2, 0]), dict(cur=[0, -1]),
               dict(pages=[16, 17, 0, 0]), dict(pages=[16, 16, -1, 0]), dict(n=(0, 65), cur=[0, 1], pages=[16, 16, 16, 1])):
        c, arrays = _cache(**kw)
        before = [list(x) for x in arrays]
        assert _append(cfg, c) == _attn(cfg, c) == _step(cfg, c) == B.logquant_evict_paged(cfg, c, [0, 0], 0, AT) == B.LQ_ERR_STATE, kw
        assert [list(x) for x in arrays] == before


def test_room():
    cfg = _cfg()
    cache, arrays = _cache((1024, 60), cur=[0, 1], pages=[16, 16, 16, 1])
    assert _append(cfg, cache, n_max=0) == B.LQ_ERR_SHAPE
    assert _append(cfg, cache, n_new=[-1, 0], n_max=4) == _append(cfg, cache, n_new=[0, 5], n_max=4) == B.LQ_ERR_SHAPE
    assert _append(cfg, cache, n_new=[1, 0], n_max=4) == _append(cfg, cache, n_new=[0, 5], n_max=5) == B.LQ_ERR_CAPACITY
    assert _append(cfg, cache, n_new=[0, 2 ** 31 - 1], n_max=2 ** 31 - 1) == B.LQ_ERR_CAPACITY
    assert _append(cfg, cache, n_new=[0, 0], n_max=4) == B.LQ_OK                         # nobody takes a token: no launch
    assert _step(cfg, cache) == B.LQ_ERR_CAPACITY
    cache2, _ = _cache((64, 3), pages=[1, 1, 0, 0])
    assert _step(cfg, cache2) == B.LQ_ERR_CAPACITY
    assert list(arrays[0]) == [1024, 60]


def test_ropes():
    cfg, (cache, _) = _cfg(d=96), _cache()
    for rope in (_rope(0), _rope(97), _rope(7), _rope(98), _rope(-2), _rope(96, 2), _rope(96, factor=math.inf), _rope(96, factor=math.nan)):
        assert _append(cfg, cache, rope=rope) == _step(cfg, cache, rope=rope) == _rotate(rope, d=96) == B.LQ_ERR_SHAPE, rope.dims
    for kw in (dict(B_=0), dict(L=0), dict(Hq=0), dict(Hkv=-1), dict(d=0), dict(dtype=2)):
        assert _rotate(**kw) == B.LQ_ERR_SHAPE, kw
    for kw in (dict(d=80), dict(d=256), dict(B_=65536), dict(L=2 ** 30), dict(B_=60000, L=40000, Hq=1, Hkv=1), dict(Hq=2 ** 28)):
        assert _rotate(**kw) == B.LQ_ERR_UNSUPPORTED, kw
    assert B.logquant_rotate(None, 2, 3, 4, 2, 128, 0, AT, AT, AT, AT, AT) == B.LQ_ERR_NULL
    for kw in (dict(q=None), dict(q_out=None), dict(k=None), dict(k_out=None), dict(q=None, q_out=None, k=None, k_out=None)):
        assert _rotate(**kw) == B.LQ_ERR_NULL, kw


def test_scores():
    cfg, (cache, _) = _cfg(), _cache((5, 5))
    inf, nan = math.inf, math.nan
    for scores, scale in ((B.lq_scores(0, -1, None), 0), (B.lq_scores(nan, 0, None), 0), (B.lq_scores(inf, 0, None), 0),
                          (B.lq_scores(3e38, 0, None), 0), (B.lq_scores(1e-40, 0, None), 1.0), (B.lq_scores(0, 0, None), inf),
                          (None, inf), (None, 3e38)):
        assert _attn(cfg, cache, scores, scale=scale) == _step(cfg, cache, scores=scores, scale=scale) == B.LQ_ERR_SHAPE


def test_evictions():
    cfg = _cfg()
    evict = lambda c, keep, recent=0, cfg=cfg: B.logquant_evict_paged(cfg, c, keep, recent, AT)  # noqa: E731
    cache, arrays = _cache((200, 100), cur=[0, 1], pages=[4, 1, 2, 2])
    assert evict(cache, [-1, 5]) == evict(cache, [5, 5], -1) == evict(cache, [5, 200], 6) == B.LQ_ERR_SHAPE
    assert evict(cache, [129, 100]) == evict(cache, [200, 65]) == B.LQ_ERR_CAPACITY
    assert evict(cache, [200, 100], 1000) == B.LQ_OK                                     # nobody loses a token: no launch
    assert [list(x) for x in arrays[:2]] == [[200, 100], [0, 1]]
    assert evict(cache, [0, 100]) == B.LQ_OK                                             # all of it: no launch either
    assert [list(x) for x in arrays[:2]] == [[0, 100], [1, 1]]
    plain, _ = _cache((200, 100), weights=None)
    assert evict(plain, [0, 0], cfg=_cfg(weighted=False)) == B.LQ_ERR_STATE


@pytest.mark.parametrize("args", [(128,), (96, 500000.0), (2, 10.0, 3.0), (64, 10000.0, 8.0, 8192.0, 1.0, 4.0), (128, 1e6, 40.0, 4096.0, 1.0, 32.0)])
def test_frequencies(args):
    # pow within one unit of fp64's last place, three operations behind it
    assert np.allclose(B.logquant_rope_frequencies(*args), paged.frequencies(*args), rtol=1e-14, atol=0)


@pytest.mark.parametrize("args", [(0,), (3,), (-2,), (8, 0.0), (8, math.inf), (8, math.nan), (8, 10.0, 0.0), (8, 10.0, math.inf),
                                  (8, 10.0, 2.0, -1.0), (8, 10.0, 2.0, math.nan), (8, 10.0, 2.0, 100.0, 4.0, 4.0), (8, 10.0, 2.0, 100.0, 4.0, math.nan)])
def test_frequencies_that_are_refused(args):
    with pytest.raises(B.LogQuantError):
        B.logquant_rope_frequencies(*args)


def test_the_owners_of_buffers_refuse_a_cpu():
    with pytest.raises(ValueError):
        B.DeviceCachePaged(_cfg(), device="cpu")
    with pytest.raises(ValueError):
        B.Rope([1.0], device="cpu")
