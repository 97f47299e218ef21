"""CPU-side checks of the 8-bit cache's entry points: sizes, and refusals before anything touches the GPU."""
import ctypes as C

import pytest

from paper_2503_19950_amd import binding as B


def _cfg(**kw):
    a = dict(B=2, Hq=32, Hkv=8, d=128, block=64, dtype="f16", capacity=1024)
    a.update(kw)
    return B.make_config8(**a)


def _cache(counts=(0, 0), **kw):
    """A cache struct with stand-ins for the device pointers."""
    counts = (C.c_int32 * len(counts))(*counts)
    c = B.lq_cache8(4096, 4096, 4096, 4096, 4096, 4096, C.cast(counts, B._I32P), 4096)
    c.keep = counts
    for k, v in kw.items():
        setattr(c, k, v)
    return c, counts


def test_sizes_match_the_documented_layouts():
    s = B.logquant_sizes8(_cfg())
    assert s.codes == 2 * 8 * 1024 * 128
    assert s.scale == 2 * 8 * (1024 // 64) * 4
    assert s.tail == 2 * 8 * 64 * 128 * 2
    assert s.seq_state >= 2 * 8 and s.workspace > 0 and s.workspace % 16 == 0
    assert B.logquant_sizes8(_cfg(d=96, block=32, Hq=8)).codes == 2 * 8 * 1024 * 96
    big = B.logquant_sizes8(_cfg(B=64, capacity=131072))
    assert big.codes == 64 * 8 * 131072 * 128 > 1 << 32


@pytest.mark.parametrize("kw,status", [
    (dict(B=0), B.LQ_ERR_SHAPE), (dict(Hq=0), B.LQ_ERR_SHAPE), (dict(capacity=0), B.LQ_ERR_SHAPE), (dict(Hq=30), B.LQ_ERR_SHAPE),
    (dict(capacity=1000), B.LQ_ERR_SHAPE), (dict(block=128, capacity=1024 + 64), B.LQ_ERR_SHAPE),
    (dict(d=80), B.LQ_ERR_UNSUPPORTED), (dict(block=16), B.LQ_ERR_UNSUPPORTED), (dict(block=256), B.LQ_ERR_UNSUPPORTED),
    (dict(B=4096, Hq=16), B.LQ_ERR_UNSUPPORTED),
    (dict(capacity=1 << 24), B.LQ_ERR_SHAPE),
    (dict(B=2000, capacity=1 << 22), B.LQ_ERR_SHAPE),
])
def test_bad_configs_are_rejected_by_every_call(kw, status):
    cfg = _cfg(**kw)
    out = B.lq_sizes8()
    assert B._lib.logquant_sizes8(C.byref(cfg), C.byref(out)) == status
    with pytest.raises(B.LogQuantError):
        B.logquant_sizes8(cfg)
    cache, _ = _cache([0] * max(1, kw.get("B", 2)))
    assert B.logquant_workspace_init8(cfg, 4096) == status
    assert B.logquant_append8(cfg, cache, 4096, 4096, None, 1) == status
    assert B.logquant_read8(cfg, cache, 0, 1, 4096, 4096) == status
    assert B.logquant_decode_attn8(cfg, cache, 4096, 0.0, 4096, 4096) == status
    assert B.logquant_decode_step8(cfg, cache, 4096, 4096, 4096, 0.0, 4096, 4096) == status


def test_a_type_that_is_none_is_rejected():
    cfg = _cfg()
    cfg.dtype = 2
    assert B._lib.logquant_sizes8(C.byref(cfg), C.byref(B.lq_sizes8())) == B.LQ_ERR_SHAPE


def test_null_pointers():
    cfg, (cache, n) = _cfg(), _cache()
    assert B.logquant_workspace_init8(None, 4096) == B.logquant_workspace_init8(cfg, None) == B.LQ_ERR_NULL
    assert B._lib.logquant_sizes8(C.byref(cfg), None) == B.LQ_ERR_NULL
    for i in range(4):
        a = [cfg, cache, 4096, 4096]
        a[i] = None
        assert B.logquant_append8(*a, None, 1) == B.LQ_ERR_NULL
    assert B.logquant_read8(None, cache, 0, 1, 4096, 4096) == B.logquant_read8(cfg, None, 0, 1, 4096, 4096) == B.LQ_ERR_NULL
    assert B.logquant_read8(cfg, cache, 0, 1, None, None) == B.LQ_ERR_NULL
    for i in range(5):
        a = [cfg, cache, 4096, 4096, 4096]
        a[i] = None
        assert B.logquant_decode_attn8(a[0], a[1], a[2], 0.0, a[3], a[4]) == B.LQ_ERR_NULL
    for i in range(7):
        a = [cfg, cache] + [4096] * 5
        a[i] = None
        assert B.logquant_decode_step8(a[0], a[1], a[2], a[3], a[4], 0.0, a[5], a[6]) == B.LQ_ERR_NULL
    for name in ("k_codes", "v_codes", "k_scale", "v_scale", "k_tail", "v_tail", "seq_state", "n"):
        c, _ = _cache(**{name: B._I32P() if name == "n" else None})
        assert B.logquant_append8(cfg, c, 4096, 4096, None, 1) == B.LQ_ERR_NULL, name
        assert B.logquant_decode_attn8(cfg, c, 4096, 0.0, 4096, 4096) == B.LQ_ERR_NULL, name
    assert list(n) == [0, 0]


def test_buffers_off_16_bytes():
    cfg, (cache, _) = _cfg(), _cache((5, 5))
    assert B.logquant_workspace_init8(cfg, 4104) == B.LQ_ERR_SHAPE
    assert B.logquant_append8(cfg, cache, 4098, 4096, None, 1) == B.logquant_append8(cfg, cache, 4096, 4098, None, 1) == B.LQ_ERR_SHAPE
    assert B.logquant_read8(cfg, cache, 0, 1, 4098, None) == B.logquant_read8(cfg, cache, 0, 1, None, 4098) == B.LQ_ERR_SHAPE
    for i in range(3):
        a = [4096, 4096, 4096]
        a[i] = 4104
        assert B.logquant_decode_attn8(cfg, cache, a[0], 0.0, a[1], a[2]) == B.LQ_ERR_SHAPE
    for i in range(5):
        a = [4096] * 5
        a[i] = 4104
        assert B.logquant_decode_step8(cfg, cache, a[0], a[1], a[2], 0.0, a[3], a[4]) == B.LQ_ERR_SHAPE
    for name in ("k_codes", "v_codes", "k_scale", "v_scale", "k_tail", "v_tail", "seq_state"):
        c, _ = _cache((5, 5), **{name: 4100})
        assert B.logquant_decode_attn8(cfg, c, 4096, 0.0, 4096, 4096) == B.LQ_ERR_SHAPE, name


def test_counts_lengths_and_capacity():
    cfg = _cfg()
    for n in ((-1, 0), (0, 1025)):
        cache, _ = _cache(n)
        assert B.logquant_append8(cfg, cache, 4096, 4096, None, 1) == B.LQ_ERR_STATE
        assert B.logquant_read8(cfg, cache, 0, 1, 4096, 4096) == B.LQ_ERR_STATE
        assert B.logquant_decode_attn8(cfg, cache, 4096, 0.0, 4096, 4096) == B.LQ_ERR_STATE
        assert B.logquant_decode_step8(cfg, cache, 4096, 4096, 4096, 0.0, 4096, 4096) == B.LQ_ERR_STATE
    cache, n = _cache((1024, 1000))
    assert B.logquant_append8(cfg, cache, 4096, 4096, None, 0) == B.LQ_ERR_SHAPE
    assert B.logquant_append8(cfg, cache, 4096, 4096, [-1, 0], 4) == B.LQ_ERR_SHAPE
    assert B.logquant_append8(cfg, cache, 4096, 4096, [0, 5], 4) == B.LQ_ERR_SHAPE
    assert B.logquant_append8(cfg, cache, 4096, 4096, [1, 0], 4) == B.LQ_ERR_CAPACITY
    assert B.logquant_append8(cfg, cache, 4096, 4096, [0, 25], 25) == B.LQ_ERR_CAPACITY
    assert B.logquant_append8(cfg, cache, 4096, 4096, [0, 2 ** 31 - 1], 2 ** 31 - 1) == B.LQ_ERR_CAPACITY
    assert B.logquant_append8(cfg, cache, 4096, 4096, [0, 0], 4) == B.LQ_OK              # nobody takes a token: no launch
    assert B.logquant_decode_step8(cfg, cache, 4096, 4096, 4096, 0.0, 4096, 4096) == B.LQ_ERR_CAPACITY
    for t0, m in ((-1, 1), (0, 0), (0, 1025), (1025, 1), (1024, 1), (1000, 25), (2 ** 31 - 1, 2 ** 31 - 1)):
        assert B.logquant_read8(cfg, cache, t0, m, 4096, 4096) == B.LQ_ERR_SHAPE, (t0, m)
    cache2, _ = _cache((3, 0))
    assert B.logquant_read8(cfg, cache2, 3, 1000, 4096, 4096) == B.LQ_OK                 # nothing of the range is there
    assert list(n) == [1024, 1000]


def test_the_owner_of_buffers_refuses_a_cpu():
    with pytest.raises(ValueError):
        B.DeviceCache8(_cfg(), device="cpu")
