"""Helpers of the GPU tests of the 8-bit cache: inputs, the oracle's caches beside it, and bounds."""
import numpy as np
import torch

from oracle import cache8
from paper_2503_19950_amd import binding

DEVICE = "cuda:0"
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
HALF_STEP = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}      # half a step of T relative to the value


def rows(seed, B, Hkv, L, d, dtype, gain=1.0, outliers=True):
    """[B][Hkv][L][d] on the CPU: normal values, four channels ten times larger."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((B, Hkv, L, d), generator=g)
    if outliers:
        x[..., torch.randperm(d, generator=g)[:4]] *= 10
    return (x * gain).to(TYPES[dtype])


def make(B, Hq, Hkv, d, G, dtype, capacity):
    return binding.DeviceCache8(binding.make_config8(B, Hq, Hkv, d, G, dtype, capacity), DEVICE, poison=True)


def f64(x):
    return x.double().cpu().numpy()


def bits16(x):
    """Bits of fp64 values that T holds exactly."""
    return x.view(torch.int16).cpu().numpy()


def check_state(cache, which, b, h, oc):
    """One slice of the device cache against the oracle's, bit for bit."""
    cfg, d, G = cache.cfg, cache.cfg.d, cache.cfg.block
    codes, scales, tail = oc.blocks()
    assert cache.n[b] == len(oc.rows)
    bh = b * cfg.Hkv + h
    flat = getattr(cache, which + "_codes").view(cfg.B * cfg.Hkv, -1)[bh, :codes.size].cpu().numpy()
    assert np.array_equal(cache8.gather(flat, cache8.code_index, which, len(codes), d), codes), (which, b, h, "codes")
    got = getattr(cache, which + "_scale").view(torch.float32).view(cfg.B * cfg.Hkv, -1)[bh, :len(scales)]
    assert np.array_equal(f64(got), scales), (which, b, h, "scales")
    flat = getattr(cache, which + "_tail").view(torch.int16).view(cfg.B * cfg.Hkv, -1)[bh].cpu().numpy()
    want = bits16(torch.from_numpy(tail).to(cache.dtype))
    assert np.array_equal(cache8.gather(flat, cache8.tail_index, which, len(tail), d), want), (which, b, h, "tail")


class Oracle:
    """One pair of oracle caches for every slice of a device cache."""

    def __init__(self, cache, dtype):
        self.cfg = cfg = cache.cfg
        self.k, self.v = ([[cache8.Cache8(cfg.block, cfg.d, dtype) for _ in range(cfg.Hkv)] for _ in range(cfg.B)] for _ in "kv")

    def append(self, K, V, n_new=None):
        for b in range(self.cfg.B):
            n = K.shape[2] if n_new is None else n_new[b]
            for h in range(self.cfg.Hkv):
                self.k[b][h].append(f64(K[b, h, :n]))
                self.v[b][h].append(f64(V[b, h, :n]))

    def check(self, cache):
        for b in range(self.cfg.B):
            for h in range(self.cfg.Hkv):
                check_state(cache, "k", b, h, self.k[b][h])
                check_state(cache, "v", b, h, self.v[b][h])


def attention_and_bound(q, K, V, scale, dtype):
    """fp64 attention of q [g][d] over K, V [n][d], and how far a kernel's output may be from it:
      A = sum p |v|, what the weights spread over;
      the rounding of a probability to fp16, 2^-11 of each, of A in all;
      logits: fp32 sums of d exact products, each addition off by at most 2^-24 of the products' magnitudes, and the
        constants folded into the exponent (two roundings of the logit itself, and of the reference, in powers of two): a
        relative error e of every weight moves the output by at most 2 e A;
      sums over n tokens in fp32 (32 at a time, then a running sum): 2^-24 per step of A, and exp2 2^-22;
      the rounding of the output to T: half a step, or half of T's smallest number."""
    q, K, V = f64(q), np.asarray(K), np.asarray(V)
    d, n = q.shape[-1], len(K)
    if not n:
        return np.zeros_like(q), np.zeros_like(q)
    scale = scale if scale > 0 else d ** -0.5
    s = scale * (q @ K.T)
    p = np.exp(s - s.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    o, A = p @ V, p @ np.abs(V)
    spread = scale * (np.abs(q) @ np.abs(K).T).max(-1, keepdims=True)
    e = (d + 8) * 2.0 ** -24 * spread + 4 * 2.0 ** -24 * np.abs(s).max(-1, keepdims=True) + 2.0 ** -22
    inner = A * (2.0 ** -11 + 2 * e + (64 + n / 16) * 2.0 ** -24)
    return o, inner + HALF_STEP[dtype] * (np.abs(o) + inner) + (2.0 ** -25 if dtype == "f16" else 0)


def check_output(out, q, oracle, dtype, scale=0.0, rows_of=None):
    """All heads of the given batch rows (default: all)."""
    cfg = oracle.cfg
    gh = cfg.Hq // cfg.Hkv
    got = f64(out)
    for b in range(cfg.B) if rows_of is None else rows_of:
        for h in range(cfg.Hkv):
            at = slice(h * gh, (h + 1) * gh)
            want, bound = attention_and_bound(q[b, at], oracle.k[b][h].held(), oracle.v[b][h].held(), scale, dtype)
            off = np.abs(got[b, at] - want)
            assert (off <= bound).all(), "row %d kv head %d: off by %.3g, bound %.3g" % (
                b, h, off[~(off <= bound)].max(), bound[~(off <= bound)].min())
