"""Helpers of the GPU tests of rotary positions and of the paged cache: inputs, a model of the cache beside it, and bounds."""
import numpy as np
import torch

from oracle import paged
from paper_2503_19950_amd import binding

DEVICE = "cuda:0"
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
HALF_STEP = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}      # half a step of T relative to the value
TINY = {"f16": 2.0 ** -25, "bf16": 0.0}                 # half of T's smallest number, where it can matter


def rows(seed, *shape, dtype, gain=1.0, outliers=False):
    """Normal values on the CPU; four channels ten times larger with `outliers`."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g)
    if outliers:
        x[..., torch.randperm(shape[-1], generator=g)[:4]] *= 10
    return (x * gain).to(TYPES[dtype])


def f64(x):
    return x.double().cpu().numpy()


def rotated_and_bound(x, positions, freq, interleaved, factor, dtype):
    """fp64 turned rows of x [..][L][d], and how far a kernel's may be from them.  An angle in turns, |p f| / 2 pi, is off by
    three fp64 roundings of it and rounded to fp32 within half a turn (2^-26); the cosine and sine of it are off by at most 4
    units of 2^-24 each, their product with the factor by one; the two products and their sum by 2 units of 2^-24 of both terms;
    and the result is rounded to T."""
    x = np.asarray(x, np.float64)
    y = paged.rotate(x, positions, freq, interleaved, factor)
    dims = 2 * len(freq)
    one, two = paged.partners(dims, interleaved)
    turns = np.abs(np.asarray(positions, np.float64)[:, None] * np.asarray(freq)) / (2 * np.pi)
    e = 2 * np.pi * (3 * 2.0 ** -53 * turns + 2.0 ** -26) + 5 * 2.0 ** -24 + 2 * 2.0 ** -24
    inner = np.zeros_like(x)
    inner[..., one] = inner[..., two] = (np.abs(x[..., one]) + np.abs(x[..., two])) * abs(factor) * e
    bound = inner + HALF_STEP[dtype] * (np.abs(y) + inner) + TINY[dtype]
    bound[..., dims:] = 0.0
    return y, bound


def attention_and_bounds(q, K, V, scale, dtype, softcap=0.0, slopes=None, window=0):
    """fp64 attention of q [g][d] over K, V [n][d], its probabilities, and how far a kernel's output and probabilities may be
    from them.
      A token's score is off by at most err (natural units): an fp32 sum of d exact products, 2^-24 of their magnitudes for each
      addition and 8 for the order of a matrix instruction's; a rounding, and that of a constant, at each of the product with the
      scale, the cap, the bias and the factor log2(e), 8 of 2^-24 of the magnitudes in all; the tanh, off by at most 2^-21;
      the subtraction of the reference and exp2, 2^-22 each.
      Weights p (1 + e_t), |e_t| <= 1.1 err_t for err_t < 0.1, move the output sum p v / sum p by at most sum p e |v| + sum p e sum p |v|.
      What the rounding of a probability into operands leaves: 2^-22 of it; sums in fp32: (64 + n / 16) 2^-24 of sum p |v|;
      the rounding of the output to T: half a step, or half of T's smallest number."""
    q, K, V = np.asarray(q, np.float64), np.asarray(K, np.float64), np.asarray(V, np.float64)
    d, n = q.shape[-1], len(K)
    if not n:
        return np.zeros_like(q), np.zeros((len(q), 0)), np.zeros_like(q), np.zeros((len(q), 0))
    scale = scale if scale > 0 else d ** -0.5
    s = paged.scores(q, K, scale, softcap, slopes, window)
    p = paged.probabilities(s)
    raw = scale * np.abs(q @ K.T)
    bias = 0 if slopes is None else np.abs(np.asarray(slopes, np.float64)[:, None] * (n - 1 - np.arange(n)))
    err = (d + 8) * 2.0 ** -24 * scale * (np.abs(q) @ np.abs(K).T) + 8 * 2.0 ** -24 * (raw + bias + np.abs(np.where(p > 0, s, 0)))
    err = err + softcap * 2.0 ** -21 + 2 * 2.0 ** -22
    err = np.where(p > 0, err, 0)
    # (a token further below than exp can tell has no weight on either side: what its error could make of it is below this)
    assert (err[p > 1e-30] < 0.1).all()
    err = np.where(p > 1e-30, 1.1 * err, 0)
    o, A = p @ V, p @ np.abs(V)
    all_of = (p * err).sum(-1, keepdims=True)
    inner = (p * err) @ np.abs(V) + all_of * A + A * (2.0 ** -22 + (64 + n / 16) * 2.0 ** -24) + n * 1e-30 * np.abs(V).max(initial=0)
    p_bound = p * (err + all_of + (64 + n / 16) * 2.0 ** -24 + 2.0 ** -22) + 1e-29
    return o, p, inner + HALF_STEP[dtype] * (np.abs(o) + inner) + TINY[dtype], p_bound


def make(B, Hq, Hkv, d, page, dtype, max_pages, n_pages=None, weighted=False, seed=0):
    """A poisoned cache whose free pages are in a scattered order."""
    n_pages = n_pages or B * max_pages * (2 if weighted else 1) + 3
    cache = binding.DeviceCachePaged(binding.make_config_paged(B, Hq, Hkv, d, page, dtype, n_pages, max_pages, weighted), DEVICE, poison=True)
    order = list(cache.free)
    np.random.RandomState(seed).shuffle(order)
    cache.free = dict.fromkeys(order)
    return cache


class Model:
    """What every row of a cache holds: K, V [Hkv][n][d] and weights [Hkv][n], fp64."""

    def __init__(self, cache, dtype):
        self.cfg, self.dtype = cache.cfg, dtype
        c = cache.cfg
        self.K = [np.zeros((c.Hkv, 0, c.d)) for _ in range(c.B)]
        self.V = [np.zeros((c.Hkv, 0, c.d)) for _ in range(c.B)]
        self.w = [np.zeros((c.Hkv, 0)) for _ in range(c.B)]

    def append(self, K, V, n_new=None):
        """K, V: CPU tensors [B][Hkv][n][d] of T (turned already)."""
        for b in range(self.cfg.B):
            n = K.shape[2] if n_new is None else n_new[b]
            self.K[b] = np.concatenate([self.K[b], f64(K[b, :, :n])], 1)
            self.V[b] = np.concatenate([self.V[b], f64(V[b, :, :n])], 1)
            self.w[b] = np.concatenate([self.w[b], np.zeros((self.cfg.Hkv, n))], 1)

    def evict(self, keep, recent):
        for b in range(self.cfg.B):
            x = keep if isinstance(keep, int) else keep[b]
            if self.K[b].shape[1] <= x:
                continue
            at = [paged.kept(self.w[b][h], x, recent) for h in range(self.cfg.Hkv)]
            self.K[b], self.V[b], self.w[b] = (np.stack([t[h][at[h]] for h in range(self.cfg.Hkv)]) for t in (self.K[b], self.V[b], self.w[b]))

    def check_output(self, out, q, scale=0.0, softcap=0.0, slopes=None, window=0, weights=None, skip=()):
        """All rows; adds the probabilities to the model's weights where `weights` (the cache's, fp32) is given, within their
        bounds, and goes on from those."""
        c = self.cfg
        gh = c.Hq // c.Hkv
        got, q = f64(out), f64(q)
        sl = None if slopes is None else f64(slopes)
        for b in range(c.B):
            if b in skip:
                continue
            for h in range(c.Hkv):
                at = slice(h * gh, (h + 1) * gh)
                want, p, bound, p_bound = attention_and_bounds(q[b, at], self.K[b][h], self.V[b][h], scale, self.dtype, softcap,
                                                               None if sl is None else sl[at], window)
                off = np.abs(got[b, at] - want)
                assert (off <= bound).all(), "row %d kv head %d: off by %.3g, bound %.3g" % (
                    b, h, off[~(off <= bound)].max(), bound[~(off <= bound)].min())
                if weights is not None:
                    now = weights[b, h, :self.K[b].shape[1]]
                    exp = self.w[b][h] + p.sum(0)
                    room = p_bound.sum(0) + (gh + 2) * 2.0 ** -24 * exp
                    assert (np.abs(now - exp) <= room).all(), (b, h, np.abs(now - exp).max())
                    self.w[b][h] = now


def live_weights(cache):
    """fp64 [B][Hkv][cap] of every row's own half."""
    w = f64(cache.weights)
    return np.stack([w[cache.cur[b], b] for b in range(cache.cfg.B)])


def pools(cache):
    """Bits of both pools, flat."""
    return {w: getattr(cache, w + "_pages").view(torch.int16).cpu().numpy().copy() for w in "kv"}


def addresses(cache, which, b, h, n):
    """[n][d] places in the pool of row b's first n tokens."""
    c = cache.cfg
    t = np.arange(n)
    g = np.array(cache.ids[cache.cur[b]][b], dtype=np.int64)[t // c.page]
    return paged.page_index(which, g[:, None], h, (t % c.page)[:, None], np.arange(c.d)[None], c.Hkv, c.page, c.d)


def check_rows(cache, model, before, written=True):
    """The pool holds the model's rows, bit for bit, and everything else as in `before`."""
    now = pools(cache)
    want = {w: before[w].copy() for w in "kv"}
    for b in range(cache.cfg.B):
        for h in range(cache.cfg.Hkv):
            for w, x in (("k", model.K[b][h]), ("v", model.V[b][h])):
                assert cache.n[b] == len(x)
                if len(x):
                    want[w][addresses(cache, w, b, h, len(x))] = torch.from_numpy(x).to(cache.dtype).view(torch.int16).numpy()
    for w in "kv":
        bad = np.nonzero(now[w] != want[w])[0]
        assert not len(bad), (w, len(bad), bad[:5])
