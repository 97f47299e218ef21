"""The 8-bit cache of one (batch row, kv head) slice and one tensor, fp64.  Test infrastructure only.

Blocks of G consecutive tokens become e4m3 codes with one power-of-two scale; the newest tokens, fewer than G, stay at
the cache type.  Everything here follows from the definition in include/logquant.h, by searching and sorting values rather
than by the bit arithmetic of the kernels.
"""
import numpy as np


def e4m3_values():
    """The 127 non-negative finite values of e4m3, by byte: subnormals m * 2^-9, normals (1 + m/8) * 2^(e-7)."""
    v = [m * 2.0 ** -9 for m in range(8)]
    v += [(1 + m / 8) * 2.0 ** (e - 7) for e in range(1, 16) for m in range(8)]
    return np.array(v[:127])                   # byte 0x7F is NaN


VALUES = e4m3_values()


def to_bytes(y):
    """fp64 values, |y| <= 448 -> e4m3 bytes, nearest, ties to the even byte."""
    y = np.asarray(y, np.float64)
    x = np.abs(y)
    assert (x <= 448).all()
    hi = np.searchsorted(VALUES, x)            # first value >= x
    lo = np.maximum(hi - 1, 0)
    below, above = x - VALUES[lo], VALUES[hi] - x
    pick = np.where((above < below) | ((above == below) & (hi % 2 == 0)), hi, lo)
    return (pick + np.where(np.signbit(y), 128, 0)).astype(np.uint8)


def from_bytes(u):
    u = np.asarray(u, np.uint8)
    return np.where(u >= 128, -1.0, 1.0) * VALUES[u & 127]


def cut(dtype):
    return 1.875 * 2.0 ** (127 if dtype == "bf16" else 15)


def scale_of(top):
    """2^e, e >= -126 the smallest integer with top <= 448 * 2^e."""
    e = -126
    while top > 448 * 2.0 ** e:
        e += 1
    return 2.0 ** e


class Cache8:
    def __init__(self, G, d, dtype):
        self.G, self.d, self.dtype = G, d, dtype
        self.rows = np.zeros((0, d))           # every token as it came

    def append(self, x):
        self.rows = np.concatenate([self.rows, np.asarray(x, np.float64)])

    def blocks(self):
        """(bytes [full][d], scales [blocks], tail [n % G][d])."""
        full = len(self.rows) // self.G * self.G
        x = np.clip(self.rows[:full], -cut(self.dtype), cut(self.dtype)).reshape(-1, self.G, self.d)
        s = np.array([scale_of(np.abs(b).max()) for b in x])
        return to_bytes((x / s[:, None, None]).reshape(-1, self.d)) if full else np.zeros((0, self.d), np.uint8), s, self.rows[full:]

    def held(self):
        """What the cache holds of every token: values of T as fp64 [n][d]."""
        u, s, tail = self.blocks()
        return np.concatenate([from_bytes(u) * np.repeat(s, self.G)[:, None], tail])


# ---- physical layout: index of (token or tail row, channel) within a slice ---------------------
def kperm(x):
    return 8 * ((x % 16) // 4) + 4 * (x // 16) + x % 4


def code_index(which, t, c, d):
    if which == "k":
        return (((t // 32) * (d // 32) + c // 32) * 64 + 16 * ((c % 32) // 8) + t % 16) * 16 + 8 * ((t % 32) // 16) + c % 8
    k = kperm(t % 32)
    return (((t // 32) * (d // 32) + c // 32) * 64 + 16 * (k // 8) + c % 16) * 16 + 8 * ((c % 32) // 16) + k % 8


def tail_index(which, r, c, d):
    if which == "k":
        return (((r // 16) * (d // 32) + c // 32) * 64 + 16 * ((c % 32) // 8) + r % 16) * 8 + c % 8
    k = kperm(r % 32)
    return (((r // 32) * (d // 16) + c // 16) * 64 + 16 * (k // 8) + c % 16) * 8 + k % 8


def gather(flat, index, which, n, d):
    """Rows 0..n-1 of a slice's flat buffer, [n][d]."""
    t, c = np.arange(n)[:, None], np.arange(d)[None]
    return np.asarray(flat)[index(which, t, c, d)]
