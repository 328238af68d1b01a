"""Plain 64-bit definitions of the low-bit formats and operators (numpy), the
reference of their tests: e4m3 cache blocks, e2m1 weight groups."""
import numpy as np

BLOCK = 32


def _grid(bits_e, bits_m, bias):
    code = np.arange(1 << (bits_e + bits_m))
    e, m = code >> bits_m, (code & ((1 << bits_m) - 1)) / (1 << bits_m)
    return np.where(e == 0, m * 2.0 ** (1 - bias), (1 + m) * 2.0 ** (e - bias))


E4M3 = _grid(4, 3, 7)
E4M3[127] = np.nan
E4M3 = np.concatenate([E4M3, -E4M3])
E2M1 = np.concatenate([_grid(2, 1, 1), -_grid(2, 1, 1)])


def pow2(scale):
    return np.ldexp(1.0, np.asarray(scale, np.int64) - 127)


def _nearest(x, grid):
    """Codes of the grid's values nearest to |x| <= grid[-1], ties to even."""
    a = np.abs(x)
    hi = np.clip(np.searchsorted(grid, a), 1, len(grid) - 1)
    up, down = grid[hi] - a, a - grid[hi - 1]
    c = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, hi - 1)
    return np.where(a == 0, 0, c)


def exponent(amax, largest):
    """The smallest e in [-100, 120] with amax <= largest * 2^e; 0 for 0."""
    if amax == 0:
        return 0
    e = -100
    while e < 120 and amax > largest * 2.0 ** e:
        e += 1
    return e


def encode_e4m3(v):
    """One block's values -> (codes, scale byte)."""
    fin = np.isfinite(v)
    e = exponent(float(np.abs(np.where(fin, v, 0)).max(initial=0)), 448.0)
    y = np.ldexp(np.where(fin, v, 0), -e)
    c = _nearest(y, E4M3[:127]) + 128 * np.signbit(y)
    return np.where(fin, c, 0x7f).astype(np.uint8), e + 127


class Cache:
    """One layer's cache in natural order: codes [2][Hkv][rows][D], scales
    [2][Hkv][blocks]."""

    def __init__(self, cache):
        k, v = cache.k.cpu().numpy(), cache.v.cpu().numpy().swapaxes(-1, -2)
        self.codes = np.stack([a.reshape(a.shape[0], -1, a.shape[-1]) for a in (k, v)]).copy()
        self.scales = np.stack([cache.k_scale.cpu().numpy(), cache.v_scale.cpu().numpy()])
        self.scales = self.scales.astype(np.uint8).copy()

    def values(self):
        return E4M3[self.codes] * np.repeat(pow2(self.scales), BLOCK, -1)[..., None]

    def write(self, rows, start):
        """rows [2][Hkv][n][D] (64 bits) to cache rows start .."""
        end = start + rows.shape[2]
        held = self.values()
        for b in range(start // BLOCK, (end - 1) // BLOCK + 1 if end > start else 0):
            lo, hi = b * BLOCK, min(end, (b + 1) * BLOCK)
            for i in range(2):
                for g in range(rows.shape[1]):
                    v = held[i, g, lo:hi].copy()
                    at = max(start, lo)
                    v[at - lo:] = rows[i, g, at - start:hi - start]
                    self.codes[i, g, lo:hi], self.scales[i, g, b] = encode_e4m3(v)

    def compact(self, accept, path, gamma, ctx):
        n = min(max(int(accept), 0), gamma - 1)
        src = [ctx + (p if t <= p < gamma else t) for t, p in enumerate(path[:n + 1])]
        self.write(self.values()[:, :, src], ctx)

    def check(self, cache):
        got = Cache(cache)
        np.testing.assert_array_equal(got.scales, self.scales)
        np.testing.assert_array_equal(got.codes, self.codes)


def attention(q, k, v, visible, scale):
    """q [g][Hq][D], k, v [Hkv][n][D] (held values), visible [g][n] -> out and
    sum_j p_j |v_j|, both [g][Hq][D], and the largest sum_d |q_d k_jd| of each
    row over its visible keys [g][Hq]."""
    g, hq, d = q.shape
    grp = hq // k.shape[0]
    out, mass, dots = np.empty(q.shape), np.empty(q.shape), np.empty((g, hq))
    for h in range(hq):
        kk, vv = k[h // grp], v[h // grp]
        z = np.where(visible, q[:, h] @ np.where(np.isfinite(kk), kk, 0).T * scale, -np.inf)
        p = np.exp(z - z.max(1, keepdims=True))
        p /= p.sum(1, keepdims=True)
        live = np.where(visible.any(0)[:, None], vv, 0)
        out[:, h], mass[:, h] = p @ live, p @ np.abs(live)
        sums = np.abs(q[:, h]) @ np.abs(np.where(np.isfinite(kk), kk, 0)).T
        dots[:, h] = np.where(visible, sums, 0).max(1)
    return out, mass, dots


def encode_e2m1(w):
    """Weight [rows][cols] -> (codes [rows][cols/2], scales [rows][cols/32])."""
    rows, cols = w.shape
    grp = w.reshape(rows, cols // 32, 32)
    scales = np.empty(grp.shape[:2], np.uint8)
    codes = np.empty(grp.shape, np.uint8)
    for r in range(rows):
        for i in range(cols // 32):
            x = grp[r, i]
            e = exponent(float(np.abs(np.where(np.isfinite(x), x, 0)).max()), 6.0)
            y = np.ldexp(np.where(np.isfinite(x), x, 0), -e)
            codes[r, i] = _nearest(y, E2M1[:8]) + 8 * np.signbit(x)
            scales[r, i] = e + 127 if np.isfinite(x).all() else 255
    c = codes.reshape(rows, cols)
    return c[:, 0::2] | (c[:, 1::2] << 4), scales


def decode_e2m1(codes, scales):
    w = np.empty((codes.shape[0], 2 * codes.shape[1]))
    w[:, 0::2], w[:, 1::2] = E2M1[codes & 15], E2M1[codes >> 4]
    s = np.where(scales == 255, np.nan, pow2(scales))
    return w * np.repeat(s, 32, 1)
