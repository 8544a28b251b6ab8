"""Plain 64-bit forms of the pointwise layers' operators, on the CPU: random numbers by counter, dropout, group norm and its
gradients with bounds of what fp32 may be off by, rows in 4 bits."""
import math

import numpy as np
import torch

U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16
LOW = np.uint64(0xFFFFFFFF)
GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def philox(counter, key):
    """Ten rounds of Philox 4x32: counter [.., 4], key [2], numbers below 2^32."""
    x = [np.asarray(counter[..., i], np.uint64) for i in range(4)]
    k = [np.uint64(v) for v in key]
    for _ in range(10):
        a, b = np.uint64(0xD2511F53) * x[0], np.uint64(0xCD9E8D57) * x[2]
        x = [(b >> np.uint64(32)) ^ x[1] ^ k[0], b & LOW, (a >> np.uint64(32)) ^ x[3] ^ k[1], a & LOW]
        k = [(k[0] + np.uint64(0x9E3779B9)) & LOW, (k[1] + np.uint64(0xBB67AE85)) & LOW]
    return np.stack(x, -1)


def uniform16(seed, step, site, rows, c):
    """Sixteen random bits for every element [rows (numbers of them), c]."""
    rows = np.arange(rows) if np.isscalar(rows) else np.asarray(rows)
    groups = (c + 7) // 8
    g = rows[:, None].astype(np.uint64) * np.uint64(groups) + np.arange(groups, dtype=np.uint64)
    one = np.ones_like(g)
    seed, step = seed & (2 ** 64 - 1), step & (2 ** 64 - 1)
    counter = np.stack([g & LOW, one * np.uint64(site), one * np.uint64(step & 0xFFFFFFFF), one * np.uint64(step >> 32)], -1)
    w = philox(counter, (seed & 0xFFFFFFFF, seed >> 32))
    u = np.stack([w & np.uint64(0xFFFF), w >> np.uint64(16)], -1).astype(np.int64)
    return u.reshape(len(rows), 8 * groups)[:, :c]


def threshold(p):
    return int(math.floor(65536 * float(np.float32(p)) + 0.5))


def factors(u, p):
    """0, or what makes up for what is dropped."""
    t = threshold(p)
    return np.where(u >= t, 65536.0 / (65536 - t) if t < 65536 else 0.0, 0.0)


# ---- rows in 4 bits ----------------------------------------------------------------------------------------------

def to_bits(x, u=None):
    """Codes q, scales and values of rows [n, c] (float64 numpy), element by element from the definition."""
    n, c = x.shape
    blocks = -(-c // 32)
    v = np.zeros((n, blocks * 32))
    v[:, :c] = x
    v = v.reshape(n, blocks, 32)
    fine = np.isfinite(v).all(2)
    a = np.where(fine[..., None], np.abs(v), 0.0)
    amax = a.max(2)
    s = np.full((n, blocks), -126)
    some = amax > 0
    s[some] = np.maximum(np.floor(np.log2(amax[some])).astype(int) - 4, -126)
    for _ in range(6):                                 # the smallest power of two with which nothing rounds past 6
        top = np.ldexp(amax, -s)
        s = np.where((top >= 7) if u is None else (top > 6), s + 1, s)
    s = np.minimum(s, 125)
    a = np.minimum(np.ldexp(a, -s[..., None]), 6.0)
    low = np.searchsorted(GRID, a, side="right") - 1
    high = np.minimum(low + 1, 7)
    gap = np.where(high > low, GRID[high] - GRID[low], 1.0)
    rest = (a - GRID[low]) / gap
    if u is None:
        up = (rest > 0.5) | ((rest == 0.5) & (low % 2 == 1))
    else:
        w = np.zeros((n, blocks * 32), np.int64)
        w[:, :c] = u
        up = np.floor(rest * 65536) + w.reshape(v.shape) >= 65536
    code = np.where(up, high, low)
    values = np.copysign(np.ldexp(GRID[code], s[..., None]), v)
    code = np.where(fine[..., None], code + 8 * np.signbit(v), 0).astype(np.uint8).reshape(n, -1)
    values = np.where(fine[..., None], values, np.nan).reshape(n, -1)[:, :c]
    scales = np.zeros((n, 4 * (-(-c // 128))), np.uint8)
    scales[:, :blocks] = np.where(fine, s + 127, 255)
    return code[:, 0::2] | code[:, 1::2] << 4, scales, values


def from_bits(q, scales, c):
    code = np.stack([q & 15, q >> 4], -1).reshape(q.shape[0], -1)[:, :c]
    e = scales[:, np.arange(c) // 32].astype(int)
    v = np.where(code >= 8, -1.0, 1.0) * GRID[code & 7]
    return np.where(e == 255, np.nan, np.ldexp(v, e - 127))


# ---- norms -------------------------------------------------------------------------------------------------------

def activate(z, act):
    return {"none": lambda v: v, "relu": torch.relu, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu}[act](z)


def bounds_of(offsets, n):
    return [(0, n)] if offsets is None else [(int(a), int(b)) for a, b in zip(offsets[:-1], offsets[1:])]


def group_norm(x, groups, w, b, offsets, act, eps, factor):
    """y, mean_rstd and how far fp32 may be off y and the statistics (rows of no cloud: zero).

    A sum in fp32 is off by at most its depth (additions on the longest way from a term to the result) times u times the sum of the
    magnitudes.  The kernels' depth is below 64 + rows / 32 here.  With k a cloud's first row the sums are those of x - k and its square, so in units of the
    deviation the mean is off by D u P, P = mean |x - k| rstd + |mean| rstd, and rstd by D u Q / 2 of itself, Q = mean (x - k)^2 rstd^2."""
    x = x.double().cpu()
    n, c = x.shape
    width = c // groups
    w = torch.ones(c, dtype=torch.float64) if w is None else w.double().cpu()
    b = torch.zeros(c, dtype=torch.float64) if b is None else b.double().cpu()
    y, off_y = torch.zeros_like(x), torch.zeros_like(x)
    ranges = bounds_of(offsets, n)
    stats, off_stats = torch.zeros(len(ranges), groups, 2, dtype=torch.float64), torch.zeros(len(ranges), groups, 2, dtype=torch.float64)
    for i, (lo, hi) in enumerate(ranges):
        if lo >= hi:
            continue
        v = x[lo:hi].view(hi - lo, groups, width)
        mean = v.mean((0, 2))
        d = v - mean[None, :, None]
        var = (d * d).mean((0, 2))
        rstd = 1.0 / torch.sqrt(var + eps)
        k = x[lo].view(1, groups, width)
        depth = 64 + (hi - lo) / 32
        P = ((v - k).abs().mean((0, 2)) + mean.abs()) * rstd
        Q = ((v - k) ** 2).mean((0, 2)) * rstd ** 2
        stats[i] = torch.stack([mean, rstd], 1)
        off_stats[i] = torch.stack([depth * U * P / rstd, depth * U * (Q + 1) * rstd], 1)
        v = d * rstd[None, :, None]
        off_v = depth * U * (P[None, :, None] + v.abs() * (Q + 1)[None, :, None]) + 4 * U * (x[lo:hi].view_as(v).abs() * rstd[None, :, None])
        v, off_v = v.reshape(hi - lo, c), off_v.reshape(hi - lo, c)
        z = w * v + b
        f = 1.0 if factor is None else torch.from_numpy(factor[lo:hi])
        out = activate(z, act)
        y[lo:hi] = f * out
        # slopes are at most 1.13; the activations' own error: exp and the reciprocal of two units, erf of four
        off_y[lo:hi] = f * (1.13 * w.abs() * off_v + 16 * U * (z.abs() + (w * v).abs() + b.abs() + out.abs()))
    return y, stats, off_y, off_stats


def slope(z, act):
    if act == "relu":
        return (z > 0).double()
    if act == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z / math.sqrt(2))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    return torch.ones_like(z)


def group_norm_grads(dy, x, stats, w, b, offsets, act, factor):
    """(value, bound) of dx, dw, db from the statistics as given; bounds as in group_norm (the second derivatives are at most 0.8)."""
    x, dy, stats = x.double().cpu(), dy.double().cpu(), stats.double().cpu()
    n, c = x.shape
    groups = stats.shape[1]
    width = c // groups
    w = torch.ones(c, dtype=torch.float64) if w is None else w.double().cpu()
    b = torch.zeros(c, dtype=torch.float64) if b is None else b.double().cpu()
    dx, off_x = torch.zeros_like(x), torch.zeros_like(x)
    dw, db, off_w, off_b = (torch.zeros(c, dtype=torch.float64) for _ in range(4))
    for i, (lo, hi) in enumerate(bounds_of(offsets, n)):
        if lo >= hi:
            continue
        rows = hi - lo
        depth = 64 + rows / 32
        mean, rstd = (stats[i, :, k].repeat_interleave(width) for k in (0, 1))
        v = (x[lo:hi] - mean) * rstd
        off_v = 4 * U * (x[lo:hi].abs() + mean.abs()) * rstd
        z = w * v + b
        g = dy[lo:hi] * (1.0 if factor is None else torch.from_numpy(factor[lo:hi]))
        dz = g * slope(z, act)
        off_z = w.abs() * off_v + 4 * U * ((w * v).abs() + b.abs())
        off_dz = g.abs() * (0.8 * off_z * (act != "none") + 16 * U * (1 + z.abs()))
        dw += (dz * v).sum(0)
        db += dz.sum(0)
        off_w += (off_dz * v.abs() + dz.abs() * off_v + 4 * U * (dz * v).abs()).sum(0) + depth * U * (dz * v).abs().sum(0)
        off_b += off_dz.sum(0) + depth * U * dz.abs().sum(0)

        def mean_of(t):
            return t.view(rows, groups, width).mean((0, 2)).repeat_interleave(width)

        t1, t2 = w * dz, w * dz * v
        m1, m2 = mean_of(t1), mean_of(t2)
        off1 = mean_of(w.abs() * off_dz) + depth * U * mean_of(t1.abs())
        off2 = mean_of(w.abs() * (off_dz * v.abs() + dz.abs() * off_v)) + depth * U * mean_of(t2.abs())
        dx[lo:hi] = rstd * (t1 - m1 - v * m2)
        off_x[lo:hi] = rstd * (w.abs() * off_dz + off1 + v.abs() * off2 + off_v * m2.abs() + 8 * U * (t1.abs() + m1.abs() + (v * m2).abs()))
    return (dx, off_x), (dw, off_w), (db, off_b)
