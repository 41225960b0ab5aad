"""Definitions in 64 bits, on the CPU, of the operators of a serving loop, and how far a kernel may be from them."""
import numpy as np
import torch

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def half_step(dt):
    return torch.finfo(dt).eps / 2


def smallest_step(dt):
    """Half the distance of the numbers next to zero (what a rounding is off by below the normal range)."""
    return {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}[dt]


def rotate(x, pos, dim, base=10000.0, scale=1.0, interleaved=False):
    """x [n, heads, d], pos [n] -> float64, and what |a| + |b| of each value's pair is."""
    x = x.double()
    ang = pos.double()[:, None, None] * scale * base ** (-torch.arange(dim // 2, dtype=torch.float64) * 2 / dim)
    c, s = ang.cos(), ang.sin()
    y, mag = x.clone(), x.abs()
    sl = (slice(0, dim, 2), slice(1, dim, 2)) if interleaved else (slice(0, dim // 2), slice(dim // 2, dim))
    a, b = x[..., sl[0]], x[..., sl[1]]
    y[..., sl[0]], y[..., sl[1]] = a * c - b * s, a * s + b * c
    mag[..., sl[0]] = mag[..., sl[1]] = a.abs() + b.abs()
    return y, mag


def check_rotated(got, want, mag, dt):
    """The fraction of a turn as a float is 2^-26 of a turn off at most (9.4e-8), sine and cosine two units of 2^-24 each, two products
    and a sum half a unit each: under 5e-7 of |a| + |b|.  Then one rounding to dt."""
    tol = half_step(dt) * want.abs() * 1.001 + 5e-7 * mag + smallest_step(dt)
    far = (got.double().cpu() - want).abs() - tol
    assert far.max() <= 0, float(far.max())


def attend(q, k, v, scale, seen=None):
    """One sequence: q [m, heads, d], k, v [n, kv heads, d] -> float64 [m, heads, d], the values' weighted magnitude sum p|v| of the
    same shape, and the largest scale sum |q||k|.  seen [m, n]: which keys a query sees; what it does not see does not enter."""
    m, nh, d = q.shape
    n, nk, _ = k.shape
    share = nh // nk
    out, mag = torch.zeros(m, nh, d, dtype=torch.float64), torch.zeros(m, nh, d, dtype=torch.float64)
    most = 0.0
    for i in range(m):
        at = torch.arange(n) if seen is None else seen[i].nonzero()[:, 0]
        if len(at) == 0:
            continue
        for h in range(nh):
            kk, vv, qq = k[at, h // share].double(), v[at, h // share].double(), q[i, h].double()
            p = torch.softmax(kk @ qq * scale, 0)
            out[i, h], mag[i, h] = p @ vv, p @ vv.abs()
            most = max(most, float((kk.abs() @ qq.abs()).max()) * abs(scale))
    return out, mag, most


def check_attended(got, want, mag, most, n, dt, weight_step=0.0):
    """A score is a float sum of d products (256 at most) of magnitude `most` in all: (d + 4) 2^-24 most off, the exponential's argument and
    result included 2^-22 more; numerator and denominator are float sums of n weights: n 2^-24 off each.  weight_step: what a
    weight is rounded to before it multiplies its value.  Then one rounding to dt."""
    c = 2 * (260 * 2.0 ** -24 * most + 2.0 ** -22 + (n + 64) * 2.0 ** -24) + weight_step
    tol = half_step(dt) * want.abs() * 1.001 + c * mag + smallest_step(dt)
    far = (got.double().cpu() - want).abs() - tol
    assert torch.isfinite(got).all()
    assert far.max() <= 0, (float(far.max()), float((got.double().cpu() - want).abs().max()))


def sample_row(z, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(id, log-probability) of one row, in numpy's float64."""
    z = np.where(np.isnan(z), -np.inf, z).astype(np.float64)
    V, top = len(z), z.max()
    if top == -np.inf:
        return -1, -np.inf
    with np.errstate(invalid="ignore"):
        rel = np.where(z == top, 0.0, z - top)
    lse = np.log(np.exp(rel).sum())
    order = np.lexsort((np.arange(V), -z))
    if not temperature > 0:
        return int(order[0]), float(-lse)
    with np.errstate(over="ignore", invalid="ignore"):
        w = np.where(rel == 0, 1.0, np.where(z == -np.inf, 0.0, np.exp(rel / float(temperature))))
    n = top_k if 0 < top_k < V else V
    if top_p < 1:
        sums = np.cumsum(w[order[:n]])
        n = min(n, int((sums < float(top_p) * sums[-1]).sum()) + 1)
    if min_p > 0:
        n = min(n, max(1, int((w >= float(min_p)).sum())))
    kept = np.sort(order[:n])
    kept = kept[w[kept] > 0]
    sums = np.cumsum(w[kept])
    i = int((sums <= max(float(u), 0.0) * sums[-1]).sum())
    i = int(kept[min(i, len(kept) - 1)])
    return i, float(rel[i] - lse)
