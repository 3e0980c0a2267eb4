"""Plain 64-bit forms of the norm and the optimizer step, and code grids, for the tests."""
import numpy as np

E4M3 = np.array([(e % 8) * 2.0 ** -9 if e < 8 else (1 + (e % 8) / 8) * 2.0 ** (e // 8 - 7) for e in range(127)])
E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6.0])


def nearest(t, grid):
    """Grid value nearest to t, ties to the even code, saturating; the sign of t kept."""
    a = np.minimum(np.abs(t), grid[-1])
    hi = np.clip(np.searchsorted(grid, a), 1, len(grid) - 1)
    up, down = grid[hi] - a, a - grid[hi - 1]
    pick = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, hi - 1)
    return np.copysign(grid[pick], t)


def stochastic(t, u, grid):
    """The neighbour above iff (a - lo)/(hi - lo) > (u + 1/2)/2^16."""
    a = np.minimum(np.abs(t), grid[-1])
    hi = np.clip(np.searchsorted(grid, a, side="right"), 1, len(grid) - 1)
    lo = hi - 1
    return np.copysign(np.where((a - grid[lo]) / (grid[hi] - grid[lo]) > (u + 0.5) / 65536, grid[hi], grid[lo]), t)


def between(code, t, slack, grid, u=None):
    """Whether each code value is what some t' with |t' - t| <= slack is rounded to (rounding is monotone in t)."""
    def rounded(v):
        return nearest(v, grid) if u is None else stochastic(v, u, grid)

    lo, hi = rounded(t - slack), rounded(t + slack)
    return (code >= np.minimum(lo, hi)) & (code <= np.maximum(lo, hi))


def code_values(codes, fmt_fp8, lines, cols):
    """uint8 codes as stored [lines][cols] -> the numbers they stand for."""
    c = np.asarray(codes)
    if not fmt_fp8:
        c = c[:lines * cols // 2].reshape(lines, cols // 2)
        c = np.stack([c & 15, c >> 4], -1).reshape(lines, cols)
        return np.where(c & 8, -1.0, 1.0) * E2M1[c & 7]
    c = c[:lines * cols].reshape(lines, cols)
    assert not np.any((c & 127) == 127)
    return np.where(c & 128, -1.0, 1.0) * E4M3[c & 127]


def bf16(x):
    """64-bit values rounded once to bf16 (nearest, ties to even), as 64-bit values; normal range."""
    x = np.asarray(x, dtype=np.float64)
    m, e = np.frexp(x)
    return np.ldexp(np.rint(m * 256) / 256, e)      # rint: ties to even


def norm(x, residual, gain, eps):
    h = x if residual is None else bf16(x + residual)
    rstd = 1 / np.sqrt(np.mean(h * h, axis=1) + eps)
    return h, rstd, h * rstd[:, None] * gain


def norm_bwd(dy, h, gain, rstd, dresidual):
    g, u = dy * gain, h * rstd[:, None]
    dx = rstd[:, None] * (g - u * np.mean(g * u, axis=1, keepdims=True))
    return dx + (0 if dresidual is None else dresidual), (dy * u).sum(0)


def philox(n, tensor, word3, seed):
    """Four output words for counters (q, q >> 32, tensor, word3), q = 0 .. n - 1."""
    m = np.uint64(0xFFFFFFFF)
    q = np.arange(n, dtype=np.uint64)
    c = [q & m, q >> np.uint64(32), np.full(n, tensor, np.uint64), np.full(n, word3 & 0xFFFFFFFF, np.uint64)]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & m, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & m]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def uniforms(n, words):
    w = np.stack([words[0] & np.uint64(0xFFFF), words[0] >> np.uint64(16), words[1] & np.uint64(0xFFFF), words[1] >> np.uint64(16)], 1)
    return w.reshape(-1)[:n].astype(np.float64)


def adamw(p, g, m, v, lr, b1, b2, eps, step, decay, grad_scale=1.0):
    g = g * grad_scale
    m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    update = lr / (1 - b1 ** step) * m / (np.sqrt(v) / np.sqrt(1 - b2 ** step) + eps)
    return p * (1 - lr * decay) - update, m, v, update


def block_scale(x):
    """Scale of each 128 elements of x."""
    whole = np.zeros(-(-len(x) // 128) * 128)
    whole[:len(x)] = np.abs(x)
    most = whole.reshape(-1, 128).max(1)
    with np.errstate(divide="ignore"):
        return np.where(most > 0, np.minimum(448.0 / np.where(most > 0, most, 1), np.finfo(np.float32).max), 1.0)
