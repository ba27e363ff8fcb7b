"""Plain 64-bit numpy forms of the 4-bit microscaled layer and of the products grouped by expert, and the error bounds that the
kernels' fp32 sums are held to."""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def padded(k):
    return -(-k // 256) * 256


def quantize(x):
    """float array [rows x k] -> (codes [rows x kp / 2], scales [rows x kp / 32], values [rows x k] float64), by the definition:
    the exponent from the largest magnitude of a block, the code from the distances to the grid, ties to the even code."""
    x = np.asarray(x, dtype=np.float64)
    rows, k = x.shape
    kp = padded(k)
    b = np.zeros((rows, kp // 32, 32))
    b.reshape(rows, kp)[:, :k] = x
    top = np.abs(b).max(-1)
    bad = ~np.isfinite(top)
    e = np.floor(np.log2(np.where((top > 0) & ~bad, top, 1.0))).astype(np.int64)
    e = np.where(np.ldexp(1.0, e) > np.where(bad, np.inf, top), e - 1, e)                 # (log2 of a value just below a power of two)
    E = np.where(top > 0, np.clip(e - 2, -127, 127), -127)
    m = np.abs(b) * np.ldexp(1.0, -E)[..., None]
    dist = np.abs(np.where(bad[..., None], 0.0, m)[..., None] - GRID)
    best = dist.min(-1, keepdims=True)
    near = dist == best
    even = near & (np.arange(8) % 2 == 0)
    code = np.where(even.any(-1), even.argmax(-1), near.argmax(-1))
    sign = np.signbit(b)
    values = np.where(sign, -1.0, 1.0) * GRID[code] * np.ldexp(1.0, E)[..., None]
    values[bad] = np.nan
    nibble = (code | (sign << 3)).astype(np.uint8).reshape(rows, kp)
    return nibble[:, 0::2] | (nibble[:, 1::2] << 4), np.where(bad, 255, E + 127).astype(np.uint8), values.reshape(rows, kp)[:, :k]


def spans(offsets, t):
    """Row ranges of the groups, clamped as documented."""
    o = [min(max(int(v), 0), t) for v in offsets]
    return [(a, max(a, b)) for a, b in zip(o[:-1], o[1:])]


# fp32 sums of n products, `step` of them to a matrix instruction: a product passes at most `step` roundings inside its
# instruction, one for every later instruction, and a few more where parts of a sum are joined and scaled; each is at most 2^-23 of
# the sum of magnitudes (the hardware may truncate).
def sum_bound(n, step, magnitudes):
    return (step + n / step + 8) * 2.0 ** -23 * magnitudes


def bf16_bound(bound, ref):
    """... and rounded to bf16: half a step of the result, which may itself be off by the bound."""
    return bound * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(ref)


def low_rank(x, A, B, scale):
    """scale (x A) B with the bound of a kernel that sums x A in fp32 and keeps it as two bf16 values (relative error 2^-17, as 2^-16)."""
    T, mag = x @ A * scale, np.abs(x) @ np.abs(A) * abs(scale)
    bound = (sum_bound(x.shape[1], 16, mag) + 2.0 ** -16 * np.abs(T)) @ np.abs(B)
    return T @ B, bound + sum_bound(2 * A.shape[1], 16, np.abs(T) @ np.abs(B))
