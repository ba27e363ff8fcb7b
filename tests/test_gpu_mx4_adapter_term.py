"""The adapter's term of the 4-bit layer keeps its inner product T = scale X A in all 24 bits of fp32, up to the largest values.

The layer's weight is zero here, so that the result is the adapter's term alone.  Every row of X selects one row of A with 1, one with 2^-8
and one with 2^-16, whose entries are whole numbers of eight bits: T has exactly 24 significant bits.  Every column of B has one entry, a
power of two.  Products and sums are then exact in fp32; the tolerance still grants eight roundings of 2^-23 (three sums in T, three in the
product, one scaling, one join).  T rounded to 16 bits would be off by up to 2^-17."""
import numpy as np
import pytest
import torch

from paper_2505_14742_amd import binding as q

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
bf16 = torch.bfloat16


def _run(gradient, t, k, n, r, lens, X, first, second, scale):
    """X [t x k], first [groups x k x r], second [groups x r x n], all float64 numpy: the term through the layer with a zero weight."""
    groups = len(lens) if lens else 0
    e = max(1, groups)
    c_in, c_out = (n, k) if gradient else (k, n)
    kp = q.mx4_padded(k)
    codes = torch.zeros(e * n, kp // 2, dtype=torch.uint8, device=DEV)
    scales = torch.full((e * n, kp // 32), 127, dtype=torch.uint8, device=DEV)
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(bf16).to(DEV)
    # the gradient's first factor is B^T, its second A^T
    A, B = (dev(second.transpose(0, 2, 1)), dev(first.transpose(0, 2, 1))) if gradient else (dev(first), dev(second))
    off = torch.tensor([0] + list(lens), dtype=torch.int64).cumsum(0).to(DEV) if groups else None
    ws = torch.empty(q.mx4_linear_workspace_bytes(t, c_in, c_out, groups, r), dtype=torch.int8, device=DEV)
    out = torch.full((t, n), 3.0, device=DEV)
    (q.mx4_linear_bwd_dx if gradient else q.mx4_linear_fwd)(dev(X), off, codes, scales, c_in, c_out, A, B, r, scale, out, ws)
    return out.double().cpu().numpy()


def _factors(g, e, k, n, r):
    first = np.where(np.arange(k)[None, :, None] % 3 == 0, g.integers(128, 256, (e, k, r)),
                     np.where(np.arange(k)[None, :, None] % 3 == 1, g.integers(0, 256, (e, k, r)), g.integers(0, 128, (e, k, r)) * 2 + 1))
    first = first * g.choice([-1.0, 1.0], (e, 1, r))
    second = np.zeros((e, r, n))
    second[:, np.arange(n) % r, np.arange(n)] = g.choice([-0.5, 0.25, 1.0, 4.0], (e, n))
    return first.astype(np.float64), second


def _spans(t, lens):
    ends = np.cumsum([0] + list(lens)) if lens else [0, t]
    return list(zip(ends[:-1], ends[1:]))


@pytest.mark.parametrize("gradient", [False, True])
@pytest.mark.parametrize("form,t,k,n,r,lens", [
    ("few rows", 1, 1040, 80, 16, None), ("few rows", 11, 528, 208, 64, [3, 0, 8]), ("64x64", 100, 272, 144, 48, None), ("64x64", 130, 400, 80, 32, [50, 80]),
    ("64x64 parts", 100, 5136, 208, 16, None), ("128x128", 1100, 2064, 2064, 64, None), ("128x128", 2000, 528, 2064, 32, [400, 377, 423, 0, 800]),
    ("256x256", 4099, 80, 4112, 48, None), ("256x256", 4300, 144, 4112, 16, [2100, 0, 2200])])
def test_the_inner_product_keeps_24_bits(gradient, form, t, k, n, r, lens):
    c_in, c_out = (n, k) if gradient else (k, n)
    assert q.debug_group_form("mx4_dx" if gradient else "mx4_fwd", t, c_in, c_out, len(lens or ())) == form
    g = np.random.default_rng(t + k)
    first, second = _factors(g, len(lens or [t]), k, n, r)
    X = np.zeros((t, k))
    for j in range(3):
        X[np.arange(t), j + 3 * g.integers(0, (k - j - 1) // 3 + 1, t)] = 2.0 ** (-8 * j)
    got = _run(gradient, t, k, n, r, lens, X, first, second, 0.5)
    want = np.full((t, n), 3.0)
    for e, (a, b) in enumerate(_spans(t, lens)):
        want[a:b] = 0.5 * X[a:b] @ first[e] @ second[e]
    worst = np.abs(got - want) - 8 * 2.0 ** -23 * np.abs(want)
    assert worst.max() <= 0, "worst excess %.3e at %s" % (worst.max(), np.unravel_index(worst.argmax(), worst.shape))


@pytest.mark.parametrize("gradient", [False, True])
@pytest.mark.parametrize("form,t,k,n,r", [("few rows", 3, 528, 208, 16), ("64x64", 100, 272, 144, 64), ("128x128", 1100, 144, 2064, 32), ("256x256", 4099, 80, 4112, 16)])
def test_the_largest_inner_products(gradient, form, t, k, n, r):
    """The largest fp32 value, which lies past what bf16 rounds to a finite value, and sums that overflow: infinite with the sign of the
    second factor's entry, as in fp32, in their rows only."""
    c_in, c_out = (n, k) if gradient else (k, n)
    assert q.debug_group_form("mx4_dx" if gradient else "mx4_fwd", t, c_in, c_out, 0) == form
    first, second = np.zeros((1, k, r)), np.zeros((1, r, n))
    first[0, :, 0] = 1.0
    first[0, 5, 0] = 4.0
    second[0, 0] = np.where(np.arange(n) % 3 == 0, -1.0, 2.0 ** -20)
    X = np.zeros((t, k))
    X[0, [1, 40, 77]] = 255 * np.array([2.0 ** 120, 2.0 ** 112, 2.0 ** 104])              # (2^24 - 1) 2^104
    X[1:, 5] = 1.0
    X[2 % t, 5] = 2.0 ** 127 if t > 2 else 1.0
    got = _run(gradient, t, k, n, r, None, X, first, second, 1.0)
    T = X @ first[0, :, 0]
    with np.errstate(over="ignore"):
        T = T.astype(np.float32).astype(np.float64)
    assert np.isinf(T).sum() == 1 and T[0] == float(np.finfo(np.float32).max)
    assert np.array_equal(got, np.outer(T, second[0, 0]))
