"""Contractions shared by several workgroups of 128 x 128 tiles, whose sums a second launch joins: the forward's transposed weight, the input gradient and
the 4-bit product with its adapter, whose term is added once."""
import pytest
import torch

from paper_2505_14742_amd import binding as q
from tests.mx4_grid_layer import GridLayer, on_grid
from tests.test_gpu_grouped import DEV, _check, _offsets, _rand

pytestmark = pytest.mark.gpu
bf16, f32 = torch.bfloat16, torch.float32
FORM = "128x128 parts"


@pytest.mark.parametrize("dtype,accumulate", [(f32, False), (f32, True), (bf16, False)])
@pytest.mark.parametrize("op,lens,c_in,c_out", [("fwd", [1300], 8208, 1040), ("fwd", [700, 0, 520], 4112, 1552), ("fwd", [100, 31, 200, 60], 4112, 4112),
                                                ("dx", [950], 528, 4112), ("dx", [400, 517], 528, 4112)])
def test_grouped_products(op, lens, c_in, c_out, dtype, accumulate):
    t = sum(lens) + 9
    assert q.debug_group_form(op, t, c_in, c_out, len(lens)) == FORM
    k, n = (c_in, c_out) if op == "fwd" else (c_out, c_in)
    P = _rand(t, k, seed=t)
    P[:4] = P[-5:] = float("nan")
    _check(op, P, _rand(len(lens), c_in, c_out, seed=2, scale=0.1), _offsets(lens, 4), torch.full((t, n), 3.0, dtype=dtype, device=DEV),
           accumulate=accumulate)


@pytest.mark.parametrize("gradient,t,k,n,lens,r,dtype", [(False, 1200, 16400, 528, None, 16, f32), (True, 1250, 16400, 528, None, 64, bf16),
                                                         (False, 850, 16400, 784, None, 0, bf16), (False, 1150, 16400, 528, [600, 541], 48, f32),
                                                         (True, 800, 16400, 784, [333, 460], 32, f32)])
def test_4bit_products(gradient, t, k, n, lens, r, dtype):
    groups = len(lens or ())
    L = GridLayer(groups, k, n, r, gradient, k + n)
    assert q.debug_group_form("mx4_dx" if gradient else "mx4_fwd", t, *L.sizes(), groups) == FORM
    X = on_grid(t, k, t)
    if lens:
        X[:4] = X[-3:] = float("nan")
    L.check(X, _offsets(lens, 4) if lens else None, dtype)
