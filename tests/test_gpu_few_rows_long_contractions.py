"""Few rows per group against long contractions: the kernel for plain weights requests sixteen units of 128 contraction bytes a trip (4096 4-bit or 1024
bf16 values); these take further trips, whole and partly filled, the adapter's operands being fetched on the first alone."""
import pytest
import torch

from paper_2505_14742_amd import binding as q
from tests.test_gpu_grouped import _check, _rand
from tests.test_gpu_mx4 import DEV, Layer, _offsets, _rows

pytestmark = pytest.mark.gpu
bf16, f32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("k,r,dtype", [(4112, 0, f32), (4112, 64, bf16), (8192, 16, f32), (8208, 48, f32), (8208, 0, bf16), (11008, 64, f32), (11008, 16, bf16)])
@pytest.mark.parametrize("gradient", [False, True])
@pytest.mark.parametrize("lens", [None, [1], [3, 0, 16, 11]])
def test_4bit_layer(lens, gradient, k, r, dtype):
    t, groups, n = (sum(lens) + 2 if lens else 5), len(lens or ()), 144
    c_in, c_out = (n, k) if gradient else (k, n)
    assert q.debug_group_form("mx4_dx" if gradient else "mx4_fwd", t, c_in, c_out, groups) == "few rows"
    L = Layer(groups, c_in, c_out, r, k + r)
    X = _rows(t, k, k)
    if lens:
        X[0] = X[-1] = float("nan")
    L.check(gradient, X, _offsets(lens, 1) if lens else None, torch.full((t, n), 3.0, dtype=dtype, device=DEV))


@pytest.mark.parametrize("dtype,accumulate", [(f32, False), (f32, True), (bf16, False)])
@pytest.mark.parametrize("k", [1024, 1040, 2064, 4112])
@pytest.mark.parametrize("lens", [[1], [14], [3, 0, 16, 11], [2] * 40])
def test_grouped_input_gradient(lens, k, dtype, accumulate):
    t, n = sum(lens) + 2, 144
    assert q.debug_group_form("dx", t, n, k, len(lens)) == "few rows"
    G = _rand(t, k, seed=k)
    G[0] = G[-1] = float("nan")
    _check("dx", G, _rand(len(lens), n, k, seed=2, scale=0.1), _offsets(lens, 1), torch.full((t, n), 3.0, dtype=dtype, device=DEV), accumulate=accumulate)
