"""4-bit products whose contraction has many stages of 256 values: every tile, with the stage counts on all sides of the loop that requests the scales
of four stages at a time (eight and more stages, each remainder of four), dense and by group, with and without an adapter."""
import itertools

import pytest
import torch

from paper_2505_14742_amd import binding as q
from tests.mx4_grid_layer import DEV, GridLayer, on_grid

pytestmark = pytest.mark.gpu
bf16, f32 = torch.bfloat16, torch.float32

# (form, rows, columns of the result, rows of the groups): 256 x 256 tiles with some left over, which are dealt out in quarters
SHAPES = [("64x64", 1029, 1040, None), ("64x64", 600, 1040, [50, 0, 61, 1, 64, 65, 127, 20, 0, 90, 33, 80]), ("128x128", 1100, 2064, None),
          ("128x128", 2000, 2064, [400, 129, 0, 711, 750]), ("256x256", 4099, 4112, None), ("256x256", 4300, 4112, [2100, 0, 2190])]
CONTRACTIONS = [2048, 2800, 2832, 3328, 4112]           # 8, 11, 12, 13 and 17 stages; the second, third and last end inside one
RANKS, DTYPES, DIRECTIONS = [0, 16, 48, 64, 32], [f32, bf16], [False, True]
CASES = [(shape, k, RANKS[(i + j) % 5], DTYPES[(i + j) % 2], DIRECTIONS[(i // 2 + j) % 2])
         for (i, shape), (j, k) in itertools.product(enumerate(SHAPES), enumerate(CONTRACTIONS))]


@pytest.mark.parametrize("shape,k,r,dtype,gradient", CASES)
def test_many_stages(shape, k, r, dtype, gradient):
    form, t, n, lens = shape
    groups = len(lens or ())
    L = GridLayer(groups, k, n, r, gradient, t + k)
    assert q.debug_group_form("mx4_dx" if gradient else "mx4_fwd", t, *L.sizes(), groups) == form
    X = on_grid(t, k, t)
    offsets = None
    if lens:
        offsets = torch.tensor([4] + lens, dtype=torch.int64).cumsum(0).to(DEV)
        X[:4] = float("nan")                             # rows of no group
    L.check(X, offsets, dtype)
