"""Weight gradients on 256 x 256 tiles whose groups have many stages of 64 rows: lengths on both sides of four, five and six whole stages, where the loop
that fetches no zeros begins, and long ones, at widths that are and are not multiples of the tile."""
import pytest
import torch

from paper_2505_14742_amd import binding as q
from tests.test_gpu_grouped import DEV, _check, _offsets, _rand

pytestmark = pytest.mark.gpu
LENS = [[256, 255, 320, 319, 0, 385, 515, 700], [257, 321, 1, 384, 383, 64, 448, 902]]


@pytest.mark.parametrize("c_in,c_out", [(1680, 1808), (1792, 1792), (2064, 1552)])
@pytest.mark.parametrize("lens", LENS)
def test_weight_gradients_of_long_groups(lens, c_in, c_out):
    t = sum(lens) + 7
    assert q.debug_group_form("dw", t, c_in, c_out, len(lens)) == "256x256"
    X, G = _rand(t, c_in, seed=t), _rand(t, c_out, seed=t + 1, scale=0.02)
    for M in (X, G):
        M[:3] = M[-4:] = float("nan")                     # rows of no group
    _check("dw", X, G, _offsets(lens, 3), torch.full((len(lens), c_in, c_out), 7.0, device=DEV))
