"""The form with 128 x 128 tiles and a shared contraction, at sizes that the GPU tests run.  No GPU needed."""
import pytest

from paper_2505_14742_amd import binding as q


@pytest.mark.parametrize("what,t,c_in,c_out,n", [("fwd", 1309, 8208, 1040, 1), ("fwd", 400, 4112, 4112, 4), ("dx", 959, 528, 4112, 1),
                                                 ("mx4_fwd", 1200, 16400, 528, 0), ("mx4_dx", 800, 784, 16400, 2)])
def test_medium_tiles_share_long_contractions(what, t, c_in, c_out, n):
    assert q.debug_group_form(what, t, c_in, c_out, n) == "128x128 parts"
