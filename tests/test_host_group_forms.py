"""The form with 128 x 128 tiles and a shared contraction, at sizes that the GPU tests run.  No GPU needed."""
import pytest

from paper_2505_14742_amd import binding as q


@pytest.mark.parametrize("what,t,c_in,c_out,n", [("fwd", 1309, 8208, 1040, 1), ("fwd", 400, 4112, 4112, 4), ("dx", 959, 528, 4112, 1),
                                                 ("mx4_fwd", 1200, 16400, 528, 0), ("mx4_dx", 800, 784, 16400, 2)])
def test_medium_tiles_share_long_contractions(what, t, c_in, c_out, n):
    assert q.debug_group_form(what, t, c_in, c_out, n) == "128x128 parts"


def test_no_part_of_the_input_pass_is_empty():
    """The contraction's steps of 128 values are dealt to the parts of a 4-bit layer's down-projection in equal runs; the workspace, which holds t x r
    floats of every part, tells their number."""
    seen = set()
    for n_groups in (0, 3, 64):
        for t in (4, 64, 300, 1024, 2048, 8192):
            for k in range(256, 20000, 256):
                t_bytes = q.mx4_linear_workspace_bytes(t, k, k, n_groups, 16) - q.mx4_linear_workspace_bytes(t, k, k, n_groups, 0)
                parts, steps = t_bytes // (t * 64), k // 128
                assert t_bytes == parts * t * 64 and 1 <= parts <= 8
                per = -(-steps // parts)
                assert (parts - 1) * per < steps, (n_groups, t, k, parts)
                seen.add(parts)
    assert seen == set(range(1, 9))
