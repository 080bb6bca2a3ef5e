"""GPU test of the largest calls of the rotation table and of the norm and rotation: what no launch takes is refused as such, before
anything is launched."""
import os
import sys

import pytest
import torch

import paper_2604_04335_amd as da

sys.path.insert(0, os.path.dirname(__file__))
from test_gpu_operators import ctx  # noqa: E402, F401

pytestmark = pytest.mark.gpu


def test_more_rows_than_a_launch_takes(ctx):
    """2^24 workgroups of 256 threads are 2^32 threads, one more than a launch takes.  32 rows a workgroup in each of these."""
    room = torch.full((4096,), 3.0, device="cuda")
    at = room.data_ptr()

    def code(call, *args):
        with pytest.raises(da.DitAttnError) as ei:
            call(ctx, *args)
        return ei.value.code

    for rows in (2 ** 29, 2 ** 30, 2 ** 34):
        assert code(da.dit_attn_rope_table, at, rows, da.RopeSpec([128]), at + 4096) == -11
        side = da.NormHeads(at, at + 4096, n_heads=1)
        assert code(da.dit_attn_qk_norm_rope, side, None, rows, 64, da.NORM_RMS, 1e-6) == -11
    torch.cuda.synchronize()
    assert bool((room == 3.0).all())
