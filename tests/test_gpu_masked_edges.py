"""GPU tests of masked attention where it can go wrong: values that are not finite among the keys that a row sees."""
import os
import sys

import pytest
import torch

import paper_2604_04335_amd as da

sys.path.insert(0, os.path.dirname(__file__))
from gpu_util import to_dev  # noqa: E402
from test_gpu_operators import _bf16, _cu, _rng, _run_masked, ctx  # noqa: E402, F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("first", [0, 4])
@pytest.mark.parametrize("few", [True, False])
@pytest.mark.parametrize("D", [64, 128])
def test_values_of_two_keys_that_are_nan_in_turn(ctx, D, few, first):
    """Key a has NaN in four elements of every eight, its neighbour a + 1 in the other four: a row that sees both has NaN everywhere,
    one that sees a alone in a's elements.  Elements of d % 8 < 4 and keys of key % 8 < 4 are kept by one half of a wavefront, the
    others by the other one, and only one half holds keys that are not finite."""
    rng = _rng(D + first)
    lq, lk, H = (16, 320, 2) if few else (200, 320, 2)
    q, k, v = to_dev(_bf16(rng, lq, H, D)), to_dev(_bf16(rng, lk, H, D)), to_dev(_bf16(rng, lk, H, D))
    pos0 = lk - lq
    a = (pos0 + 12) // 8 * 8 + first  # a tile and a block begin at a multiple of 32
    mask = da.AttnMask(causal=True)
    clean, clean_lse = _run_masked(ctx, q, k, v, _cu([lq]), _cu([lk]), D ** -0.5, mask)
    mine = torch.arange(D, device="cuda") % 8 // 4 == first // 4
    v[a, :, mine] = float("nan")
    v[a + 1, :, ~mine] = float("nan")
    out, lse = _run_masked(ctx, q, k, v, _cu([lq]), _cu([lk]), D ** -0.5, mask)
    want = torch.zeros((lq, H, D), dtype=torch.bool, device="cuda")
    want[a - pos0:, :, mine] = True
    want[a + 1 - pos0:] = True
    assert 0 < a - pos0 < lq - 2
    assert torch.equal(torch.isnan(out), want)
    assert torch.equal(out[~want].view(torch.int16), clean[~want].view(torch.int16)) and torch.equal(lse, clean_lse)
