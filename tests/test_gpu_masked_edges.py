"""GPU tests of masked attention where it can go wrong: values that are not finite among seen and unseen keys, and a distance bias
in runs of whole tiles, with and without document ids."""
import os
import sys

import numpy as np
import pytest
import torch

import paper_2604_04335_amd as da

sys.path.insert(0, os.path.dirname(__file__))
from gpu_util import to_dev  # noqa: E402
from test_gpu_operators import _bf16, _check_masked, _cu, _make, _mask, _rng, _run_masked, ctx  # noqa: E402, F401

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


@pytest.mark.parametrize("rows", [1, 40])
@pytest.mark.parametrize("D", [64, 128])
def test_values_that_are_not_finite_in_a_part_of_no_weight(ctx, D, rows):
    """Keys in several parts, and a bias that leaves those far away a probability of 0 in 32 bits: their values are seen all the same."""
    rng = _rng(D + rows)
    n, H = 5000, 2
    q, k, v = to_dev(_bf16(rng, rows, H, D)), to_dev(_bf16(rng, n, H, D)), to_dev(_bf16(rng, n, H, D))
    mask = da.AttnMask(slopes=torch.full((H,), 2.0, device="cuda"))
    clean, clean_lse = _run_masked(ctx, q, k, v, _cu([rows]), _cu([n]), D ** -0.5, mask)
    v[3, 0, 5] = float("nan")
    v[900, 1, 7] = float("nan")
    out, lse = _run_masked(ctx, q, k, v, _cu([rows]), _cu([n]), D ** -0.5, mask)
    want = torch.zeros((rows, H, D), dtype=torch.bool, device="cuda")
    want[:, 0, 5] = want[:, 1, 7] = True
    assert torch.equal(torch.isnan(out), want)
    assert torch.equal(out[~want].view(torch.int16), clean[~want].view(torch.int16)) and torch.equal(lse, clean_lse)


def test_an_unseen_value_costs_nothing(ctx):
    """A key of another document whose value is NaN, at every place of a tile: the call takes as long as for any other place, not a
    walk over all keys."""
    rng = _rng(4)
    lq, lk, H, D = 128, 8192, 64, 64
    q, k, v = to_dev(_bf16(rng, lq, H, D)), to_dev(_bf16(rng, lk, H, D)), to_dev(_bf16(rng, lk, H, D))
    out = torch.empty_like(q)
    q_doc = torch.zeros(lq, dtype=torch.int32, device="cuda")

    def time_of(place):
        ids = torch.zeros(lk, dtype=torch.int32, device="cuda")
        ids[place::64] = 1
        values = v.clone()
        values[place::64] = float("nan")
        mask = da.AttnMask(q_doc=q_doc, k_doc=ids)
        best = float("inf")
        for _ in range(4):
            start, end = torch.cuda.Event(True), torch.cuda.Event(True)
            start.record()
            da.dit_attn_masked_varlen_fwd(ctx, q, k, values, _cu([lq]), _cu([lk]), H, H, D, 0.125, mask, out)
            end.record()
            torch.cuda.synchronize()
            best = min(best, start.elapsed_time(end))
        assert bool(torch.isfinite(out.float()).all())
        return best

    usual = time_of(30)
    for place in (0, 31, 32, 63):
        assert time_of(place) < 3 * usual, place


@pytest.mark.parametrize("rows", [3, 200])
def test_ids_of_no_keys_and_of_no_rows(ctx, rows):
    """Empty tensors have no address: rows with ids against no keys at all, and keys with ids for no rows."""
    rng = _rng(rows)
    H, D = 2, 64
    q, none = to_dev(_bf16(rng, rows, H, D)), torch.empty((0, H, D), dtype=torch.bfloat16, device="cuda")
    ids, no_ids = torch.zeros(rows, dtype=torch.int32, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda")
    out, lse = _run_masked(ctx, q, none, none, _cu([rows]), _cu([0]), 0.1, da.AttnMask(q_doc=ids, k_doc=no_ids))
    assert not bool(out.any()) and bool((lse == float("-inf")).all())
    _run_masked(ctx, none, q, q, _cu([0]), _cu([rows]), 0.1, da.AttnMask(q_doc=no_ids, k_doc=ids))
    _run_masked(ctx, none, none, none, _cu([0]), None, 0.1, da.AttnMask(q_doc=no_ids, k_doc=no_ids))
    for mask in (da.AttnMask(k_doc=ids), da.AttnMask(q_doc=no_ids, k_doc=ids), da.AttnMask(q_doc=ids)):
        with pytest.raises((da.DitAttnError, ValueError)):
            _run_masked(ctx, q, q, q, _cu([rows]), None, 0.1, mask)


BIAS_CASES = [
    # q lens, k lens (None: the same), H, G, D, options: runs that begin and end at documents, behind the rows and before them
    ([1500], None, 2, 2, 64, dict(bias=True, docs=2, pad=101)),
    ([1500], None, 2, 1, 128, dict(bias=True, docs=2, pad=101)),
    ([1500], None, 2, 2, 128, dict(bias=True, docs=2, pad=0, causal=True)),
    ([1500], None, 2, 2, 64, dict(bias=True, docs=2, pad=64, causal=True, prefix=[700])),
    ([1300], None, 2, 2, 128, dict(bias=True)),                        # over 600 keys behind the first rows
    ([200, 900], [1200, 900], 2, 2, 128, dict(bias=True, docs=1, pad=5)),
    ([700, 130], [700, 2000], 2, 1, 64, dict(bias=True, docs=3, pad=0, shuffle=True)),
    ([3], [900], 4, 2, 128, dict(bias=True, docs=3, pad=50)),
    ([9], [2100], 2, 1, 64, dict(bias=True, docs=2, pad=0, causal=True)),
]


@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("i", range(len(BIAS_CASES)))
def test_bias_with_and_without_documents(ctx, i, sign):
    print(BIAS_CASES[i], flush=True)
    q, k, v, cu_q, cu_k, kw = _make(BIAS_CASES[i], 400 + i)
    kw["slopes"] = (sign * kw["slopes"]).astype(np.float32)
    scale = q.shape[2] ** -0.5
    out, lse = _run_masked(ctx, to_dev(q), to_dev(k), to_dev(v), cu_q, cu_k, scale, _mask(kw))
    _check_masked(out, lse, q, k, v, cu_q, cu_k, scale, **kw)
    plain, _ = _run_masked(ctx, to_dev(q), to_dev(k), to_dev(v), cu_q, cu_k, scale, _mask(kw), want_lse=False)
    assert torch.equal(plain.view(torch.int16), out.view(torch.int16))


@pytest.mark.parametrize("where", ["left", "right"])
@pytest.mark.parametrize("D", [64, 128])
def test_bias_where_the_keys_that_count_lie_far_away(ctx, D, where):
    """Keys that count at a distance of 2^19 and a bias there of 2^18: fp32 has steps of 2^-5 at that size, so a sum of products
    that begins with the bias is off by several per cent of a probability.  Relative to the largest bias of the row the scores
    that count are small, and the result is as near as without a bias.  In whole tiles, where no mask is looked at.
      left   rows at the end, a slope of -1/2 (the farthest keys count: the first ones)
      right  rows at the beginning of as many (without a document: they see nothing), keys of the rows' document far behind them"""
    rng = _rng(D)
    far, near, H = 2 ** 19, 4096, 1
    slope = 0.5
    scale = D ** -0.5
    live = 128  # a whole item: no row of it without a document
    if where == "left":
        lq, lk, sign, keys = live, far, -1.0, slice(0, near)
        ids = {}
    else:
        lq = lk = far + near
        sign, keys = 1.0, slice(far, far + near)
        q_doc, k_doc = torch.full((lq,), -1, dtype=torch.int32, device="cuda"), torch.full((lk,), -1, dtype=torch.int32, device="cuda")
        q_doc[:live] = 0
        k_doc[keys] = 0
        ids = dict(q_doc=q_doc, k_doc=k_doc)
    q, k, v = (torch.randn((n, H, D), device="cuda", generator=torch.Generator("cuda").manual_seed(D + n_)).to(torch.bfloat16)
               for n_, n in enumerate((lq, lk, lk)))
    slopes = torch.full((H,), sign * slope, device="cuda")
    out, lse = _run_masked(ctx, q, k, v, _cu([lq]), _cu([lk]), scale, da.AttnMask(slopes=slopes, **ids))
    # the keys that count, in 64 bits; others are under 2^-1000 of them
    kk, vv, qq = (x.double().cpu().numpy() for x in (k[keys, 0], v[keys, 0], q[:live, 0]))
    dist = np.abs(np.arange(live)[:, None] + (lk - lq) - np.arange(lk)[keys][None, :])
    s = qq @ kk.T * scale - sign * slope * dist
    m = s.max(1, keepdims=True)
    p = np.exp(s - m)
    want, spread = p @ vv / p.sum(1, keepdims=True), p @ np.abs(vv) / p.sum(1, keepdims=True)
    # half a step of the result; the probabilities' rounding and, a tenth of it, fp32 scores of up to 64
    bound = 2.0 ** -8 * np.abs(want) + 1.1 * 2.0 ** -8 * (spread + np.abs(want))
    got = out[:live, 0].double().cpu().numpy()
    assert np.all(np.abs(got - want) <= bound), float(np.max(np.abs(got - want) / bound))
    # the bias, the reference taken off and put on again, two products and the result: half a step of the largest each
    want_lse = m[:, 0] + np.log(p.sum(1))
    assert np.all(np.abs(lse[:live, 0].double().cpu().numpy() - want_lse) <= 8 * 2.0 ** -24 * np.abs(m[:, 0]) + 1e-5)
