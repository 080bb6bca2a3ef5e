"""GPU parity of the rotation table, the norm and rotation of queries and keys, and masked attention, against the fp64 oracle.

Tolerances.  table: fp32, the angle's fp32 rounding, the polynomial's last two roundings and the product with the magnitude, half
a step (2^-24 relative) each.  norm: bf16, half a step (2^-8) of the result; before it fp32 sums of at most 128 terms, whose
roundings stay under 2^-18 of the pair's values and of what a mean takes off.  attention: half a step of the result, and the
probabilities' rounding to bf16, each off by at most 2^-8, which moves a mean of v by at most 2^-8 times the mean of |v - out|,
that is of |v| + |out|; fp32 scores move it by under a tenth of that.  lse: fp32 scores, some 2^-19 of the largest, and sums of a
row's probabilities in turn, half a step for every term of a half-wave.
"""
import os
import sys

import numpy as np
import pytest
import torch

import paper_2604_04335_amd as da
from dit_workloads import f32_to_bf16_bits
from oracle import operators_oracle as orc

sys.path.insert(0, os.path.dirname(__file__))
from gpu_util import to_bits, to_dev, widen  # noqa: E402

pytestmark = pytest.mark.gpu

GUARD = 64
SENTINEL = 0x7FC1


@pytest.fixture(scope="module")
def ctx():
    h = da.dit_attn_create(0)
    yield h
    torch.cuda.synchronize()
    da.dit_attn_destroy(h)


def _rng(seed):
    return np.random.Generator(np.random.PCG64(seed))


def _bf16(rng, *shape, scale=1.0):
    return f32_to_bf16_bits((rng.standard_normal(shape, dtype=np.float32) * scale))


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _guarded(rows, heads, dim):
    """A bf16 output [rows, heads, dim] between guard rows, and the check of those."""
    buf = torch.full((rows + 2 * GUARD, heads, dim), SENTINEL, dtype=torch.int16, device="cuda")

    def check():
        assert bool((buf[:GUARD] == SENTINEL).all()) and bool((buf[GUARD + rows:] == SENTINEL).all()), "guard rows were written"

    return buf[GUARD:GUARD + rows].view(torch.bfloat16), check


# ---------------------------------------------------------------- table

SCALINGS = {"plain": da.ROPE_PLAIN, "linear": da.ROPE_LINEAR, "base": da.ROPE_BASE, "bands": da.ROPE_BANDS}


@pytest.mark.parametrize("dims,scaling,rows,magnitude", [
    ([128], "plain", 1, 1.0), ([16, 56, 56], "linear", 300, 1.0), ([44, 42, 42], "bands", 1000, 1.0 + 0.1 * np.log(4.0)),
    ([2], "base", 777, 1.0), ([2, 6, 4, 10], "base", 33, -2.5), ([30, 8, 16, 24], "bands", 129, 1.0), ([62, 2], "plain", 5, 1.0),
])
def test_table(ctx, dims, scaling, rows, magnitude):
    rng = _rng(rows)
    A = len(dims)
    pos = rng.integers(-5000, 100000, (rows, A)).astype(np.int32)
    far = np.array([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 2 ** 30 + 1, 8191, 123456789], dtype=np.int32)
    pos[:min(rows, 8)] = far[:min(rows, 8), None]
    theta, factor, length = [10000.0, 256.0, 10000.0, 500000.0][:A], [4.0, 1.0, 2.5, 16.0][:A], [4096.0, 64.0, 128.0, 8192.0][:A]
    spec = da.RopeSpec(dims, theta, SCALINGS[scaling], factor, length, low=1.0, high=32.0, magnitude=magnitude)
    P = spec.rot_dim // 2
    buf = torch.full((rows * P * 2 + 128,), 7.0, device="cuda")
    table = buf[64:64 + rows * P * 2]
    da.dit_attn_rope_table(ctx, torch.from_numpy(pos).cuda(), rows, spec, table, _stream())
    torch.cuda.synchronize()
    assert bool((buf[:64] == 7.0).all()) and bool((buf[64 + rows * P * 2:] == 7.0).all())
    f, axis = orc.frequencies(dims, theta, scaling, factor, length)
    want = orc.rope_table(pos, f, axis, magnitude)
    # a frequency that differs in its last bit of 53 turns a position of 2^31 by 2^-22 of a radian
    slack = np.abs(pos[:, axis].astype(np.float64))[:, :, None] * (f * 2.0 ** -52)[None, :, None]
    assert np.all(np.abs(table.view(rows, P, 2).cpu().numpy() - want) <= abs(magnitude) * (4 * 2.0 ** -24 + slack))


# ---------------------------------------------------------------- norm and rotation

def _norm_bound(x, y, normed, bias, norm, weight, eps):
    """Half a bf16 step of the result, 2^-18 of what it was made of."""
    D = x.shape[2]
    made = np.abs(normed).max(2, keepdims=True)
    if norm == "layer":
        c = x - x.mean(2, keepdims=True)
        r = 1.0 / np.sqrt((c * c).mean(2, keepdims=True) + eps)
        made = made + np.abs(x).max(2, keepdims=True) * r * (1.0 if weight is None else np.abs(weight).max())
    if bias is not None:
        made = made + np.abs(bias).max()
    assert D <= 128
    return 2.0 ** -8 * np.abs(y) + 2.0 ** -18 * made * 2.0


@pytest.mark.parametrize("n,H,G,D,norm,half,rot,affine,fused", [
    (1, 24, 8, 128, "rms", True, 128, "weight", False),
    (1, 1, 1, 64, "rms", False, 64, "none", False),
    (17, 3, 1, 128, "rms", False, 128, "both", False),
    (130, 5, 2, 128, "layer", True, 96, "both", True),
    (257, 10, 10, 64, "layer", False, 24, "weight", True),
    (300, 4, 4, 64, "none", True, 64, "none", False),
    (41, 7, 7, 128, "none", False, 40, "none", True),
    (33, 9, 3, 128, "rms", True, 8, "both", False),
    (129, 2, 1, 64, "rms", True, 0, "weight", False),
    (1000, 24, 24, 128, "rms", True, 64, "weight", True),
])
def test_norm_rope(ctx, n, H, G, D, norm, half, rot, affine, fused):
    rng = _rng(n * 7 + H)
    width = (H + 2 * G) * D
    bits = _bf16(rng, n, width, scale=3.0) + np.uint16(0)
    qkv = to_dev(bits)
    kinds = {"none": da.NORM_NONE, "rms": da.NORM_RMS, "layer": da.NORM_LAYER}
    angle = rng.standard_normal((n, rot // 2)) * 100.0
    table = np.stack([np.cos(angle), np.sin(angle)], 2).astype(np.float32)
    tab = torch.from_numpy(table).cuda() if rot else None
    sides, checks = [], []
    for a, heads in ((0, H), (H * D, G)):
        w = (1 + 0.2 * rng.standard_normal(D)).astype(np.float32) if affine != "none" else None
        b = (0.3 * rng.standard_normal(D)).astype(np.float32) if affine == "both" else None
        x = qkv[:, a:a + heads * D].unflatten(1, (heads, D))
        if not fused:
            x = x.contiguous()
        out, check = _guarded(n, heads, D)
        sides.append((x, out, w, b, heads, a))
        checks.append(check)
    args = [da.NormHeads(x, out, *(None if z is None else torch.from_numpy(z).cuda() for z in (w, b))) for x, out, w, b, _, _ in sides]
    da.dit_attn_qk_norm_rope(ctx, args[0], args[1], n, D, kinds[norm], 1e-6, tab, rot, da.ROPE_HALF if half else da.ROPE_INTERLEAVED, _stream())
    torch.cuda.synchronize()
    first = []
    for (x, out, w, b, heads, a), check in zip(sides, checks):
        check()
        x64 = widen(bits[:, a:a + heads * D]).reshape(n, heads, D)
        y, normed = orc.norm_rope(x64, norm, 1e-6, w, b, table.astype(np.float64), rot, half)
        got = widen(to_bits(out))
        assert np.all(np.abs(got - y) <= _norm_bound(x64, y, normed, b, norm, w, 1e-6))
        first.append(to_bits(out))
    # one side alone, and in place in the fused rows, whose values stay
    for i, (x, out, w, b, heads, a) in enumerate(sides):
        view = qkv[:, a:a + heads * D].unflatten(1, (heads, D))
        side = da.NormHeads(view, view, *(None if z is None else torch.from_numpy(z).cuda() for z in (w, b)))
        pair = (side, None) if i == 0 else (None, side)
        da.dit_attn_qk_norm_rope(ctx, *pair, n, D, kinds[norm], 1e-6, tab, rot, da.ROPE_HALF if half else da.ROPE_INTERLEAVED, _stream())
        assert np.array_equal(to_bits(view), first[i])
    assert np.array_equal(to_bits(qkv[:, (H + G) * D:]), bits[:, (H + G) * D:])


@pytest.mark.parametrize("D,rot,half,norm", [(128, 128, True, da.NORM_RMS), (128, 40, True, da.NORM_LAYER), (64, 64, False, da.NORM_RMS),
                                             (64, 48, True, da.NORM_NONE)])
@pytest.mark.parametrize("rows", [7001, 30011])
def test_large_calls_give_the_bits_of_small_ones(ctx, rows, D, rot, half, norm):
    """Sizes with streaming loads (over 64 MB) and with streaming stores too (over 160 MB), out of place and in place."""
    H, G = (24, 8) if D == 128 else (48, 16)
    gen = torch.Generator(device="cuda").manual_seed(rows + rot)
    q, k = (torch.randn((rows, h, D), device="cuda", generator=gen).to(torch.bfloat16) for h in (H, G))
    angle = torch.randn((rows, rot // 2), device="cuda", generator=gen) * 100
    table = torch.stack([angle.cos(), angle.sin()], 2)
    w = torch.randn(D, device="cuda", generator=gen) if norm != da.NORM_NONE else None
    layout = da.ROPE_HALF if half else da.ROPE_INTERLEAVED

    def call(a, b, qo, ko):
        da.dit_attn_qk_norm_rope(ctx, da.NormHeads(q[a:b], qo[a:b], w, w), da.NormHeads(k[a:b], ko[a:b], w, w), b - a, D, norm, 1e-6,
                                 table[a:b], rot, layout, _stream())

    small, large = [[torch.empty_like(q), torch.empty_like(k)] for _ in range(2)]
    for a in range(0, rows, 1000):
        call(a, min(rows, a + 1000), *small)
    call(0, rows, *large)
    for x, y in zip(small, large):
        assert torch.equal(x.view(torch.int16), y.view(torch.int16))
    call(0, rows, q, k)
    for x, y in zip(small, (q, k)):
        assert torch.equal(x.view(torch.int16), y.view(torch.int16))


def test_norm_of_zeros_and_of_rows_with_infinities(ctx):
    """A row of zeros stays zero (with eps), and rows that are not finite do not reach the others."""
    x = torch.ones((64, 2, 128), dtype=torch.bfloat16, device="cuda")
    x[3] = 0.0
    x[5, 0, 7] = float("inf")
    x[9, 1, 100] = float("nan")
    out = torch.empty_like(x)
    da.dit_attn_qk_norm_rope(ctx, da.NormHeads(x, out), None, 64, 128, da.NORM_RMS, 1e-6, None, 0, da.ROPE_HALF, _stream())
    bad = ~torch.isfinite(out.float()).all(2).cpu()
    want = torch.zeros((64, 2), dtype=torch.bool)
    want[5, 0] = want[9, 1] = True
    assert torch.equal(bad, want) and not bool(out[3].any())
    assert bool((out[0] == 1.0).all())


# ---------------------------------------------------------------- masked attention

def _cu(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


def _run_masked(ctx, q, k, v, cu_q, cu_k, scale, mask, want_lse=True, stream=None):
    rows, H, D = q.shape
    out, check = _guarded(rows, H, D)
    lse = torch.full((rows + 2, H), 123.0, device="cuda")
    da.dit_attn_masked_varlen_fwd(ctx, q, k, v, cu_q, cu_k, H, k.shape[1], D, scale, mask, out, lse[1:1 + rows] if want_lse else None,
                                  _stream() if stream is None else stream)
    torch.cuda.synchronize()
    check()
    assert bool((lse[0] == 123.0).all()) and bool((lse[-1] == 123.0).all())
    return out, lse[1:1 + rows]


def _check_masked(out, lse, q, k, v, cu_q, cu_k, scale, what="", **kw):
    """out, lse against the oracle on the same bits (q, k, v: uint16 arrays)."""
    want, wlse, spread, top = orc.masked_attention(widen(q), widen(k), widen(v), cu_q, cu_k, scale, **kw)
    got = widen(to_bits(out))
    assert np.all(np.isfinite(got)), what
    drift = 1.0 + 2.0 ** -14 * top[:, :, None]  # fp32 scores with a bias are off by half a step of the bias
    bound = 2.0 ** -8 * np.abs(want) + 1.1 * 2.0 ** -8 * drift * (spread + np.abs(want)) + 1e-30
    assert np.all(np.abs(got - want) <= bound), (what, float(np.max(np.abs(got - want) / bound)))
    if lse is not None:
        l = lse.cpu().numpy().astype(np.float64)
        keys = int(np.max(np.diff(cu_k))) if len(cu_k) > 1 else 0
        dead = np.isneginf(wlse)
        assert np.array_equal(np.isneginf(l), dead), what
        tol = (keys / 2 + 32) * 2.0 ** -24 + 2.0 ** -19 * (1.0 + top)
        assert np.all(np.abs(l[~dead] - wlse[~dead]) <= tol[~dead]), what
        assert not got[dead].any(), what


def _docs(rng, lens, n_docs, pad, shuffle=False):
    out = []
    for n in lens:
        ids = np.full(n, -1, np.int32)
        live = max(0, n - pad)
        ids[:live] = rng.integers(0, n_docs, live) if shuffle else np.arange(live) * n_docs // max(live, 1)
        out.append(ids)
    return np.concatenate(out) if out else np.zeros(0, np.int32)


CASES = [
    # q lens, k lens (None: the same), H, G, D, options
    ([1], [1], 1, 1, 64, dict(causal=True)),
    ([1], [63], 2, 1, 128, dict(causal=True)),
    ([1, 1, 1], [64, 65, 200], 6, 2, 64, dict(causal=True)),
    ([1, 1], [1000, 3], 24, 8, 128, dict(causal=True, cap=20.0)),
    ([1], [5000], 8, 1, 64, dict(bias=True)),
    ([4, 2], [300, 7], 8, 2, 128, dict(causal=True, bias=True)),
    ([16], [31], 2, 1, 64, dict(causal=True, prefix=[20])),
    ([5, 32], [2, 9], 1, 1, 128, dict(causal=True)),                      # rows before their first key see nothing
    ([7, 0, 3], [130, 4, 0], 2, 2, 64, dict()),                           # no rows; no keys
    ([12], [700], 2, 1, 128, dict(docs=3, pad=9)),
    ([33], None, 1, 1, 128, dict(causal=True)),
    ([127, 128, 129, 1, 0], None, 3, 3, 64, dict(causal=True, prefix=[0, 50, 500, 3, 9])),
    ([300], [1], 2, 1, 128, dict(causal=True, prefix=[1])),
    ([300], [40], 4, 2, 64, dict(cap=5.0)),
    ([200, 500], [500, 200], 2, 2, 128, dict(causal=True, bias=True)),
    ([257], None, 4, 4, 128, dict(cap=30.0, causal=True)),
    ([513, 70], None, 2, 1, 64, dict(docs=4, pad=33)),
    ([400, 64, 65], None, 2, 2, 128, dict(docs=7, pad=0, shuffle=True, causal=True)),
    ([640], None, 3, 3, 64, dict(docs=2, pad=639)),                       # all but one row see nothing
    ([129, 500], None, 2, 2, 128, dict(docs=3, pad=64, cap=10.0, bias=True, causal=True, prefix=[7, 300])),
    ([300], [3000], 2, 2, 128, dict(bias=True, cap=50.0)),                # split keys of the 128-row items
    ([130], [4100], 4, 2, 64, dict(causal=True, docs=5, pad=100)),
    ([40], [2500], 1, 1, 128, dict()),
    ([1000], None, 8, 8, 128, dict(causal=True)),
    ([1100], None, 8, 2, 64, dict(bias=True)),
    # few rows and others in one pack: two kernels, both of which split their keys, and one kernel
    ([1, 300, 2, 0, 40], [3000, 300, 5000, 10, 1500], 2, 1, 128, dict(causal=True, docs=2, pad=20, prefix=[0, 40, 10, 0, 9])),
    ([3, 1, 500], [900, 4000, 2500], 3, 1, 64, dict(cap=20.0, bias=True)),
    ([20, 200], [20, 200], 2, 2, 128, dict(causal=True)),
]


def _make(case, seed):
    q_lens, k_lens, H, G, D, opt = case
    k_lens = q_lens if k_lens is None else k_lens
    rng = _rng(seed)
    q, k, v = _bf16(rng, sum(q_lens), H, D), _bf16(rng, sum(k_lens), G, D), _bf16(rng, sum(k_lens), G, D)
    kw = dict(causal=opt.get("causal", False), prefix=opt.get("prefix"), cap=opt.get("cap", 0.0))
    if opt.get("bias"):
        kw["slopes"] = (2.0 ** (-8.0 * np.arange(1, H + 1) / H)).astype(np.float32)
    if opt.get("docs"):
        kw["k_doc"] = _docs(rng, k_lens, opt["docs"], opt["pad"], opt.get("shuffle", False))
        cu = _cu(k_lens)
        kw["q_doc"] = np.concatenate([kw["k_doc"][cu[i + 1] - n:cu[i + 1]] for i, n in enumerate(q_lens)])
    return q, k, v, _cu(q_lens), _cu(k_lens), kw


def _mask(kw):
    dev = {n: None if kw.get(n) is None else torch.from_numpy(kw[n]).cuda() for n in ("slopes", "q_doc", "k_doc")}
    return da.AttnMask(causal=kw["causal"], prefix=kw["prefix"], softcap=kw["cap"], **dev)


@pytest.mark.parametrize("i", range(len(CASES)))
def test_masked(ctx, i):
    print(CASES[i], flush=True)
    q, k, v, cu_q, cu_k, kw = _make(CASES[i], 100 + i)
    D = q.shape[2]
    scale = D ** -0.5
    dq, dk, dv, mask = to_dev(q), to_dev(k), to_dev(v), _mask(kw)
    out, lse = _run_masked(ctx, dq, dk, dv, cu_q, cu_k, scale, mask)
    _check_masked(out, lse, q, k, v, cu_q, cu_k, scale, **kw)
    plain, _ = _run_masked(ctx, dq, dk, dv, cu_q, cu_k, scale, mask, want_lse=False)
    again, lse2 = _run_masked(ctx, dq, dk, dv, cu_q, cu_k, scale, mask)
    assert torch.equal(again.view(torch.int16), out.view(torch.int16)) and torch.equal(lse2, lse)
    assert torch.equal(plain.view(torch.int16), out.view(torch.int16))


@pytest.mark.parametrize("cap", [1e-38, 1e-20, 1e20])
def test_masked_extreme_caps(ctx, cap):
    q, k, v, cu_q, cu_k, kw = _make(CASES[13], 300)
    kw["cap"] = cap
    q[0] = 0
    out, lse = _run_masked(ctx, to_dev(q), to_dev(k), to_dev(v), cu_q, cu_k, 0.125, _mask(kw))
    _check_masked(out, lse, q, k, v, cu_q, cu_k, 0.125, **dict(kw, cap=float(np.float32(cap))))


@pytest.mark.parametrize("scale", [0.0, -0.3, 2.0])
@pytest.mark.parametrize("i", [2, 5, 13, 15, 19])
def test_masked_scales(ctx, i, scale):
    q, k, v, cu_q, cu_k, kw = _make(CASES[i], 200 + i)
    out, lse = _run_masked(ctx, to_dev(q), to_dev(k), to_dev(v), cu_q, cu_k, scale, _mask(kw))
    # scores of a scale of 2 are sums of 128 products of up to 16: fp32 rounding of the largest moves them by 2^-14
    _check_masked(out, lse, q, k, v, cu_q, cu_k, scale, **kw)


@pytest.mark.parametrize("cap,low,high", [(5.0, -6.0, 0.5), (5.0, -30.0, -3.0), (50.0, -20.0, 2.0), (500.0, -300.0, -90.0), (2.0, -1e4, 0.1), (1e6, -400.0, 400.0)])
@pytest.mark.parametrize("D", [64, 128])
def test_capped_scores_far_from_their_row_largest(ctx, cap, low, high, D):
    """Nearly all scores of a row near `low`, a few near `high`, in every tile or in the first, a middle or the last one only."""
    rng = _rng(D + int(cap))
    n, H = 700, 1
    u = rng.standard_normal(D)
    u /= np.linalg.norm(u)
    scale = 0.125
    q = f32_to_bf16_bits((8.0 * u[None, None] + 0.05 * rng.standard_normal((n, H, D))).astype(np.float32))
    level = np.full(n, low)
    level[rng.integers(0, n, 5)] = high
    level[[3, 350, 699]] = high
    k = f32_to_bf16_bits((level[:, None, None] * u[None, None] + 0.05 * rng.standard_normal((n, H, D))).astype(np.float32))
    v = _bf16(rng, n, H, D)
    cu = _cu([n])
    out, lse = _run_masked(ctx, to_dev(q), to_dev(k), to_dev(v), cu, None, scale, da.AttnMask(softcap=cap))
    _check_masked(out, lse, q, k, v, cu, cu, scale, cap=cap)


@pytest.mark.parametrize("few,D,parts", [(False, 64, False), (False, 128, False), (False, 128, True), (True, 64, False), (True, 128, True)])
def test_what_a_row_does_not_see_has_no_effect(ctx, few, D, parts):
    """NaN and infinite keys and values behind a causal mask: rows before them keep their bits, rows that see them get them."""
    rng = _rng(D + parts)
    lk = 2500 if parts else 300
    lq = 8 if few else 200
    H = 2
    q, k, v = _bf16(rng, lq, H, D), _bf16(rng, lk, H, D), _bf16(rng, lk, H, D)
    cu_q, cu_k = _cu([lq]), _cu([lk])
    at = [lk - lq + (1 if few else 50), lk - lq + (3 if few else 100), lk - lq + (6 if few else 170)]  # the rows 1, 3, 6 or 50, 100, 170 see them first
    dk, dv = to_dev(k), to_dev(v)
    mask = da.AttnMask(causal=True)
    clean, clean_lse = _run_masked(ctx, to_dev(q), dk, dv, cu_q, cu_k, D ** -0.5, mask)
    dv[at[0], 0, 5] = float("nan")
    dv[at[1], :, 9] = float("-inf")
    dv[at[1], :, 11] = float("inf")
    dk[at[2], 1, 3] = float("nan")
    out, lse = _run_masked(ctx, to_dev(q), dk, dv, cu_q, cu_k, D ** -0.5, mask)
    r = [a - (lk - lq) for a in at]
    same = out.view(torch.int16) == clean.view(torch.int16)
    want = torch.ones_like(same)
    want[r[0]:, 0, 5] = False
    want[r[1]:, :, 9] = False
    want[r[1]:, :, 11] = False
    want[r[2]:, 1, :] = False
    assert torch.equal(same, want)
    f = out.float()
    assert bool(torch.isnan(f[r[0]:, 0, 5]).all()) and bool(torch.isnan(f[r[2]:, 1]).all()) and bool(torch.isnan(lse[r[2]:, 1]).all())
    assert bool((f[r[1]:, 0, 9] == float("-inf")).all()) and bool((f[r[1]:r[2], :, 11] == float("inf")).all())
    assert torch.equal(lse[:r[2]], clean_lse[:r[2]]) and torch.equal(lse[:, 0], clean_lse[:, 0])


@pytest.mark.parametrize("rows", [2, 700])
def test_values_that_are_nowhere_finite(ctx, rows):
    """All values NaN, or one element of each infinite: every row that sees a key gets them, and the call ends soon."""
    rng = _rng(rows)
    n, H, D = 3000, 4, 128
    q, k, v = to_dev(_bf16(rng, rows, H, D)), to_dev(_bf16(rng, n, H, D)), to_dev(_bf16(rng, n, H, D))
    mask = da.AttnMask(causal=True)
    clean, _ = _run_masked(ctx, q, k, v, _cu([rows]), _cu([n]), 0.1, mask)
    v[:, :, 77] = float("inf")
    out, _ = _run_masked(ctx, q, k, v, _cu([rows]), _cu([n]), 0.1, mask)
    assert bool(torch.isinf(out[:, :, 77]).all())
    keep = [d for d in range(D) if d != 77]
    assert torch.equal(out[:, :, keep].view(torch.int16), clean[:, :, keep].view(torch.int16))
    v.fill_(float("nan"))
    out, _ = _run_masked(ctx, q, k, v, _cu([rows]), _cu([n]), 0.1, mask)
    assert bool(torch.isnan(out).all())


@pytest.mark.parametrize("lq,lk,D", [(400, 400, 64), (200, 400, 128), (6, 700, 64), (6, 700, 128), (140, 3000, 128)])
def test_padding_and_other_documents_may_hold_anything(ctx, lq, lk, D):
    rng = _rng(lq + D)
    H, G = 4, 2
    q, k, v = _bf16(rng, lq, H, D), _bf16(rng, lk, G, D), _bf16(rng, lk, G, D)
    ids = rng.integers(0, 3, lk).astype(np.int32)
    ids[lk - lq:] = np.where(rng.random(lq) < 0.2, -1, ids[lk - lq:])
    q_ids = ids[lk - lq:].copy()
    q_ids[q_ids == 2] = 1  # nobody is of document 2
    dirty = (ids < 0) | (ids == 2)
    q_dev = to_dev(q)
    q_dev[torch.from_numpy(q_ids < 0).cuda()] = float("nan")
    dk, dv = to_dev(k), to_dev(v)
    for t in (dk, dv):
        t[torch.from_numpy(dirty).cuda()] = float("nan")
        t[int(np.flatnonzero(dirty)[0])] = float("inf")
    kw = dict(causal=True, prefix=[lk // 2], cap=0.0, q_doc=q_ids, k_doc=ids)
    out, lse = _run_masked(ctx, q_dev, dk, dv, _cu([lq]), _cu([lk]), D ** -0.5, _mask(kw))
    _check_masked(out, lse, q, k, v, _cu([lq]), _cu([lk]), D ** -0.5, **kw)
    # the lowest ids are ids like others
    ids2, q_ids2 = np.where(ids < 0, -2 ** 31, ids).astype(np.int32), np.where(q_ids < 0, -2 ** 31, q_ids).astype(np.int32)
    out2, lse2 = _run_masked(ctx, q_dev, dk, dv, _cu([lq]), _cu([lk]), D ** -0.5, _mask(dict(kw, q_doc=q_ids2, k_doc=ids2)))
    assert torch.equal(out2.view(torch.int16), out.view(torch.int16)) and torch.equal(lse2, lse)


@pytest.mark.parametrize("few", [True, False])
def test_more_sequences_than_a_launch_takes(ctx, few):
    rng = _rng(5 + few)
    n, H, G, D = 150, 4, 2, 64
    k_lens = rng.integers(0, 150, n).tolist()
    q_lens = [1] * n if few else rng.integers(0, 40, n).tolist()
    k_lens = [max(a, b) for a, b in zip(k_lens, q_lens)]
    q, k, v = _bf16(rng, sum(q_lens), H, D), _bf16(rng, sum(k_lens), G, D), _bf16(rng, sum(k_lens), G, D)
    k_doc = _docs(rng, k_lens, 3, 5, shuffle=True)
    cu_q, cu_k = _cu(q_lens), _cu(k_lens)
    kw = dict(causal=True, prefix=rng.integers(0, 30, n).tolist(), cap=0.0, k_doc=k_doc,
              q_doc=np.concatenate([k_doc[cu_k[i + 1] - m:cu_k[i + 1]] for i, m in enumerate(q_lens)]))
    out, lse = _run_masked(ctx, to_dev(q), to_dev(k), to_dev(v), cu_q, cu_k, 0.125, _mask(kw))
    _check_masked(out, lse, q, k, v, cu_q, cu_k, 0.125, **kw)


def test_strided_rows_give_the_same_bits(ctx):
    rng = _rng(31)
    H, G, D = 6, 2, 64
    for q_lens, k_lens in (([300, 7], [300, 7]), ([1, 2], [400, 33])):
        Tq, Tk = sum(q_lens), sum(k_lens)
        fused = to_dev(_bf16(rng, max(Tq, Tk), (H + 2 * G) * D))
        q = fused[:Tq, :H * D].unflatten(1, (H, D))
        k, v = fused[:Tk, H * D:(H + G) * D].unflatten(1, (G, D)), fused[:Tk, (H + G) * D:].unflatten(1, (G, D))
        mask = da.AttnMask(causal=True)
        a, la = _run_masked(ctx, q, k, v, _cu(q_lens), _cu(k_lens), 0.125, mask)
        b, lb = _run_masked(ctx, q.contiguous(), k.contiguous(), v.contiguous(), _cu(q_lens), _cu(k_lens), 0.125, mask)
        assert torch.equal(a.view(torch.int16), b.view(torch.int16)) and torch.equal(la, lb)


def test_rows_beyond_four_gib(ctx):
    """Row strides of 2^24 elements: the rows lie over 6 GB."""
    n, D = 200, 128
    print("rows over 6 GB", flush=True)
    big = torch.empty(n * 2 ** 24, dtype=torch.bfloat16, device="cuda")
    far = big.as_strided((n, 1, D), (2 ** 24, D, 1))
    x = to_dev(_bf16(_rng(8), n, 1, D))
    far.copy_(x)
    for rows in (1, n):
        a, la = _run_masked(ctx, x[:rows], far, far, _cu([rows]), _cu([n]), 0.1, None)
        b, lb = _run_masked(ctx, x[:rows], x, x, _cu([rows]), _cu([n]), 0.1, None)
        assert torch.equal(a.view(torch.int16), b.view(torch.int16)) and torch.equal(la, lb)
    a, _ = _run_masked(ctx, far, x, x, _cu([n]), _cu([n]), 0.1, None)
    assert torch.equal(a.view(torch.int16), b.view(torch.int16))
    y = torch.empty_like(x)
    da.dit_attn_qk_norm_rope(ctx, da.NormHeads(x, y), None, n, D, da.NORM_RMS, 1e-6, None, 0, da.ROPE_HALF, _stream())
    da.dit_attn_qk_norm_rope(ctx, da.NormHeads(far, far), None, n, D, da.NORM_RMS, 1e-6, None, 0, da.ROPE_HALF, _stream())
    assert torch.equal(far.contiguous().view(torch.int16), y.view(torch.int16))


def test_without_a_mask_it_is_the_unmasked_operation(ctx):
    rng = _rng(77)
    lens, H, D = [500, 129, 1], 3, 128
    q, k, v = (_bf16(rng, sum(lens), H, D) for _ in range(3))
    cu = _cu(lens)
    out, lse = _run_masked(ctx, to_dev(q), to_dev(k), to_dev(v), cu, None, 0.09, None)
    ref, ref_lse = torch.empty_like(out), torch.empty_like(lse)
    da.dit_attn_varlen_fwd_lse(ctx, to_dev(q), to_dev(k), to_dev(v), cu, H, D, 0.09, ref, ref_lse, _stream())
    _check_masked(out, lse, q, k, v, cu, cu, 0.09)
    _check_masked(ref, None, q, k, v, cu, cu, 0.09)
    assert float((lse - ref_lse).abs().max()) <= 4e-3 + 1e-4


def test_captured_calls_replay(ctx):
    """Calls with parts and ids in a graph, replayed between eager calls of other packs; a context that has not run such a call
    refuses the capture."""
    rng = _rng(55)
    H, G, D = 4, 2, 128
    q, k, v = to_dev(_bf16(rng, 3, H, D)), to_dev(_bf16(rng, 5000, G, D)), to_dev(_bf16(rng, 5000, G, D))
    ids = torch.from_numpy(_docs(rng, [5000], 3, 9, shuffle=True)).cuda()
    mask = da.AttnMask(causal=True, q_doc=ids[-3:].clone(), k_doc=ids)
    cu_q, cu_k = _cu([3]), _cu([5000])
    own = da.dit_attn_create(0)
    side = torch.cuda.Stream()
    out, lse = torch.empty_like(q), torch.empty((3, H), device="cuda")
    pos = torch.arange(3, dtype=torch.int32, device="cuda")[:, None].contiguous() + 4997
    spec, table, turned = da.RopeSpec([128]), torch.empty((3, 64, 2), device="cuda"), torch.empty_like(q)

    def call(h, stream):
        da.dit_attn_rope_table(h, pos, 3, spec, table, stream)
        da.dit_attn_qk_norm_rope(h, da.NormHeads(q, turned), None, 3, D, da.NORM_RMS, 1e-6, table, 128, da.ROPE_HALF, stream)
        da.dit_attn_masked_varlen_fwd(h, turned, k, v, cu_q, cu_k, H, G, D, 0.09, mask, out, lse, stream)

    try:
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            with pytest.raises(da.DitAttnError) as ei:
                da.dit_attn_masked_varlen_fwd(own, q, k, v, cu_q, cu_k, H, G, D, 0.09, mask, out, lse, side.cuda_stream)
            assert ei.value.code == -12
        with torch.cuda.stream(side):
            call(own, side.cuda_stream)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            call(own, side.cuda_stream)
        for i in range(4):
            q.copy_(torch.randn_like(q))
            k[i::7] *= 1.5
            out.zero_()
            lse.zero_()
            g.replay()
            torch.cuda.synchronize()
            got, got_lse = out.clone(), lse.clone()
            # an eager call that outgrows the workspace of the captured one
            _run_masked(own, to_dev(_bf16(rng, 2, 16, 128)), to_dev(_bf16(rng, 9000 + 4000 * i, 8, 128)), to_dev(_bf16(rng, 9000 + 4000 * i, 8, 128)),
                        _cu([2]), _cu([9000 + 4000 * i]), 0.1, da.AttnMask(causal=True))
            call(ctx, _stream())
            torch.cuda.synchronize()
            assert torch.equal(got.view(torch.int16), out.view(torch.int16)) and torch.equal(got_lse, lse), i
    finally:
        torch.cuda.synchronize()
        da.dit_attn_destroy(own)


def test_a_block_from_projection_to_attention(ctx):
    """Table, norm and rotation in place in the fused projection, attention on its rows: each step against the oracle on the bits
    that the step before left."""
    rng = _rng(91)
    lens, H, G, D, R = [300, 77], 4, 2, 128, 96
    T = sum(lens)
    qkv = to_dev(_bf16(rng, T, (H + 2 * G) * D))
    pos = rng.integers(0, 5000, (T, 3)).astype(np.int32)
    spec = da.RopeSpec([32, 32, 32])
    table = torch.empty((T, R // 2, 2), device="cuda")
    views = [qkv[:, a:b].unflatten(1, (-1, D)) for a, b in ((0, H * D), (H * D, (H + G) * D), ((H + G) * D, (H + 2 * G) * D))]
    before = [widen(to_bits(x)) for x in views]
    w = (1 + 0.1 * rng.standard_normal(D)).astype(np.float32)
    dw = torch.from_numpy(w).cuda()
    out, lse = torch.empty((T, H, D), dtype=torch.bfloat16, device="cuda"), torch.empty((T, H), device="cuda")
    mask = da.AttnMask(causal=True, prefix=[64, 8], softcap=30.0)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    s = stream.cuda_stream  # none of these tensors' own stream, and not the current one
    da.dit_attn_rope_table(ctx, torch.from_numpy(pos).cuda(), T, spec, table, s)
    da.dit_attn_qk_norm_rope(ctx, da.NormHeads(views[0], views[0], dw), da.NormHeads(views[1], views[1], dw), T, D, da.NORM_RMS, 1e-6, table, R,
                             da.ROPE_INTERLEAVED, s)
    da.dit_attn_masked_varlen_fwd(ctx, *views, _cu(lens), None, H, G, D, D ** -0.5, mask, out, lse, s)
    torch.cuda.synchronize()
    f, axis = orc.frequencies([32, 32, 32], [1e4] * 3, "plain", [1.0] * 3)
    tab = orc.rope_table(pos, f, axis)
    assert np.abs(table.cpu().numpy() - tab).max() <= 4 * 2.0 ** -24 + 5000 * 2.0 ** -52
    for i in (0, 1):
        y, normed = orc.norm_rope(before[i], "rms", 1e-6, w, None, table.cpu().numpy().astype(np.float64), R, False)
        assert np.all(np.abs(widen(to_bits(views[i])) - y) <= _norm_bound(before[i], y, normed, None, "rms", w, 1e-6))
    bits = [to_bits(x) for x in views]
    _check_masked(out, lse, *bits, _cu(lens), _cu(lens), D ** -0.5, causal=True, prefix=[64, 8], cap=30.0)


# ---------------------------------------------------------------- refusals

def test_refusals(ctx):
    x = torch.zeros((4, 2, 64), dtype=torch.bfloat16, device="cuda")
    out = torch.full((4, 2, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    f = torch.zeros(4 * 64, device="cuda")
    ids = torch.zeros(4, dtype=torch.int32, device="cuda")
    cu = [0, 1, 4]

    def masked(q=x, k=x, v=x, cu_q=cu, cu_k=None, H=2, G=2, D=64, scale=1.0, mask=None, o=out, lse=None, **kw):
        with pytest.raises(da.DitAttnError) as ei:
            da.dit_attn_masked_varlen_fwd(ctx, q, k, v, cu_q, cu_k, H, G, D, scale, mask, o, lse, _stream(), **kw)
        assert da.dit_attn_last_error(ctx)
        return ei.value.code

    def spec(dims=(16,), **kw):
        s = da.RopeSpec(dims, **kw)
        return s

    def table(s, pos=ids, n=4, tab=f):
        with pytest.raises(da.DitAttnError) as ei:
            da.dit_attn_rope_table(ctx, pos, n, s, tab, _stream())
        return ei.value.code

    def norm(q=None, k=None, n=4, D=64, kind=da.NORM_RMS, eps=1e-6, tab=f, rot=8, layout=0, none=False):
        if q is None and not none:
            q = da.NormHeads(x, out)
        with pytest.raises(da.DitAttnError) as ei:
            da.dit_attn_qk_norm_rope(ctx, q, k, n, D, kind, eps, tab, rot, layout, _stream())
        return ei.value.code

    nan, inf = float("nan"), float("inf")
    assert masked(D=96) == -2 and masked(cu_q=[0, 3, 1]) == -3 and masked(cu_q=[1, 2, 4]) == -3 and masked(cu_k=[0, 5, 2]) == -3
    assert masked(scale=nan) == -5 and masked(scale=inf) == -5 and masked(H=0) == -6 and masked(H=3, G=2) == -6 and masked(G=0) == -6
    assert masked(q=0) == -1 and masked(k=0, row_strides=(128, 128, 128)) == -1 and masked(o=0) == -1
    assert masked(q=x.data_ptr() + 2) == -7 and masked(lse=f.data_ptr() + 2) == -7 and masked(mask=da.AttnMask(slopes=f.data_ptr() + 1)) == -7
    assert masked(mask=da.AttnMask(q_doc=ids.data_ptr() + 2, k_doc=ids)) == -7
    assert masked(mask=da.AttnMask(causal=2)) == -13 and masked(mask=da.AttnMask(softcap=-1.0)) == -13 and masked(mask=da.AttnMask(softcap=nan)) == -13
    assert masked(mask=da.AttnMask(softcap=inf)) == -13 and masked(mask=da.AttnMask(prefix=[1, 1])) == -13
    assert masked(mask=da.AttnMask(causal=True, prefix=[1, -1])) == -13 and masked(mask=da.AttnMask(q_doc=ids)) == -13 and masked(mask=da.AttnMask(k_doc=ids)) == -13
    for bad in (120, 132, 2 ** 24 + 8, -128):
        for i in range(3):
            assert masked(row_strides=[bad if j == i else 128 for j in range(3)]) == -16
    assert table(spec(), pos=0) == -1 and table(spec(), tab=0) == -1 and table(spec(), n=-1) == -3 and table(None) == -1
    assert table(spec(), pos=ids.data_ptr() + 2) == -7 and table(spec(), tab=f.data_ptr() + 4) == -7 and table(spec(), n=2 ** 34 + 1) == -11
    for bad in (spec((3,)), spec((0,)), spec((-2,)), spec((130,)), spec((66, 64)), spec(theta=0.5), spec(theta=nan), spec(theta=inf), spec(scaling=4),
                spec(scaling=-1), spec(scaling=da.ROPE_LINEAR, factor=0.5), spec(scaling=da.ROPE_BASE, factor=nan), spec(magnitude=inf),
                spec(scaling=da.ROPE_BANDS, original_length=0.0), spec(scaling=da.ROPE_BANDS, original_length=64.0, low=3.0, high=3.0)):
        assert table(bad) == -14
    assert norm(none=True) == -1 and norm(D=96) == -2 and norm(kind=3) == -15 and norm(kind=-1) == -15 and norm(eps=-1.0) == -15 and norm(eps=nan) == -15
    assert norm(rot=12) == -14 and norm(rot=72) == -14 and norm(rot=-8) == -14 and norm(layout=2) == -14 and norm(n=-1) == -3 and norm(tab=None) == -1
    assert norm(tab=f.data_ptr() + 8) == -7 and norm(n=2 ** 36) == -11
    P = x.data_ptr()
    side = lambda a=P, b=out.data_ptr(), **kw: da.NormHeads(a, b, **dict(dict(n_heads=2), **kw))
    assert norm(side(n_heads=0)) == -6 and norm(side(n_heads=65536)) == -6 and norm(side(a=0)) == -1 and norm(side(b=0)) == -1
    assert norm(side(a=P + 8)) == -7 and norm(side(b=out.data_ptr() + 2)) == -7 and norm(side(weight=f.data_ptr() + 4)) == -7
    assert norm(side(bias=f), kind=da.NORM_NONE) == -15 and norm(side(weight=f), kind=da.NORM_NONE) == -15
    assert norm(side(row_stride=120)) == -16 and norm(side(row_stride=130)) == -16 and norm(side(out_row_stride=64)) == -16
    assert norm(side(), side()) == -16 and norm(side(), side(a=out.data_ptr(), b=f.data_ptr())) == -16
    assert norm(side(b=P, out_row_stride=256)) == -16 and norm(side(), side(n_heads=0)) == -6
    torch.cuda.synchronize()
    assert bool((out == 3.0).all())
    # nothing to do
    da.dit_attn_rope_table(ctx, 0, 0, spec(), 0)
    da.dit_attn_qk_norm_rope(ctx, side(), None, 0, 64, da.NORM_RMS, 1e-6, None, 64)
    da.dit_attn_masked_varlen_fwd(ctx, x, x, x, [0, 0], [0, 4], 2, 2, 64, 1.0, None, 0)
    da.dit_attn_masked_varlen_fwd(ctx, x, x, x, [0], None, 2, 2, 64, 1.0, None, 0)
    # rows without any keys at all
    empty = torch.empty((0, 2, 64), dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros((4, 2), device="cuda")
    da.dit_attn_masked_varlen_fwd(ctx, x, empty, empty, [0, 4], [0, 0], 2, 2, 64, 1.0, None, out, lse, _stream())
    torch.cuda.synchronize()
    assert not bool(out.any()) and bool((lse == float("-inf")).all())
