"""The operators around a block's attention, as cases that can be timed and compared: the rotation table of token positions, the
norm and rotation of queries and keys for each head, and attention with masks, capped scores and a distance bias.

A case is a dict of plain values.  Lengths are texts ("4352*4 20506": four sequences of 4352 tokens and one of 20506).
`prepare` makes what a program holds before the call, `run` is one call, `work` the bytes and operations that it cannot do
without, `exact` the result in 64 bits.  With `own` false `run` computes the plain form, in elementary torch operations; with
`own` true it calls the library.
"""
from __future__ import annotations

import functools
import math

import numpy as np
import torch

own = False


def _lens(text: str) -> list:
    """"4352*2 7" -> [4352, 4352, 7]."""
    out = []
    for part in text.split():
        length, _, times = part.partition("*")
        out += [int(length)] * int(times or 1)
    return out


def _text(lens) -> str:
    return " ".join(str(n) for n in lens)


def _table(rows, axes, scaling="plain", factor=1.0, start=0) -> dict:
    return dict(op="table", rows=rows, axes=axes, scaling=scaling, factor=factor, start=start)


def _norm(rows, heads, kv_heads, head_dim, rot, norm="rms", layout="half", affine="weight", fused=False) -> dict:
    return dict(op="norm", rows=rows, heads=heads, kv_heads=kv_heads, head_dim=head_dim, rot=rot, norm=norm, layout=layout,
                affine=affine, fused=fused)


def _masked(q_lens, k_lens, heads, kv_heads, head_dim, causal=False, prefix="", cap=0.0, bias=False, docs=0, pad=0, lse=False,
            fused=False) -> dict:
    return dict(op="masked", q_lens=q_lens, k_lens=k_lens, heads=heads, kv_heads=kv_heads, head_dim=head_dim, causal=causal,
                prefix=prefix, cap=cap, bias=bias, docs=docs, pad=pad, lse=lse, fused=fused)


def listed() -> list:
    return [
        # Positions of one low-resolution image (text axis, row, column) at head dimension 64: latency.
        dict(_table(410, "16 24 24"), name="table_image"),
        # Positions of the long video (frame, row, column), slow frequencies stretched fourfold, far from the origin.
        dict(_table(76112, "44 42 42", scaling="bands", factor=4.0, start=100000), name="table_video"),
        # One new token: queries and keys of one row.
        dict(_norm(1, 24, 8, 128, 128), name="norm_token"),
        # The batch of four images straight from the fused projection (rows of query, key and value heads).
        dict(_norm(17408, 24, 24, 128, 128, layout="interleaved", fused=True), name="norm_images"),
        # Ragged rows of an image batch at head dimension 64: mean and variance, weights and biases, a part of the head rotated.
        dict(_norm(16989, 24, 24, 64, 32, norm="layer", affine="both"), name="norm_images_d64"),
        # One GPU's ten heads of the long video.
        dict(_norm(76112, 10, 10, 128, 128), name="norm_video"),
        # One new token of one short sequence: the smallest attention call.
        dict(_masked("1", "410", 24, 24, 64, causal=True), name="token_small"),
        # One new token for each of a batch of requests with caches of several lengths, three query heads to a key head.
        dict(_masked("1*8", "20506 4352*4 1280*2 77", 24, 8, 128, causal=True, lse=True), name="token_batch"),
        # The text rows of a video request against all of its keys, capped scores.
        dict(_masked("226", "20506", 24, 24, 128, cap=30.0), name="text_rows"),
        # A padded batch of images at head dimension 64: three documents to a row of the batch, the rest of it padding that sees
        # nothing, and a bias on the distance.
        dict(_masked("4352*6", "", 24, 24, 64, bias=True, docs=3, pad=101), name="padded_docs_d64"),
        # Images generated in order behind their text, which all tokens see; values read in place from the fused projection.
        dict(_masked("4352*4", "", 24, 24, 128, causal=True, prefix="256*4", lse=True, fused=True), name="prefix_images"),
        # Images batched with a video, capped scores: the largest call.
        dict(_masked("4352*2 1280 20506 4352*2 1280", "", 24, 24, 128, cap=50.0), name="cap_mixed"),
    ]


MAX_FLOPS = 6.2e12  # under the largest listed case (cap_mixed)
MAX_PAIRS = 5.1e8   # keys seen or not, a head: what the plain form goes through


def _log_int(rng, lo: int, hi: int) -> int:
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng) -> dict:
    """One more case of the listed ranges."""
    while True:
        case = _draw_kind(rng, rng.choice(["table", "norm", "norm", "token", "rows", "self", "self", "docs"]))
        if case["op"] != "masked":
            return case
        q_lens, k_lens = _both_lens(case)
        if sum(a * b for a, b in zip(q_lens, k_lens)) * case["heads"] <= MAX_PAIRS * 24 and work(case)["flops"] <= MAX_FLOPS:
            return case


def _draw_kind(rng, kind: str) -> dict:
    head_dim = rng.choice([64, 128, 128])
    kv = rng.choice([1, 2, 3, 8])
    heads = kv * rng.choice([1, 2, 3, 4])
    if kind == "table":
        n = rng.randint(1, 4)
        axes = [2 * rng.randint(1, head_dim // (2 * n)) for _ in range(n)]
        scaling = rng.choice(["plain", "linear", "base", "bands"])
        return _table(_log_int(rng, 1, 76112), _text(axes), scaling, 1.0 if scaling == "plain" else round(rng.uniform(1.0, 16.0), 2),
                      rng.choice([0, rng.randint(0, 1000000)]))
    if kind == "norm":
        rows = _log_int(rng, 1, 76112 if heads + kv <= 20 else 17408)
        return _norm(rows, heads, kv, head_dim, 8 * rng.randint(0, head_dim // 8), rng.choice(["rms", "rms", "layer", "none"]),
                     rng.choice(["half", "interleaved"]), rng.choice(["none", "weight", "both"]), rng.random() < 0.5)
    cap = rng.choice([0.0, 0.0, 20.0, 30.0, 50.0])
    bias, lse = rng.random() < 0.3, rng.random() < 0.5
    if kind == "token":  # one or a few new tokens against caches
        n = rng.randint(1, 8)
        k_lens = [_log_int(rng, 16, 40000) for _ in range(n)]
        q_lens = [rng.choice([1, 1, 1, rng.randint(1, 16)])] * n
        return _masked(_text(q_lens), _text(k_lens), heads, kv, head_dim, True, "", cap, bias, 0, 0, lse)
    if kind == "rows":  # some rows against many keys, or many against few
        n = rng.randint(1, 4)
        q_lens, k_lens = [[_log_int(rng, 16, 20506) for _ in range(n)] for _ in range(2)]
        return _masked(_text(q_lens), _text(k_lens), heads, kv, head_dim, rng.random() < 0.3, "", cap, bias, 0, 0, lse)
    n = rng.randint(1, 6)
    lens = [_log_int(rng, 16, 20506 if n == 1 else 8192) for _ in range(n)]
    fused = rng.random() < 0.3
    if kind == "docs":
        return _masked(_text(lens), "", heads, kv, head_dim, rng.random() < 0.5, "", cap, bias, rng.randint(1, 6),
                       rng.choice([0, rng.randint(1, 300)]), lse, fused)
    causal = rng.random() < 0.7
    prefix = _text([rng.randint(0, 512) for _ in lens]) if causal and rng.random() < 0.6 else ""
    return _masked(_text(lens), "", heads, kv, head_dim, causal, prefix, cap, bias, 0, 0, lse, fused)


# ---------------------------------------------------------------- what a case's fields mean

def _both_lens(case):
    q_lens = _lens(case["q_lens"])
    return q_lens, _lens(case["k_lens"]) if case["k_lens"] else q_lens


def _prefix(case, n):
    return _lens(case["prefix"]) if case["prefix"] else [0] * n


def _doc_ids(case, n) -> np.ndarray:
    """Ids of a sequence of n positions: `docs` runs of nearly equal length, then `pad` positions without a document."""
    ids = np.full(n, -1, dtype=np.int32)
    live = max(0, n - case["pad"])
    ids[:live] = np.arange(live, dtype=np.int64) * case["docs"] // max(live, 1)
    return ids


def _frequencies(case) -> np.ndarray:
    """Radians per position of every rotated pair, and the axis of each."""
    out, axis = [], []
    s = case["factor"]
    for a, d in enumerate(_lens(case["axes"])):
        for j in range(d // 2):
            f = 10000.0 ** (-2.0 * j / d)
            if case["scaling"] == "linear":
                f /= s
            elif case["scaling"] == "base" and d > 2:
                f = (10000.0 * s ** (d / (d - 2.0))) ** (-2.0 * j / d)
            elif case["scaling"] == "bands":
                turns = 4096.0 * f / (2.0 * math.pi)
                g = min(1.0, max(0.0, (turns - 1.0) / (32.0 - 1.0)))
                f = f * (g + (1.0 - g) / s)
            out.append(f)
            axis.append(a)
    return np.array(out), np.array(axis)


def _magnitude(case) -> float:
    return 0.1 * math.log(case["factor"]) + 1.0 if case["scaling"] == "bands" else 1.0


def _inputs(case: dict, seed: int) -> dict:
    """The tensors that a call reads, from the seed alone."""
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def noise(*shape):
        return torch.randn(shape, device="cuda", generator=gen)

    if case["op"] == "table":
        # A grid walked in order, its last axis fastest, from a random corner.
        n, axes = case["rows"], len(_lens(case["axes"]))
        corner = torch.randint(0, 64, (axes,), device="cuda", generator=gen) + case["start"]
        i = torch.arange(n, device="cuda")
        side = max(1, round(n ** (1.0 / axes)))
        grid = [(i // side ** (axes - 1 - a)) % side if a else i // side ** (axes - 1) for a in range(axes)]
        return dict(positions=(torch.stack(grid, 1) + corner).to(torch.int32))
    H, G, D = case["heads"], case["kv_heads"], case["head_dim"]
    if case["op"] == "norm":
        n, R = case["rows"], case["rot"]
        x = dict()
        if case["fused"]:
            qkv = noise(n, (H + 2 * G) * D).mul_(2.0).to(torch.bfloat16)
            x["q"], x["k"] = qkv[:, :H * D].unflatten(1, (H, D)), qkv[:, H * D:(H + G) * D].unflatten(1, (G, D))
        else:
            x["q"], x["k"] = noise(n, H, D).mul_(2.0).to(torch.bfloat16), noise(n, G, D).mul_(2.0).to(torch.bfloat16)
        angle = noise(n, R // 2) * 100.0
        x["table"] = torch.stack([angle.cos(), angle.sin()], 2) if R else None
        for side in "qk":
            x[side + "_weight"] = 1.0 + 0.2 * noise(D) if case["affine"] != "none" and case["norm"] != "none" else None
            x[side + "_bias"] = 0.2 * noise(D) if case["affine"] == "both" and case["norm"] != "none" else None
        return x
    q_lens, k_lens = _both_lens(case)
    if case["fused"]:
        qkv = noise(sum(q_lens), (H + 2 * G) * D).to(torch.bfloat16)
        x = dict(q=qkv[:, :H * D].unflatten(1, (H, D)), k=qkv[:, H * D:(H + G) * D].unflatten(1, (G, D)),
                 v=qkv[:, (H + G) * D:].unflatten(1, (G, D)))
    else:
        x = dict(q=noise(sum(q_lens), H, D).to(torch.bfloat16), k=noise(sum(k_lens), G, D).to(torch.bfloat16),
                 v=noise(sum(k_lens), G, D).to(torch.bfloat16))
    x["cu_q"], x["cu_k"] = (np.concatenate([[0], np.cumsum(n)]).astype(np.int32) for n in (q_lens, k_lens))
    x["scale"] = 1.0 / math.sqrt(D)
    # Slopes of a geometric series; a factor of the seed's own.
    x["slopes"] = (0.5 + torch.rand(1, device="cuda", generator=gen)) * 2.0 ** (
        -8.0 * torch.arange(1, H + 1, device="cuda", dtype=torch.float32) / H) if case["bias"] else None
    x["k_doc"] = x["q_doc"] = None
    if case["docs"]:
        ids = [_doc_ids(case, n) for n in k_lens]
        x["k_doc"] = torch.from_numpy(np.concatenate(ids)).to("cuda")
        x["q_doc"] = torch.from_numpy(np.concatenate([i[n - m:] for i, n, m in zip(ids, k_lens, q_lens)])).to("cuda")
    return x


# ---------------------------------------------------------------- the library's calls

@functools.lru_cache(maxsize=None)
def _context() -> int:
    """The context a program creates once and keeps."""
    import paper_2604_04335_amd as da

    return da.dit_attn_create(torch.cuda.current_device())


def prepare(case: dict, seed: int) -> dict:
    st = dict(case)
    st.update(_inputs(case, seed))
    if case["op"] == "table":
        f, axis = _frequencies(case)
        st["freq"] = torch.from_numpy(f).to("cuda")
        st["axis"] = torch.from_numpy(axis).to("cuda")
    if not own:
        return st
    import paper_2604_04335_amd as da

    st.update(da=da, ctx=_context(), stream=torch.cuda.current_stream().cuda_stream)
    if case["op"] == "table":
        kind = {"plain": da.ROPE_PLAIN, "linear": da.ROPE_LINEAR, "base": da.ROPE_BASE, "bands": da.ROPE_BANDS}[case["scaling"]]
        st["spec"] = da.RopeSpec(_lens(case["axes"]), theta=10000.0, scaling=kind, factor=case["factor"], original_length=4096.0,
                                 low=1.0, high=32.0, magnitude=_magnitude(case))
        st["table"] = torch.empty((case["rows"], st["spec"].rot_dim // 2, 2), device="cuda")
    elif case["op"] == "norm":
        n, H, G, D = case["rows"], case["heads"], case["kv_heads"], case["head_dim"]
        st["q_out"] = torch.empty((n, H, D), dtype=torch.bfloat16, device="cuda")
        st["k_out"] = torch.empty((n, G, D), dtype=torch.bfloat16, device="cuda")
        st["kind"] = {"none": da.NORM_NONE, "rms": da.NORM_RMS, "layer": da.NORM_LAYER}[case["norm"]]
        st["pairs"] = {"half": da.ROPE_HALF, "interleaved": da.ROPE_INTERLEAVED}[case["layout"]]
    else:
        st["mask"] = da.AttnMask(causal=case["causal"], softcap=case["cap"], slopes=st["slopes"], q_doc=st["q_doc"], k_doc=st["k_doc"],
                                 prefix=_prefix(case, len(st["cu_q"]) - 1) if case["prefix"] else None)
        st["out"] = torch.empty(st["q"].shape, dtype=torch.bfloat16, device="cuda")
        st["row_lse"] = torch.empty(st["q"].shape[:2], device="cuda") if case["lse"] else None
    return st


def run(st: dict):
    if not own:
        return {"table": _plain_table, "norm": _plain_norm, "masked": _plain_masked}[st["op"]](st)
    da, ctx, stream = st["da"], st["ctx"], st["stream"]
    if st["op"] == "table":
        da.dit_attn_rope_table(ctx, st["positions"], st["rows"], st["spec"], st["table"], stream)
        return st["table"]
    if st["op"] == "norm":
        da.dit_attn_qk_norm_rope(ctx, da.NormHeads(st["q"], st["q_out"], st["q_weight"], st["q_bias"]),
                                 da.NormHeads(st["k"], st["k_out"], st["k_weight"], st["k_bias"]), st["rows"], st["head_dim"], st["kind"], 1e-6,
                                 st["table"], st["rot"], st["pairs"], stream)
        return st["q_out"], st["k_out"]
    da.dit_attn_masked_varlen_fwd(ctx, st["q"], st["k"], st["v"], st["cu_q"], st["cu_k"], st["heads"], st["kv_heads"], st["head_dim"],
                                  st["scale"], st["mask"], st["out"], st["row_lse"], stream)
    return (st["out"], st["row_lse"]) if st["lse"] else st["out"]


# ---------------------------------------------------------------- the plain forms

def _plain_table(st):
    # 64 bits: an angle far from the origin has no bits left behind the point in 32
    angle = st["positions"].double()[:, st["axis"]] * st["freq"]
    return (torch.stack([angle.cos(), angle.sin()], 2) * _magnitude(st)).float()


def _plain_norm(st):
    R = st["rot"]

    def side(x, weight, bias):
        y = x.float()
        if st["norm"] == "layer":
            y = y - y.mean(2, keepdim=True)
        if st["norm"] != "none":
            y = y * torch.rsqrt((y * y).mean(2, keepdim=True) + 1e-6)
        if weight is not None:
            y = y * weight
        if bias is not None:
            y = y + bias
        if R:
            c, s = st["table"][:, None, :, 0], st["table"][:, None, :, 1]
            if st["layout"] == "half":
                a, b = y[..., :R // 2], y[..., R // 2:R]
                turned = torch.cat([a * c - b * s, b * c + a * s], 2)
            else:
                a, b = y[..., 0:R:2], y[..., 1:R:2]
                turned = torch.stack([a * c - b * s, b * c + a * s], 3).flatten(2)
            y = torch.cat([turned, y[..., R:]], 2)
        return y.to(torch.bfloat16)

    return side(st["q"], st["q_weight"], st["q_bias"]), side(st["k"], st["k_weight"], st["k_bias"])


def _visible(st, pos, j, q_ids, k_ids, prefix):
    """[rows, keys] of truth values, or None where every row sees every key."""
    seen = None
    if st["causal"]:
        seen = j[None, :] <= pos[:, None]
        if prefix:
            seen = seen | (j < prefix)[None, :]
    if q_ids is not None:
        same = (q_ids[:, None] == k_ids[None, :]) & (k_ids >= 0)[None, :]
        seen = same if seen is None else seen & same
    return seen


def _plain_masked(st):
    H, G = st["heads"], st["kv_heads"]
    out = torch.empty(st["q"].shape, dtype=torch.bfloat16, device="cuda")
    lse = torch.empty(st["q"].shape[:2], device="cuda")
    group = torch.arange(H, device="cuda") // (H // G)
    cu_q, cu_k = st["cu_q"].tolist(), st["cu_k"].tolist()
    for i, prefix in enumerate(_prefix(st, len(cu_q) - 1)):
        q0, q1, k0, k1 = cu_q[i], cu_q[i + 1], cu_k[i], cu_k[i + 1]
        kt = st["k"][k0:k1].float().permute(1, 2, 0)[group].contiguous()  # [H, D, keys]
        v = st["v"][k0:k1].float().transpose(0, 1)[group].contiguous()    # [H, keys, D]
        j = torch.arange(k1 - k0, device="cuda")
        step = max(1, int(5e8 // (H * (k1 - k0))))
        for r0 in range(q0, q1, step):
            r1 = min(q1, r0 + step)
            pos = torch.arange(r0, r1, device="cuda") + ((k1 - k0) - (q1 - q0) - q0)
            s = (st["q"][r0:r1].float().transpose(0, 1).contiguous() @ kt).mul_(st["scale"])
            if st["cap"]:
                s = s.div_(st["cap"]).tanh_().mul_(st["cap"])
            if st["bias"]:
                s -= st["slopes"][:, None, None] * (pos[:, None] - j[None, :]).abs().float()
            seen = _visible(st, pos, j, None if st["q_doc"] is None else st["q_doc"][r0:r1],
                            None if st["k_doc"] is None else st["k_doc"][k0:k1], prefix)
            if seen is not None:
                s.masked_fill_(~seen, -math.inf)
            m = s.amax(2, keepdim=True).clamp_min_(-1e30)  # a row that sees nothing keeps a finite reference
            p = s.sub_(m).exp_()
            total = p.sum(2, keepdim=True)
            o = (p @ v) / torch.where(total > 0, total, 1.0)
            out[r0:r1] = o.transpose(0, 1).to(torch.bfloat16)
            lse[r0:r1] = (m + total.log())[..., 0].t()
    return (out, lse) if st["lse"] else out


# ---------------------------------------------------------------- 64 bits

def exact(case: dict, seed: int):
    """What `run` returns, in 64 bits from the definitions."""
    x = _inputs(case, seed)
    if case["op"] == "table":
        f, axis = _frequencies(case)
        p = x["positions"].cpu().numpy().astype(np.float64)
        out = np.empty((case["rows"], len(f), 2))
        for i in range(len(f)):
            out[:, i, 0] = np.cos(p[:, axis[i]] * f[i]) * _magnitude(case)
            out[:, i, 1] = np.sin(p[:, axis[i]] * f[i]) * _magnitude(case)
        return torch.from_numpy(out)
    if case["op"] == "norm":
        return tuple(_exact_side(case, x[s].double(), x[s + "_weight"], x[s + "_bias"], x["table"]) for s in "qk")
    H, G = case["heads"], case["kv_heads"]
    q, k, v = x["q"], x["k"], x["v"]
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    cu_q, cu_k = x["cu_q"].tolist(), x["cu_k"].tolist()
    prefix = _prefix(case, len(cu_q) - 1)
    for i in range(len(cu_q) - 1):
        q0, q1, k0, k1 = cu_q[i], cu_q[i + 1], cu_k[i], cu_k[i + 1]
        keys = torch.arange(k1 - k0, device="cuda")
        step = max(1, int(2.5e8 // (k1 - k0)))
        for h in range(H):
            kt, vh = k[k0:k1, h * G // H].double().t().contiguous(), v[k0:k1, h * G // H].double()
            for r0 in range(q0, q1, step):
                r1 = min(q1, r0 + step)
                at = torch.arange(r0 - q0, r1 - q0, device="cuda") + (k1 - k0) - (q1 - q0)
                distance = at[:, None] - keys[None, :]
                s = (q[r0:r1, h].double() @ kt) * x["scale"]
                if case["cap"]:
                    s = torch.tanh(s / case["cap"]) * case["cap"]
                if case["bias"]:
                    s = s - x["slopes"][h].double() * distance.abs()
                hidden = torch.zeros_like(distance, dtype=torch.bool)
                if case["causal"]:
                    hidden |= (distance < 0) & (keys >= prefix[i])[None, :]
                if case["docs"]:
                    hidden |= x["q_doc"][r0:r1, None] != x["k_doc"][None, k0:k1]
                    hidden |= x["k_doc"][None, k0:k1] < 0
                s[hidden] = -math.inf
                row = torch.logsumexp(s, 1)
                live = row > -math.inf
                lse[r0:r1, h] = row
                out[r0:r1, h] = torch.exp(s - torch.where(live, row, 0.0)[:, None]) @ vh
    return (out, lse) if case["lse"] else out


def _exact_side(case, x, weight, bias, table):
    if case["norm"] == "layer":
        x = (x - x.mean(-1, keepdim=True)) / torch.sqrt(x.var(-1, unbiased=False, keepdim=True) + 1e-6)
    elif case["norm"] == "rms":
        x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / case["head_dim"] + 1e-6)
    x = x if weight is None else x * weight.double()
    x = (x if bias is None else x + bias.double()).clone()
    R = case["rot"]
    first = torch.arange(R // 2, device="cuda") * (2 if case["layout"] == "interleaved" else 1)
    second = first + (1 if case["layout"] == "interleaved" else R // 2)
    if R:
        turn = torch.view_as_complex(table.double())[:, None, :]
        z = torch.complex(x[..., first], x[..., second]) * turn
        x[..., first], x[..., second] = z.real, z.imag
    return x


# ---------------------------------------------------------------- floors

def work(case: dict) -> dict:
    if case["op"] == "table":
        axes = _lens(case["axes"])
        return {"bytes": case["rows"] * 4 * (len(axes) + sum(axes)), "flops": 0}
    H, G, D = case["heads"], case["kv_heads"], case["head_dim"]
    if case["op"] == "norm":
        return {"bytes": case["rows"] * (4 * D * (H + G) + 4 * case["rot"]), "flops": 0}
    q_lens, k_lens = _both_lens(case)
    pairs = keys = 0
    for lq, lk, prefix in zip(q_lens, k_lens, _prefix(case, len(q_lens))):
        pos = np.arange(lq, dtype=np.int64) + lk - lq
        if case["docs"]:
            ids = _doc_ids(case, lk)
            live = int((ids >= 0).sum())
            mine = ids[lk - lq:]
            first = np.searchsorted(ids[:live], mine)
            last = np.where(mine >= 0, np.searchsorted(ids[:live], mine, side="right"), first)
        else:
            live, first, last = lk, np.zeros_like(pos), np.full_like(pos, lk)
        if case["causal"]:
            last = np.minimum(last, np.maximum(pos + 1, prefix))
        pairs += int(np.maximum(last - first, 0).sum())
        keys += live
    rows = sum(q_lens)
    # Queries and outputs once, keys and values that anyone can see once, ids and the log-sum-exp where there are any
    nbytes = 4 * D * (H * rows + G * keys) + (4 * rows * H if case["lse"] else 0) + (4 * (rows + sum(k_lens)) if case["docs"] else 0)
    return {"bytes": nbytes, "flops": 4 * D * H * pairs}
