"""Operators for long samples: the quantised feature cache, norms fused with gate and residual, attention over selected blocks.

Each case is one operator as a sampling program calls it.  The cache holds a feature in 8 or 4 bits (groups of 64
values, one fp32 scale each) and is read back or forecast from; a module's output is normed, gated and added to the
residual stream and the stream normed for the next module; attention runs over the key blocks that a cheap score
selects for every block of queries.
"""
import math

import torch

own = False   # True: the framework's calls, False: the same in elementary operations

DEV = "cuda:0"
GROUP = 64          # values of a quantised feature that share a scale
QB, KB = 128, 64    # queries and keys of a block


def listed():
    return [
        # The tiny fp32 model's feature into an 8-bit slot and back: latency.
        dict(name="cache_rw_tiny_q8", op="cache_rw", n=2 * 64 * 128, dtype="f32", bits=8, out="f32"),
        # The video model's feature, 14 310 tokens, into a 4-bit slot and back.
        dict(name="cache_rw_video_q4", op="cache_rw", n=14310 * 3072, dtype="bf16", bits=4, out="bf16"),
        # A forecast step of the ordinary class-conditional batch from an 8-bit ring.
        dict(name="forecast_dit_q8", op="forecast", K=3, n=16 * 256 * 1152, dtype="bf16", bits=8, out="bf16"),
        # The forecast sweep's features [8, 16384, 3072] from an 8-bit ring: memory alone.
        dict(name="forecast_large_q8", op="forecast", K=3, n=8 * 16384 * 3072, dtype="bf16", bits=8, out="bf16"),
        # Four 4-bit nodes of an odd number of values (1021 tokens of 1155) into fp32.
        dict(name="forecast_odd_q4", op="forecast", K=4, n=1021 * 1155, dtype="f32", bits=4, out="f32"),
        # One token through a module's epilogue: norm, gate, residual, next norm; launch latency.
        dict(name="norm_one_token", op="norm", B=1, T=1, D=1152, post="rms", pre="layer", affine=False, mod=True,
             gate=True, res_scale=1.0, dtype="bf16"),
        # The class-conditional batch: module output added through its gate, LayerNorm and modulation of the next.
        dict(name="norm_dit_b16", op="norm", B=16, T=256, D=1152, post="none", pre="layer", affine=False, mod=True,
             gate=True, res_scale=1.0, dtype="bf16"),
        # The video model's rows with a norm on both sides of the module.
        dict(name="norm_video", op="norm", B=1, T=14566, D=3072, post="rms", pre="rms", affine=True, mod=True,
             gate=True, res_scale=1.0, dtype="bf16"),
        # Which key blocks each query block of a 1024 x 1024 image attends to, ragged samples.
        dict(name="select_image", op="select", B=4, H=16, Tq=4096, Tk=4096, d=72, keep=13, last=0, ragged=True,
             dtype="bf16"),
        # The same for the video model's joint sequence; the text blocks at its end always.
        dict(name="select_video", op="select", B=1, H=24, Tq=14566, Tk=14566, d=128, keep=46, last=5, ragged=False,
             dtype="bf16"),
        # One query per head against a long context's selected blocks: few rows, a long axis.
        dict(name="sparse_one_query", op="sparse", B=1, H=16, Tq=1, Tk=65536, d=64, keep=128, prescaled=False,
             ragged=False, holes=False, dtype="bf16"),
        # The video model's joint attention over a fifth of its key blocks.
        dict(name="sparse_video", op="sparse", B=1, H=24, Tq=14566, Tk=14566, d=128, keep=46, prescaled=True,
             ragged=False, holes=False, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["cache_rw", "forecast", "norm", "norm", "select", "sparse", "sparse"])
    if op == "cache_rw":
        return dict(op=op, n=_log(rng, 100, 44_000_000), dtype=rng.choice(["bf16", "bf16", "f32"]),
                    bits=rng.choice([8, 4]), out=rng.choice(["bf16", "f32"]))
    if op == "forecast":
        K = rng.randint(1, 8)
        return dict(op=op, K=K, n=_log(rng, 1000, 400_000_000 // K), dtype=rng.choice(["bf16", "bf16", "f32"]),
                    bits=rng.choice([8, 4]), out=rng.choice(["bf16", "bf16", "f32"]))
    if op == "norm":
        D = rng.choice([16 * rng.randint(4, 256), 4 * rng.randint(16, 900), rng.randint(30, 2000)])
        T = _log(rng, 1, 8192)
        post, pre = rng.choice(["none", "rms", "layer"]), rng.choice(["none", "rms", "layer", "layer"])
        return dict(op=op, B=max(1, min(8, 20_000_000 // (T * D), rng.randint(1, 8))), T=T, D=D, post=post, pre=pre,
                    affine=rng.random() < 0.5, mod=rng.random() < 0.7, gate=rng.random() < 0.8,
                    res_scale=rng.choice([1.0, 1.0, 0.5, 1.25]), dtype=rng.choice(["bf16", "bf16", "f32"]))
    f32 = rng.random() < 0.15
    d = rng.choice([32, 64] if f32 else [32, 64, 72, 128])
    B, H = rng.randint(1, 3), rng.randint(2, 16)
    if op == "select":
        Tk = _log(rng, 40, 12000)
        return dict(op=op, B=B, H=H, Tq=Tk if rng.random() < 0.6 else _log(rng, 1, 12000), Tk=Tk, d=d,
                    keep=rng.randint(2, 60), last=rng.randint(0, 2), ragged=rng.random() < 0.5,
                    dtype="f32" if f32 else "bf16")
    Tq = _log(rng, 1, 1000 if f32 else 8192)
    Tk = Tq if rng.random() < 0.5 and Tq > 64 else _log(rng, 40, 4000 if f32 else 30000)
    nqb = -(-Tq // QB)
    most = max(2, min(64, 300_000_000 // (B * H * nqb * KB * d)))     # what the plain form gathers
    return dict(op=op, B=B, H=H, Tq=Tq, Tk=Tk, d=d, keep=max(1, min(most, -(-Tk // KB), _log(rng, 2, 64))),
                prescaled=not f32 and rng.random() < 0.5, ragged=rng.random() < 0.5, holes=rng.random() < 0.5,
                dtype="f32" if f32 else "bf16")


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _dt(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _randn(g, shape, scale=1.0, dtype=torch.float32):
    return torch.empty(shape, device=DEV, dtype=torch.float32).normal_(0.0, scale, generator=g).to(dtype)


def _features(g, K, n, dtype):
    """K successive features of a run, newest first: a common part that drifts, and channels of unequal size."""
    size = torch.exp(_randn(g, (min(n, 1152),), 0.7))
    size = size.repeat(-(-n // size.numel()))[:n]
    base = _randn(g, (n,)) * size
    drift = _randn(g, (n,), 0.1) * size
    out = torch.empty((K, n), device=DEV, dtype=dtype)
    for j in range(K):
        out[j] = (base - float(j) * drift).to(dtype)
    return out


def _weights(K):
    """Weights that add up to one, of both signs, as extrapolating ones are."""
    w = [(-1.0) ** j * (1.0 + 0.25 * (K - j)) for j in range(K)]
    s = sum(w)
    return [x / s for x in w]


def _lens(g, case):
    if not case["ragged"]:
        return None
    lens = torch.randint(max(1, case["Tk"] // 3), case["Tk"] + 1, (case["B"],), generator=g, device=DEV)
    return lens.to(torch.int32)


def _blocks(case, g, lens):
    """For every query block an ascending list of `keep` key blocks, near ones favoured; -1 behind a shorter list."""
    B, H, keep = case["B"], case["H"], case["keep"]
    nq, nk = -(-case["Tq"] // QB), -(-case["Tk"] // KB)
    at = torch.arange(nq, device=DEV)[:, None] * (float(nk) / nq)
    near = torch.exp(-(torch.arange(nk, device=DEV)[None, :] - at).abs() / 4.0)
    score = torch.rand((B, H, nq, nk), device=DEV, generator=g) + near
    if lens is not None:
        valid = torch.arange(nk, device=DEV) * KB < lens[:, None]
        score = score.masked_fill(~valid[:, None, None, :], -1.0)
    best = torch.topk(score, min(keep, nk), dim=-1)
    idx = torch.where(best.values >= 0, best.indices, nk)
    if case["holes"]:
        short = torch.arange(B * H * nq, device=DEV).reshape(B, H, nq, 1) % 5
        rank = torch.arange(idx.shape[-1], device=DEV)
        idx = torch.where((short == 1) & (rank >= idx.shape[-1] // 2) | (short == 3), nk, idx)
    idx = torch.sort(idx, dim=-1).values
    idx = torch.where(idx < nk, idx, -1)
    full = torch.full((B, H, nq, keep), -1, dtype=torch.int32, device=DEV)
    full[..., :idx.shape[-1]] = idx.to(torch.int32)
    return full


def _inputs(case, seed):
    g, op = _gen(seed), case["op"]
    if op == "cache_rw":
        return dict(feat=_features(g, 1, case["n"], _dt(case["dtype"]))[0])
    if op == "forecast":
        return dict(feats=_features(g, case["K"], case["n"], _dt(case["dtype"])), w=_weights(case["K"]))
    dt = _dt(case["dtype"])
    if op == "norm":
        B, T, D = case["B"], case["T"], case["D"]
        mods = _randn(g, (B, 3 * D), 0.3)      # gate, shift and scale rows of one modulation vector
        s = dict(y=_randn(g, (B * T, D), 0.7, dt), x=_randn(g, (B * T, D), 2.0) + _randn(g, (1, D)),
                 gate=mods[:, :D] if case["gate"] else None, shift=mods[:, D:2 * D] if case["mod"] else None,
                 scale=mods[:, 2 * D:] if case["mod"] else None)
        for side in ("post", "pre"):
            a = case["affine"] and case[side] != "none"
            s[side + "_w"] = (1.0 + _randn(g, (D,), 0.1)).to(dt) if a else None
            s[side + "_b"] = _randn(g, (D,), 0.1, dt) if a and case[side] == "layer" else None
        return s
    B, H, Tq, Tk, d = (case[k] for k in ("B", "H", "Tq", "Tk", "d"))
    s = dict(lens=_lens(g, case))
    # Tokens near each other look alike: a part common to 32 neighbours.
    q = _randn(g, (B, Tq, H, d)) + _randn(g, (B, -(-Tq // 32), H, d), 0.7).repeat_interleave(32, 1)[:, :Tq]
    s["k"] = (_randn(g, (B, Tk, H, d)) + _randn(g, (B, -(-Tk // 32), H, d), 0.7).repeat_interleave(32, 1)[:, :Tk]).to(dt)
    if op == "sparse":
        if case["prescaled"]:
            q = q * (math.log2(math.e) / math.sqrt(d))
        s["v"] = _randn(g, (B, Tk, H, d), 1.0, dt)
        s["idx"] = _blocks(case, g, s["lens"])
    s["q"] = q.to(dt)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    op = case["op"]
    if op in ("cache_rw", "forecast"):
        s["out"] = torch.empty(case["n"], device=DEV, dtype=_dt(case["out"]))
        K = case.get("K", 1)
        if own:
            import paper_2608_28670_amd as bc
            store = torch.empty(bc.quant_cache_bytes(K, case["n"], case["bits"]), dtype=torch.uint8, device=DEV)
            s["ring"] = bc.QuantCacheRing(K, case["n"], _dt(case["dtype"]), case["bits"], store)
            if op == "forecast":
                for j in reversed(range(K)):
                    s["ring"].push(s["feats"][j], float(-j))
        if not own:
            if op == "forecast":
                s["codes"] = [_quantise(f, case["bits"]) for f in s["feats"]]
        s.pop("feats", None)
    elif op == "norm":
        s["x_out"] = torch.empty_like(s["x"])
        s["h"] = torch.empty_like(s["y"]) if case["pre"] != "none" or case["mod"] else None
    else:
        if op == "select":
            s["idx"] = torch.empty((case["B"], case["H"], -(-case["Tq"] // QB), case["keep"]), dtype=torch.int32, device=DEV)
        else:
            s["out"] = torch.empty_like(s["q"])
        if own:
            import paper_2608_28670_amd as bc
            size = bc.attention_select_workspace_size if op == "select" else bc.attention_sparse_workspace_size
            n = size(case["B"], case["H"], case["Tq"], case["Tk"], case["d"], case["keep"], bc.dtype_code(s["q"]))
            s["ws"] = torch.empty(max(n, 256), dtype=torch.uint8, device=DEV)
    return s


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def _quantise(x, bits):
    """(codes, scales) of a flat feature.  The quotients in 64 bits: half-way ones must not move."""
    top = 127 if bits == 8 else 7
    n = x.numel()
    g = torch.nn.functional.pad(x.float(), (0, -n % GROUP)).reshape(-1, GROUP).double()
    s = (g.abs().amax(1, keepdim=True) / top).float()
    s = torch.where(s < 2.0 ** -120, 0.0, s)
    q = torch.round(g / torch.where(s > 0, s, 1.0).double()) * (s > 0)
    return q.to(torch.int8), s


def _dequantise(codes, n):
    q, s = codes
    return (q.float() * s).reshape(-1)[:n]


def _norm(v, kind, w, b, eps=1e-6):
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
    if kind != "none":
        v = v / torch.sqrt((v * v).mean(-1, keepdim=True) + eps)
    if w is not None:
        v = v * w.float()
    return v if b is None else v + b.float()


def _rows(t, case):
    """A per-sample row for every token's row."""
    return t.repeat_interleave(case["T"], 0)


def _pad_blocks(t, size):
    """[B, T, H, d] -> [B, H, blocks, size, d], zeros behind the end."""
    t = torch.nn.functional.pad(t, (0, 0, 0, 0, 0, -t.shape[1] % size))
    return t.reshape(t.shape[0], -1, size, t.shape[2], t.shape[3]).permute(0, 3, 1, 2, 4)


def _valid(case, lens):
    """[B, key blocks, KB]: which keys there are."""
    nk = -(-case["Tk"] // KB)
    pos = torch.arange(nk * KB, device=DEV).reshape(1, nk, KB)
    if lens is None:
        return (pos < case["Tk"]).expand(case["B"], nk, KB)
    return pos < lens.long().clamp(0, case["Tk"])[:, None, None]


def run(s):
    case = s["case"]
    op = case["op"]
    if own:
        import paper_2608_28670_amd as bc
        if op == "cache_rw":
            s["ring"].push(s["feat"], 0.0)
            s["ring"].read(0, s["out"])
            return s["out"]
        if op == "forecast":
            bc.bary_extrapolate(s["ring"], s["w"], s["out"])
            return s["out"]
        if op == "norm":
            kinds = {"none": bc.NORM_NONE, "rms": bc.NORM_RMS, "layer": bc.NORM_LAYER}
            bc.norm_gate_residual(s["y"], s["x"], s["x_out"], s["h"], rows_per_sample=case["T"], post=kinds[case["post"]],
                                  post_w=s["post_w"], post_b=s["post_b"], gate=s["gate"], res_scale=case["res_scale"],
                                  pre=kinds[case["pre"]], pre_w=s["pre_w"], pre_b=s["pre_b"], shift=s["shift"],
                                  scale=s["scale"])
            return {"x": s["x_out"]} if s["h"] is None else {"x": s["x_out"], "h": s["h"]}
        if op == "select":
            bc.attention_select(s["q"], s["k"], s["idx"], lens=s["lens"], keep_last=case["last"], ws=s["ws"])
            return s["idx"]
        bc.attention_sparse(s["q"], s["k"], s["v"], s["idx"], s["out"], lens=s["lens"], ws=s["ws"],
                            prescaled=case["prescaled"])
        return s["out"]
    if op == "cache_rw":
        return s["out"].copy_(_dequantise(_quantise(s["feat"], case["bits"]), case["n"]))
    if op == "forecast":
        return s["out"].copy_(sum(w * _dequantise(c, case["n"]) for w, c in zip(s["w"], s["codes"])))
    if op == "norm":
        z = _norm(s["y"].float(), case["post"], s["post_w"], s["post_b"])
        if s["gate"] is not None:
            z = z * _rows(s["gate"], case)
        x = case["res_scale"] * s["x"] + z
        if s["h"] is None:
            return {"x": s["x_out"].copy_(x)}
        h = _norm(x, case["pre"], s["pre_w"], s["pre_b"])
        if s["scale"] is not None:
            h = h * (1.0 + _rows(s["scale"], case)) + _rows(s["shift"], case)
        return {"x": s["x_out"].copy_(x), "h": s["h"].copy_(h)}
    valid = _valid(case, s["lens"])
    if op == "select":
        # In 64 bits: which of two blocks with nearly the same score is taken must not hang on a rounding.
        qb, kb = _pad_blocks(s["q"], QB).double(), _pad_blocks(s["k"], KB).double()
        cq = torch.full((qb.shape[2],), QB, device=DEV, dtype=torch.float64)
        cq[-1] = case["Tq"] - QB * (qb.shape[2] - 1)
        ck = valid.sum(-1)
        kb = torch.where(valid[:, None, :, :, None], kb, 0.0)
        qm, km = qb.sum(3) / cq[:, None], kb.sum(3) / ck.clamp(min=1)[:, None, :, None]
        score = torch.matmul(qm, km.transpose(2, 3).contiguous())
        there = (ck > 0)[:, None, None, :]
        nb = (ck > 0).sum(-1)[:, None, None, None]
        j = torch.arange(score.shape[-1], device=DEV)
        score = torch.where(j >= nb - case["last"], math.inf, score)
        score = torch.where(there, score, -math.inf)
        best = torch.sort(score, dim=-1, descending=True, stable=True)
        idx = torch.where(torch.isneginf(best.values), score.shape[-1], best.indices)[..., :case["keep"]]
        idx = torch.sort(idx, dim=-1).values
        s["idx"].fill_(-1)
        s["idx"][..., :idx.shape[-1]] = torch.where(idx < score.shape[-1], idx, -1).to(torch.int32)
        return s["idx"]
    # Gathers every query block's keys and values and attends to them.
    B, H, d, keep = case["B"], case["H"], case["d"], case["keep"]
    idx = s["idx"].long()
    some = idx >= 0
    at = idx.clamp(min=0)
    bi, hi = torch.arange(B, device=DEV)[:, None, None, None], torch.arange(H, device=DEV)[None, :, None, None]
    qb = _pad_blocks(s["q"], QB).float()
    kb, vb = _pad_blocks(s["k"], KB), _pad_blocks(s["v"], KB)
    ok = (valid[bi, at] & some[..., None]).flatten(3)
    kg = kb[bi, hi, at].flatten(3, 4).float()
    unit = math.log(2.0) if case["prescaled"] else 1.0 / math.sqrt(d)
    sc = torch.matmul(qb, kg.transpose(-1, -2).contiguous()) * unit
    del kg
    sc = sc.masked_fill(~ok[..., None, :], -math.inf)
    top = sc.amax(-1, keepdim=True)
    p = torch.exp(sc - torch.where(torch.isneginf(top), 0.0, top))
    del sc
    den = p.sum(-1, keepdim=True)
    vg = torch.where(ok[..., None], vb[bi, hi, at].flatten(3, 4), 0.0).float()
    o = torch.matmul(p, vg) / torch.where(den > 0, den, 1.0)
    o = o.permute(0, 2, 3, 1, 4).reshape(B, -1, H, d)[:, :case["Tq"]]
    return s["out"].copy_(o)


# ---------------------------------------------------------------------------
# What a pass cannot do without, and what it should give
# ---------------------------------------------------------------------------
def work(case):
    op, e = case["op"], 2 if case["dtype"] == "bf16" else 4
    if op in ("cache_rw", "forecast"):
        n, eo = case["n"], 2 if case["out"] == "bf16" else 4
        slot = n * case["bits"] / 8 + 4 * -(-n // GROUP)
        if op == "cache_rw":
            return {"bytes": float(n * (e + eo) + 2 * slot), "flops": 4.0 * n}
        return {"bytes": float(case["K"] * slot + n * eo), "flops": 2.0 * case["K"] * n}
    if op == "norm":
        h = case["pre"] != "none" or case["mod"]
        n = case["B"] * case["T"] * case["D"]
        return {"bytes": float(n * (e + 8 + (e if h else 0)) + case["B"] * case["D"] * 4 * (case["gate"] + 2 * case["mod"])),
                "flops": 14.0 * n}
    B, H, Tq, Tk, d, keep = (case[k] for k in ("B", "H", "Tq", "Tk", "d", "keep"))
    nq, nk = -(-Tq // QB), -(-Tk // KB)
    if op == "select":
        return {"bytes": float(B * H * (d * (Tq + Tk) * e + nq * keep * 4)),
                "flops": float(B * H * d * (Tq + Tk + 2 * nq * nk))}
    some = min(keep, nk) * (0.7 if case["holes"] else 1.0)
    seen = min(nk, nq * some)
    return {"bytes": float(B * H * (d * (2 * Tq + 2 * min(Tk, seen * KB)) * e + nq * keep * 4)),
            "flops": 4.0 * B * H * Tq * min(Tk, some * KB) * d}


def _exact_codes(x, bits):
    """A feature's held values in 64 bits, group by group of the flat order."""
    top = 127.0 if bits == 8 else 7.0
    n = x.numel()
    full = torch.zeros(-(-n // GROUP) * GROUP, dtype=torch.float64, device=x.device)
    full[:n] = x.double()
    full = full.view(-1, GROUP)
    scale = (full.abs().max(1).values / top).to(torch.float32).double()
    scale[scale < 2.0 ** -120] = 0.0
    ratio = full / scale.clamp(min=2.0 ** -140)[:, None]
    ratio[scale == 0] = 0.0
    return (torch.round(ratio) * scale[:, None]).view(-1)[:n]


def exact(case, seed):
    s, op = _inputs(case, seed), case["op"]
    if op == "cache_rw":
        return _exact_codes(s["feat"], case["bits"])
    if op == "forecast":
        out = torch.zeros(case["n"], dtype=torch.float64, device=DEV)
        for j, w in enumerate(s["w"]):
            out += w * _exact_codes(s["feats"][j], case["bits"])
        return out
    if op == "norm":
        B, T, D = case["B"], case["T"], case["D"]
        y, x = (s[k].double().view(B, T, D) for k in ("y", "x"))

        def normed(v, side):
            if case[side] == "layer":
                var, mean = torch.var_mean(v, dim=2, unbiased=False, keepdim=True)
                v = (v - mean) * (var + 1e-6) ** -0.5
            elif case[side] == "rms":
                v = v * (v.square().sum(2, keepdim=True) / D + 1e-6) ** -0.5
            if s[side + "_w"] is not None:
                v = v * s[side + "_w"].double()
            if s[side + "_b"] is not None:
                v = v + s[side + "_b"].double()
            return v

        z = normed(y, "post")
        x2 = case["res_scale"] * x + (z if s["gate"] is None else s["gate"].double()[:, None] * z)
        if case["pre"] == "none" and not case["mod"]:
            return {"x": x2.view(B * T, D)}
        h = normed(x2, "pre")
        if case["mod"]:
            h = h + h * s["scale"].double()[:, None] + s["shift"].double()[:, None]
        return {"x": x2.view(B * T, D), "h": h.view(B * T, D)}
    if op == "select":
        return None
    # Dense attention of one head at a time under a mask of its blocks.
    B, H, Tq, Tk, d = (case[k] for k in ("B", "H", "Tq", "Tk", "d"))
    out = torch.zeros((B, Tq, H, d), dtype=torch.float64, device=DEV)
    key_block = torch.arange(Tk, device=DEV) // KB
    query_block = torch.arange(Tq, device=DEV) // QB
    for b in range(B):
        n = Tk if s["lens"] is None else int(s["lens"][b])
        for h in range(H):
            idx = s["idx"][b, h].long()
            table = torch.zeros((idx.shape[0], -(-Tk // KB) + 1), dtype=torch.bool, device=DEV)
            table.scatter_(1, torch.where(idx < 0, table.shape[1] - 1, idx), True)
            seen = table[query_block][:, key_block]
            seen[:, n:] = False
            sc = s["q"][b, :, h].double() @ s["k"][b, :, h].double().t()
            sc *= math.log(2.0) if case["prescaled"] else d ** -0.5
            p = torch.softmax(sc.masked_fill_(~seen, -math.inf), -1)
            out[b, :, h] = torch.nan_to_num(p, nan=0.0) @ s["v"][b, :, h].double()
    return out
