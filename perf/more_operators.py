"""Operators for samples made piece by piece: rotary positions, attention with masks, caps and distance biases, and a
key-value cache in 8 bits with the attention that reads it.

Each case is one operator as a sampling program calls it.  Queries and keys are turned by their positions (a frame, row
and column each, or one running number, with frequencies scaled for long contexts); attention runs over packed samples,
over the frames before a frame, over a prefix; the keys and values of finished pieces are held in 8 bits, one power of
two as scale for each 64 tokens of a head, and the queries of the next piece, or of one token, attend to them.
"""
import math

import torch

own = False   # True: the framework's calls, False: the same in elementary operations

DEV = "cuda:0"
KB = 64       # tokens of a cache block, which share a scale


def _attn(name, op, B, Hq, Hk, Tq, Tk, d, dtype="bf16", cap=0.0, slopes=False, causal=False, window=0, prefix=False,
          ragged=False, docs=0):
    c = dict(op=op, B=B, Hq=Hq, Hk=Hk, Tq=Tq, Tk=Tk, d=d, dtype=dtype, cap=cap, slopes=slopes, causal=causal,
             window=window, prefix=prefix, ragged=ragged, docs=docs)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # One token's queries and keys at a far position: launch latency.
        dict(name="rope_one_token", op="rope", B=1, T=1, Hq=16, Hk=16, d=72, rot=72, axes=1, layout="pairs",
             scaling="linear", far=100_000, strided=False, dtype="bf16"),
        # The video model's image tokens, (frame, row, column) positions, in place among the projection's rows.
        dict(name="rope_video", op="rope", B=1, T=14310, Hq=24, Hk=24, d=128, rot=128, axes=3, layout="pairs",
             scaling="parts", far=0, strided=True, dtype="bf16"),
        # Part of each head in two halves, few heads, an odd number of tokens, fp32.
        dict(name="rope_partial_f32", op="rope", B=3, T=1021, Hq=10, Hk=5, d=64, rot=48, axes=1, layout="halves",
             scaling="ntk", far=5000, strided=False, dtype="f32"),
        # One query per head over an uncompressed context, scores capped, nearer keys favoured: few rows, a long axis.
        _attn("masked_one_query", "masked", 4, 32, 8, 1, 8192, 128, cap=30.0, slopes=True),
        # Images of many sizes packed into one sequence: each token sees its own image only.
        _attn("masked_packed_images", "masked", 1, 16, 16, 16384, 16384, 72, docs=24),
        # The video model's joint sequence with frames in order, capped scores: the largest call.
        _attn("masked_video_causal", "masked", 1, 24, 24, 14566, 14566, 128, cap=50.0, causal=True),
        # A padded fp32 batch: a prefix seen by all, then a sliding window; an odd number of tokens.
        _attn("masked_prefix_f32", "masked", 2, 6, 6, 777, 777, 64, dtype="f32", causal=True, window=200, prefix=True,
              ragged=True),
        # One token's keys and values into the cache and back: latency.
        dict(name="kv_push_one", op="push", B=8, H=8, d=128, held=1000, T=1, ragged=True, dtype="bf16"),
        # A whole video's keys and values into the cache and back.
        dict(name="kv_push_video", op="push", B=1, H=24, d=128, held=0, T=14310, ragged=False, dtype="bf16"),
        # One token of a small fp32 model over a short cache.
        _attn("kv_one_query_tiny", "cached", 2, 4, 4, 1, 300, 32, dtype="f32"),
        # One token per sample over long caches, four query heads a key head: the cache's bytes.
        _attn("kv_one_query_long", "cached", 4, 32, 8, 1, 65536, 128, causal=True, ragged=True),
        # The next latent frame's queries over the frames before it and its own.
        _attn("kv_next_frame", "cached", 1, 24, 24, 1590, 14310, 128),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "rope", "masked", "masked", "masked", "push", "cached", "cached", "cached"])
    f32 = rng.random() < 0.25
    dtype = "f32" if f32 else "bf16"
    if op == "rope":
        d = rng.choice([32, 64, 72, 96, 128, 2 * rng.randint(10, 64)])
        Hk = rng.randint(1, 12)
        rot = d if rng.random() < 0.6 else 2 * rng.randint(2, d // 2)
        axes = rng.choice([1, 1, 2, 3]) if rot >= 12 else 1
        return dict(op=op, B=rng.randint(1, 4), T=_log(rng, 1, 8192), Hq=Hk * rng.choice([1, 1, 2, 4]), Hk=Hk, d=d, rot=rot,
                    axes=axes, layout=rng.choice(["pairs", "halves"]), scaling=rng.choice(["none", "linear", "ntk", "parts"]),
                    far=rng.choice([0, 0, _log(rng, 100, 1_000_000)]), strided=rng.random() < 0.5, dtype=dtype)
    d = rng.choice([32, 64, 72, 128])
    if op == "push":
        B, H = rng.randint(1, 8), rng.randint(1, 24)
        return dict(op=op, B=B, H=H, d=d, held=rng.choice([0, _log(rng, 1, 3000)]),
                    T=_log(rng, 1, max(1, min(16384, 40_000_000 // (B * H * d)))), ragged=rng.random() < 0.5, dtype=dtype)
    B, Hk, G = rng.randint(1, 4), rng.randint(1, 12), rng.choice([1, 1, 1, 2, 4, 8])
    if op == "masked":
        Tq = _log(rng, 1, 1500 if f32 else 8192)
        Tk = Tq if Tq > 16 and rng.random() < 0.6 else _log(rng, 16, 4000 if f32 else 16384)
    else:
        Tk = _log(rng, 16, 8000 if f32 else 65536)
        Tq = min(Tk, rng.choice([1, 1, 2, 4, _log(rng, 5, 1000 if f32 else 4096)]))
    while B * Hk * G * Tq * Tk > 2_000_000_000 or B * Hk * Tk * d > 300_000_000:
        if B > 1:
            B -= 1
        elif Hk > 1:
            Hk = (Hk + 1) // 2
        else:
            Tq = max(1, Tq // 2)
    same = Tq == Tk
    ragged = rng.random() < 0.4
    window = _log(rng, 1, Tk) if rng.random() < 0.3 and (same or op == "cached" or not ragged) else 0   # (else: few see a key)
    return _attn(None, op, B, Hk * G, Hk, Tq, Tk, d, dtype=dtype, cap=rng.choice([0.0, 0.0, 20.0, 50.0]), slopes=rng.random() < 0.3,
                 causal=rng.random() < 0.5, window=window, prefix=rng.random() < 0.3, ragged=ragged,
                 docs=rng.randint(2, 1 + max(1, Tq // 40)) if op == "masked" and same and rng.random() < 0.5 else 0)


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


def _ints(g, lo, hi, n):
    """n integers from lo to hi."""
    return torch.randint(lo, hi + 1, (n,), generator=g, device=DEV)


def _keys(g, shape, dtype):
    """Keys or values: channels of unequal size, tokens near each other alike."""
    B, T, H, d = shape
    size = torch.exp(_randn(g, (1, 1, H, d), 0.5))
    x = _randn(g, shape)
    x += _randn(g, (B, -(-T // 32), H, d), 0.7).repeat_interleave(32, 1)[:, :T]
    return x.mul_(size).to(dtype)


def _axis_dims(case):
    """Widths of the rotated part's axes: the last ones equal, the first takes what is left."""
    n, rot = case["axes"], case["rot"]
    each = rot // n // 2 * 2 if n < 3 else 2 * (7 * rot // 32)
    return [rot - (n - 1) * each] + [each] * (n - 1)


def _positions(case, g):
    """int32 [B, T, axes]."""
    B, T, n = case["B"], case["T"], case["axes"]
    t = torch.arange(T, device=DEV)
    if n == 1:
        at = t[:, None]
    else:
        w = max(1, int(math.sqrt(T / 3.0)))
        at = torch.stack([t // w, t % w] if n == 2 else [t // (w * w), t // w % w, t % w], -1)
    first = _ints(g, case["far"] // 2, case["far"], B)
    at = at[None].repeat(B, 1, 1)
    at[..., 0] += first[:, None]
    return at.to(torch.int32).contiguous()


def _lens(g, case, n):
    """Tokens that a sample has: up to n."""
    if not case["ragged"]:
        return torch.full((case["B"],), n, dtype=torch.int32, device=DEV)
    return _ints(g, max(1, n // 3), n, case["B"]).to(torch.int32)


def _documents(g, case):
    """int32 [B, T]: which document a token belongs to, in order; -1 for the padding behind the last."""
    B, T, n = case["B"], case["Tq"], case["docs"]
    cuts = torch.sort(torch.randint(0, T, (B, n), generator=g, device=DEV), -1).values
    doc = (torch.arange(T, device=DEV)[None, :, None] >= cuts[:, None, :]).sum(-1)
    end = _ints(g, T - T // 16, T, B)
    return torch.where(torch.arange(T, device=DEV) < end[:, None], doc, -1).to(torch.int32)


def _inputs(case, seed):
    g, op, dt = _gen(seed), case["op"], _dt(case["dtype"])
    B = case["B"]
    if op == "rope":
        T, Hq, Hk, d = case["T"], case["Hq"], case["Hk"], case["d"]
        if case["strided"]:      # rows of a projection: [q | k | v]
            qkv = _randn(g, (B, T, Hq + 2 * Hk, d), 1.0, dt)
            q, k = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hk]
        else:
            q, k = _randn(g, (B, T, Hq, d), 1.0, dt), _randn(g, (B, T, Hk, d), 1.0, dt)
        return dict(q=q, k=k, pos=_positions(case, g))
    if op == "push":
        held = _lens(g, case, case["held"]) if case["held"] else torch.zeros(B, dtype=torch.int32, device=DEV)
        counts = _lens(g, case, case["T"])
        shape = lambda n: (B, n, case["H"], case["d"])   # noqa: E731
        s = dict(held=held, counts=counts, k=_keys(g, shape(case["T"]), dt), v=_keys(g, shape(case["T"]), dt))
        if case["held"]:
            s["k0"], s["v0"] = _keys(g, shape(case["held"]), dt), _keys(g, shape(case["held"]), dt)
            s["k0"] *= 0.5      # the later tokens enlarge their block's scale
        return s
    Hq, Hk, Tq, Tk, d = (case[k] for k in ("Hq", "Hk", "Tq", "Tk", "d"))
    s = dict(k=_keys(g, (B, Tk, Hk, d), dt), v=_keys(g, (B, Tk, Hk, d), dt), q=_randn(g, (B, Tq, Hq, d), 1.3, dt))
    s["lens"] = _lens(g, case, Tk) if op == "cached" or case["ragged"] else None
    s["counts"] = torch.minimum(_lens(g, case, Tq), s["lens"]) if op == "cached" and case["ragged"] else None
    s["prefix"] = _ints(g, 0, Tk // 3, B).to(torch.int32) if case["prefix"] else None
    # Slopes that halve from head to head over a factor of 256.
    s["slopes"] = 2.0 ** (-8.0 * torch.arange(1, Hq + 1, device=DEV, dtype=torch.float32) / Hq) if case["slopes"] else None
    s["docs"] = _documents(g, case) if case["docs"] else None
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    op = case["op"]
    if op == "rope":
        s["q_out"], s["k_out"] = torch.empty_like(s["q"].contiguous()), torch.empty_like(s["k"].contiguous())
        s["freqs"] = _frequencies(case)
        if own:
            import paper_2608_28670_amd as bc
            s["freqs"] = [f for i, n in enumerate(_axis_dims(case)) for f in bc.rope_frequencies(n, **_rope_scaling(case, i))]
        return s
    if op == "push":
        s["lens"] = s["held"] + s["counts"]
        n = case["held"] + case["T"]
        for x in ("k_out", "v_out"):
            s[x] = torch.empty((case["B"], n, case["H"], case["d"]), dtype=_dt(case["dtype"]), device=DEV)
        if own:
            import paper_2608_28670_amd as bc
            s["cache"] = _own_cache(bc, case["B"], case["H"], case["d"], n)
            if case["held"]:
                s["cache"].push(s["k0"], s["v0"], s["held"], counts=s["held"])
        elif case["held"]:
            for x in ("k", "v"):
                s[x + "_held"] = _quantise(_blocks(s[x + "0"], s["held"], torch.zeros_like(s["held"]), n))
        s.pop("k0", None)
        s.pop("v0", None)
        return s
    s["out"] = torch.empty_like(s["q"])
    if own:
        import paper_2608_28670_amd as bc
    if op == "cached":
        if own:
            s["cache"] = _own_cache(bc, case["B"], case["Hk"], case["d"], case["Tk"])
            s["cache"].push(s["k"], s["v"], s["lens"], counts=s["lens"])
            n = s["cache"].attention_workspace_size(case["Hq"], case["Tq"], bc.dtype_code(s["q"]))
        else:
            for x in ("k", "v"):
                codes, scale = _quantise(_blocks(s[x], s["lens"], torch.zeros_like(s["lens"]), case["Tk"]))
                s[x + "_held"] = codes.to(torch.float8_e4m3fn), scale
        s["k"] = s["v"] = None
    elif own:
        n = bc.attention_masked_workspace_size(case["B"], case["Hq"], case["Hk"], case["Tq"], case["Tk"], case["d"],
                                               bc.dtype_code(s["q"]))
    if own:
        s["ws"] = torch.empty(max(n, 256), dtype=torch.uint8, device=DEV)
    return s


def _own_cache(bc, B, H, d, n):
    store = torch.empty(bc.kv_cache_bytes(B, H, d, n), dtype=torch.uint8, device=DEV)
    return bc.KVCache(B, H, d, n, store)


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def _rope_scaling(case, axis):
    """Contexts four times as long as the original one; the first axis alone is scaled where there are several."""
    kind = case["scaling"] if axis == 0 else "none"
    return dict(theta=256.0 if case["axes"] == 3 else 10000.0, scaling=kind, factor=4.0, original=2048)


def _frequencies(case):
    """Radians per position of every rotated pair, axis after axis, in 64 bits."""
    out = []
    for axis, n in enumerate(_axis_dims(case)):
        c = _rope_scaling(case, axis)
        theta = c["theta"] * (c["factor"] ** (n / (n - 2.0)) if c["scaling"] == "ntk" and n > 2 else 1.0)
        f = torch.tensor(theta, dtype=torch.float64) ** (-2.0 * torch.arange(n // 2, dtype=torch.float64) / n)
        if c["scaling"] == "linear":
            f = f / c["factor"]
        if c["scaling"] == "parts":      # pairs that turn often keep their frequency, slow ones are stretched
            turns = c["original"] * f / (2.0 * math.pi)
            ramp = ((turns - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)
            f = f * (ramp + (1.0 - ramp) / c["factor"])
        out.append(f)
    return torch.cat(out).to(DEV)


def _turn(x, ang, case, amplitude):
    """The rotated part of each head turned; ang [B, T, rot / 2], pairs axis after axis."""
    rot, halves = case["rot"], case["layout"] == "halves"
    c, s = (torch.cos(ang) * amplitude).float()[:, :, None], (torch.sin(ang) * amplitude).float()[:, :, None]
    out = x.float().clone()
    first = torch.arange(rot // 2, device=DEV) * 2
    second = first + 1
    if halves:
        base = torch.cat([torch.arange(n // 2, device=DEV) + sum(_axis_dims(case)[:i]) for i, n in enumerate(_axis_dims(case))])
        half = torch.cat([torch.full((n // 2,), n // 2, device=DEV) for n in _axis_dims(case)])
        first, second = base, base + half
    a, b = x[..., first].float(), x[..., second].float()
    out[..., first] = a * c - b * s
    out[..., second] = a * s + b * c
    return out


def _amplitude(case):
    return 0.1 * math.log(4.0) + 1.0 if case["scaling"] == "parts" else 1.0


def _axis_of_pairs(case):
    return torch.repeat_interleave(torch.arange(case["axes"], device=DEV), torch.tensor(_axis_dims(case), device=DEV) // 2)


def _blocks(x, counts, first, n):
    """[B, T, H, d] tokens laid at positions first.. of a cache of n tokens: [B, blocks, 64, H, d] fp32; NaN where none is."""
    B, T = x.shape[:2]
    nb = -(-n // KB)
    t = torch.arange(nb * KB, device=DEV)[None, :] - first.long()[:, None]
    there = (t >= 0) & (t < counts[:, None])
    rows = x[torch.arange(B, device=DEV)[:, None], t.clamp(0, T - 1)].float()
    return torch.where(there[:, :, None, None], rows, math.nan).reshape(B, nb, KB, *x.shape[2:])


def _pow2(e):
    """2^e, exactly."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _scale(x):
    """The least power of two from 2^-100 up with which a block's largest magnitude is at most 448: [B, blocks, 1, H, 1]."""
    m, e = torch.frexp(torch.nan_to_num(x, nan=0.0).abs().amax((2, 4), keepdim=True))
    return _pow2(torch.where(m > 0, e - 9 + (m > 0.875), -100).clamp(min=-100))


def _round8(y):
    """To the nearest value with four significant bits from 2^-6 up, a multiple of 2^-9 below; ties to even."""
    step = _pow2((torch.frexp(y).exponent - 1).clamp(min=-6) - 3)
    return torch.round(y / step) * step


def _quantise(x, least=None):
    """(codes as values, scales) of blocks; tokens that are not there are zeros."""
    s = _scale(x) if least is None else torch.maximum(_scale(x), least)
    return _round8(torch.nan_to_num(x, nan=0.0) / s), s


def _attend(case, q, k, v, s, key_count, query_at, rows):
    """Attention of q [B, Tq, Hq, d] over k, v [B, Tk, Hk, d] in fp32: query t stands at query_at [B, Tq], sample b has
    key_count[b] keys and rows[b] queries."""
    B, Tq, Hq, d = q.shape
    Hk, Tk = k.shape[2], k.shape[1]
    qh = q.float().permute(0, 2, 1, 3).reshape(B * Hk, (Hq // Hk) * Tq, d)
    kt = k.permute(0, 2, 3, 1).reshape(B * Hk, d, Tk).contiguous()
    sc = torch.matmul(qh, kt).view(B, Hq, Tq, Tk).mul_(1.0 / math.sqrt(d))
    if case["cap"]:
        sc.div_(case["cap"]).tanh_().mul_(case["cap"])
    j = torch.arange(Tk, device=DEV)
    dist = query_at[:, :, None] - j
    if case["slopes"]:
        sc.sub_(s["slopes"][None, :, None, None] * dist[:, None].abs())
    seen = torch.ones_like(dist, dtype=torch.bool)
    if case["causal"]:
        seen &= dist >= 0
    if case["window"]:
        seen &= dist.abs() < case["window"]
    if case["prefix"]:
        seen |= j < s["prefix"][:, None, None]
    seen &= (j < key_count[:, None, None]) & (torch.arange(Tq, device=DEV)[:, None] < rows[:, None, None])
    if case["docs"]:
        seen &= (s["docs"][:, :, None] == s["docs"][:, None, :]) & (s["docs"][:, :, None] >= 0)
    sc.masked_fill_(~seen[:, None], -math.inf)
    del seen, dist
    top = sc.amax(-1, keepdim=True)
    sc.sub_(top.masked_fill(torch.isneginf(top), 0.0)).exp_()
    den = sc.sum(-1)
    vh = v.permute(0, 2, 1, 3).reshape(B * Hk, Tk, d).contiguous()
    o = torch.matmul(sc.view(B * Hk, -1, Tk), vh).view(B, Hq, Tq, d)
    return (o / torch.where(den > 0, den, 1.0)[..., None]).permute(0, 2, 1, 3)


def run(s):
    case = s["case"]
    op, B = case["op"], case["B"]
    if op == "rope":
        if own:
            import paper_2608_28670_amd as bc
            bc.rope(s["q"], s["q_out"], s["freqs"], k=s["k"], k_out=s["k_out"], pos=s["pos"], axes=_axis_dims(case),
                    layout=case["layout"], amplitude=_amplitude(case))
            return {"q": s["q_out"], "k": s["k_out"]}
        ang = s["pos"][..., _axis_of_pairs(case)].double() * s["freqs"]
        return {x: s[x + "_out"].copy_(_turn(s[x], ang, case, _amplitude(case))) for x in ("q", "k")}
    if op == "push":
        if own:
            s["cache"].push(s["k"], s["v"], s["lens"], counts=s["counts"])
            s["cache"].read(s["k_out"], s["v_out"], s["lens"])
            return {"k": s["k_out"], "v": s["v_out"]}
        out = {}
        for x in ("k", "v"):
            n = s[x + "_out"].shape[1]
            new = _blocks(s[x], s["counts"], s["held"], n)
            if case["held"]:
                # Blocks that hold tokens already keep at least their scale, and those tokens are rounded to the new one.
                codes, scale = s[x + "_held"]
                there = torch.arange(new.shape[1], device=DEV) * KB < s["held"][:, None]
                least = torch.where(there[:, :, None, None, None], scale, 2.0 ** -100)
                now, scale = _quantise(new, least)
                held = torch.arange(new.shape[1] * KB, device=DEV).view(1, -1, KB) < s["held"][:, None, None]
                val = torch.where(held[..., None, None], _round8(codes * (least / scale)), now) * scale
            else:
                now, scale = _quantise(new)
                val = now * scale
            out[x] = s[x + "_out"].copy_(val.flatten(1, 2)[:, :n])
        return out
    if op == "cached":
        if own:
            s["cache"].attention(s["q"], s["out"], s["lens"], counts=s["counts"], cap=case["cap"], slopes=s["slopes"],
                                 causal=case["causal"], window=case["window"], prefix=s["prefix"], ws=s["ws"])
            return s["out"]
        k, v = (((s[x + "_held"][0].float() * s[x + "_held"][1]).flatten(1, 2)[:, :case["Tk"]]) for x in ("k", "v"))
        rows = torch.full_like(s["lens"], case["Tq"]) if s["counts"] is None else s["counts"]
        at = (s["lens"] - rows).long()[:, None] + torch.arange(case["Tq"], device=DEV)
        return s["out"].copy_(_attend(case, s["q"], k, v, s, s["lens"], at, rows))
    if own:
        import paper_2608_28670_amd as bc
        bc.attention_masked(s["q"], s["k"], s["v"], s["out"], lens=s["lens"], q_docs=s["docs"], k_docs=s["docs"],
                            cap=case["cap"], slopes=s["slopes"], causal=case["causal"], window=case["window"],
                            prefix=s["prefix"], ws=s["ws"])
        return s["out"]
    at = (torch.arange(case["Tq"], device=DEV) + (case["Tk"] - case["Tq"])).expand(B, -1)
    full = torch.full((B,), case["Tk"], device=DEV)
    return s["out"].copy_(_attend(case, s["q"], s["k"].float(), s["v"].float(), s, full if s["lens"] is None else s["lens"],
                                  at, torch.full((B,), case["Tq"], device=DEV)))


# ---------------------------------------------------------------------------
# What a pass cannot do without, and what it should give
# ---------------------------------------------------------------------------
def _seen_pairs(case):
    """About how many (query, key) pairs of a head the masks leave."""
    Tq, Tk = case["Tq"], case["Tk"]
    if case["docs"]:
        return Tq * Tk * 1.8 / (case["docs"] + 1) * (0.5 if case["causal"] else 1.0)
    some = (0.67 if case["ragged"] else 1.0) * Tk
    if case["causal"]:
        some = some - 0.5 * min(some, Tq)
    if case["window"]:
        some = min(some, case["window"] * (1.0 if case["causal"] else 2.0) + (Tk / 6.0 if case["prefix"] else 0.0))
    return Tq * some * (0.67 if case["ragged"] and case["op"] == "cached" and Tq > 1 else 1.0)


def work(case):
    op, e = case["op"], 2 if case["dtype"] == "bf16" else 4
    if op == "rope":
        n = case["B"] * case["T"] * (case["Hq"] + case["Hk"]) * case["d"]
        return {"bytes": float(2 * n * e + case["B"] * case["T"] * case["axes"] * 4), "flops": 3.0 * n}
    if op == "push":
        new = case["B"] * case["H"] * case["d"] * case["T"] * 2 * (0.67 if case["ragged"] else 1.0)
        out = case["B"] * case["H"] * case["d"] * (case["T"] + case["held"]) * 2
        return {"bytes": float(new * e + new + out * (1 + e)), "flops": 4.0 * new}
    B, Hq, Hk, Tq, Tk, d = (case[k] for k in ("B", "Hq", "Hk", "Tq", "Tk", "d"))
    pairs = _seen_pairs(case)
    # Keys that some query sees; in the cache a byte each and its share of the scale.
    reach = Tk * (0.67 if case["ragged"] else 1.0)
    if case["window"] and not case["docs"]:
        reach = min(reach, Tq + case["window"] * 2 + (Tk / 6.0 if case["prefix"] else 0.0))
    kv = 2 * B * Hk * reach * (d * (1 if op == "cached" else e) + (4.0 / KB if op == "cached" else 0.0))
    return {"bytes": float(2 * B * Hq * Tq * d * e + kv), "flops": 4.0 * B * Hq * pairs * d}


def _exact_positions(case, s):
    ang = []
    pos = s["pos"].double()
    for axis, n in enumerate(_axis_dims(case)):
        c, pairs = _rope_scaling(case, axis), torch.arange(n // 2, device=DEV, dtype=torch.float64)
        base = math.log(c["theta"])
        if c["scaling"] == "ntk" and n > 2:
            base += math.log(c["factor"]) * n / (n - 2)
        f = torch.exp(-pairs * (2.0 / n) * base)
        if c["scaling"] == "linear":
            f /= c["factor"]
        elif c["scaling"] == "parts":
            keep = torch.clamp((c["original"] * f / math.tau - 1.0) / 31.0, min=0.0, max=1.0)
            f = keep * f + (1.0 - keep) * (f / c["factor"])
        ang.append(torch.einsum("bt,f->btf", pos[..., axis], f))
    return ang


def _exact_code(x, scale):
    return (x / scale).to(torch.float8_e4m3fn).double() * scale.double()


def _exact_scale(top):
    """The first of the powers of two from 2^-100 up that 1 / 448 of `top` does not exceed."""
    powers = torch.tensor([2.0 ** e for e in range(-100, 128)], dtype=torch.float64, device=DEV)
    return powers[torch.searchsorted(448.0 * powers, top.double().contiguous())].float()


def _exact_held(x, n):
    """What a cache holds of x [n, H, d] fp32 pushed at once."""
    full = torch.zeros((-(-n // KB) * KB,) + tuple(x.shape[1:]), device=DEV)
    full[:n] = x[:n]
    full = full.view(-1, KB, *x.shape[1:])
    scale = _exact_scale(full.abs().amax((1, 3)))[:, None, :, None]
    return _exact_code(full, scale).flatten(0, 1)[:n], scale


def exact(case, seed):
    s, op, B = _inputs(case, seed), case["op"], case["B"]
    if op == "rope":
        dims, out = _axis_dims(case), {}
        for x in ("q", "k"):
            o, at = s[x].double().clone(), 0
            for n, ang in zip(dims, _exact_positions(case, s)):
                z = torch.polar(torch.full_like(ang, _amplitude(case)), ang)[:, :, None]
                part = s[x][..., at:at + n].double()
                w = (torch.complex(part[..., 0::2].contiguous(), part[..., 1::2].contiguous()) if case["layout"] == "pairs" else
                     torch.complex(part[..., :n // 2].contiguous(), part[..., n // 2:].contiguous())) * z
                o[..., at:at + n] = torch.view_as_real(w).flatten(-2) if case["layout"] == "pairs" else torch.cat([w.real, w.imag], -1)
                at += n
            out[x] = o
        return out
    if op == "push":
        out, n = {}, case["held"] + case["T"]
        for x in ("k", "v"):
            o = torch.zeros((B, n, case["H"], case["d"]), dtype=torch.float64, device=DEV)
            for b in range(B):
                h, c = int(s["held"][b]), int(s["counts"][b])
                new, first = s[x][b, :c].float(), 0
                if h:
                    o[b, :h], old = _exact_held(s[x + "0"][b].float(), h)
                    first = min(c, -h % KB)      # tokens that join the last block held
                    if first:
                        i = h // KB
                        scale = torch.maximum(old[i], _exact_scale(new[:first].abs().amax((0, 2)))[None, :, None])
                        o[b, i * KB:h] = _exact_code(o[b, i * KB:h].float(), scale)
                        o[b, h:h + first] = _exact_code(new[:first], scale)
                if c > first:
                    o[b, h + first:h + c] = _exact_held(new[first:], c - first)[0]
            out[x] = o
        return out
    # One head of one sample at a time.
    Hq, Hk, Tq, Tk, d = (case[k] for k in ("Hq", "Hk", "Tq", "Tk", "d"))
    out = torch.zeros((B, Tq, Hq, d), dtype=torch.float64, device=DEV)
    for b in range(B):
        n = Tk if s["lens"] is None else int(s["lens"][b])
        rows = Tq if s["counts"] is None else int(s["counts"][b])
        if n == 0 or rows == 0:
            continue
        i = torch.arange(rows, device=DEV)[:, None] + (n - rows if op == "cached" else Tk - Tq)
        j = torch.arange(n, device=DEV)[None, :]
        hidden = torch.zeros((rows, n), dtype=torch.bool, device=DEV)
        if case["causal"]:
            hidden |= j > i
        if case["window"]:
            hidden |= (i - j >= case["window"]) | (j - i >= case["window"])
        if case["prefix"]:
            hidden[:, :min(n, int(s["prefix"][b]))] = False
        if case["docs"]:
            doc = s["docs"][b]
            hidden |= doc[:rows, None] != doc[None, :n]
            hidden |= doc[:rows, None] < 0
        for hk in range(Hk):
            k, v = s["k"][b, :n, hk:hk + 1].float(), s["v"][b, :n, hk:hk + 1].float()
            k, v = ((_exact_held(x, n)[0] if op == "cached" else x.double())[:, 0] for x in (k, v))
            for h in range(hk * (Hq // Hk), (hk + 1) * (Hq // Hk)):
                sc = s["q"][b, :rows, h].double() @ k.t() / d ** 0.5
                if case["cap"]:
                    sc = case["cap"] * torch.tanh(sc / case["cap"])
                if case["slopes"]:
                    sc -= float(s["slopes"][h]) * (i - j).abs()
                p = torch.softmax(sc.masked_fill_(hidden, -math.inf), -1)
                out[b, :rows, h] = torch.nan_to_num(p, nan=0.0) @ v
    return out
