"""bc_attention_masked: refusals on the CPU; on the GPU against float64."""
import ctypes as C
import math

import numpy as np
import pytest

from oracle import score
from score_checks import compare, tolerance

torch = pytest.importorskip("torch")
DEV = "cuda:0"
TDT = {"f32": torch.float32, "bf16": torch.bfloat16}
FAR = 1 << 24


# ---------------------------------------------------------------------------
# CPU
# ---------------------------------------------------------------------------
def _call(bc, ws=None, ws_bytes=0, opts=None, **kw):
    s = dict(B=1, Hq=2, Hk=2, Tq=200, Tk=300, d=64, dtype=1, q=FAR, k=2 * FAR, v=3 * FAR, q_batch=200 * 128, q_row=128, k_batch=300 * 128, k_row=128,
             v_batch=300 * 128, v_row=128, out=4 * FAR, q_start=100, lens=None, q_docs=None, k_docs=None)
    s.update(kw)
    return bc.lib().bc_attention_masked(C.byref(bc.MaskedDesc(opts=bc.ScoreOpts(**(opts or {})), **s)), ws, ws_bytes, None)


def test_refusals(bclib):
    bad, no = bclib.ERR_INVALID_ARG, bclib.ERR_UNSUPPORTED
    lim = 1 << 24
    cases = [(dict(B=0), bad), (dict(Hq=0), bad), (dict(Hk=0), bad), (dict(Tq=0), bad), (dict(Tk=0), bad), (dict(d=0), bad), (dict(Hq=3), bad),
             (dict(dtype=2), bad), (dict(d=40), no), (dict(d=256), no), (dict(Tk=lim + 1), no), (dict(Tq=lim + 1), no), (dict(B=1 << 20), no),
             (dict(B=200, Tk=lim), no), (dict(q=None), bad), (dict(k=None), bad), (dict(v=None), bad), (dict(out=None), bad), (dict(q=FAR + 8), bad),
             (dict(k=2 * FAR + 2), bad), (dict(v=3 * FAR + 4), bad), (dict(q_row=132), bad), (dict(k_row=-128), bad), (dict(B=2, v_batch=300 * 128 + 4), bad),
             (dict(out=4 * FAR + 1), bad), (dict(out=4 * FAR + 2, dtype=0), bad), (dict(q_docs=5 * FAR), bad), (dict(k_docs=5 * FAR), bad),
             (dict(lens=5 * FAR + 2), bad), (dict(q_docs=5 * FAR + 1, k_docs=6 * FAR), bad), (dict(q_start=lim), bad), (dict(q_start=-lim - 1), bad)]
    for kw, want in cases:
        assert _call(bclib, **kw) == want, kw
    for o in (dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(scale=1e-9), dict(cap=-1.0), dict(cap=math.nan), dict(cap=1e9),
              dict(cap=1e-6), dict(window=-1), dict(window=lim + 1), dict(slopes=5 * FAR + 2), dict(prefix=5 * FAR + 1)):
        assert _call(bclib, opts=o) == bad, o
    for at in (FAR, FAR + 4096, 2 * FAR, 3 * FAR, 5 * FAR, 6 * FAR, 7 * FAR, 8 * FAR, 9 * FAR):      # the output on another operand
        assert _call(bclib, out=at, lens=5 * FAR, q_docs=6 * FAR, k_docs=7 * FAR, ws=10 * FAR, ws_bytes=FAR, opts=dict(slopes=8 * FAR, prefix=9 * FAR)) == bad, at
    for at in (FAR, 2 * FAR, 3 * FAR, 4 * FAR, 6 * FAR, 7 * FAR):                                    # the workspace on another
        assert _call(bclib, q_docs=6 * FAR, k_docs=7 * FAR, ws=at, ws_bytes=FAR) == bad, at
    docs = dict(q_docs=6 * FAR, k_docs=7 * FAR)
    assert _call(bclib, **docs) == bad and _call(bclib, ws=8 * FAR + 128, ws_bytes=FAR, **docs) == bad and _call(bclib, ws=8 * FAR, ws_bytes=100, **docs) == bad
    split = dict(Tq=1, Tk=6400, k=16 * FAR, v=32 * FAR)                                              # few queries, many keys: in parts
    n = C.c_size_t()
    size = bclib.lib().bc_attention_masked_workspace_size
    assert size(1, 2, 2, 1, 6400, 64, 1, C.byref(n)) == bclib.OK and n.value > 1024
    assert _call(bclib, **split) == bad and _call(bclib, ws=64 * FAR, ws_bytes=256, **split) == bad and _call(bclib, ws=64 * FAR + 16, ws_bytes=n.value, **split) == bad
    assert bclib.lib().bc_attention_masked(None, None, 0, None) == bad
    assert size(1, 2, 2, 200, 300, 64, 1, None) == bad and size(1, 3, 2, 200, 300, 64, 1, C.byref(n)) == bad and size(1, 2, 2, 200, 300, 48, 1, C.byref(n)) == no


def test_binding_refuses_tensors_that_do_not_fit(bclib):
    bf, i32 = torch.bfloat16, torch.int32
    q, k = torch.zeros(2, 20, 6, 32, dtype=bf), torch.zeros(2, 30, 3, 32, dtype=bf)
    ok = dict(q=q, k=k, v=k.clone(), out=q.clone())
    for kw in (dict(k=k.float()), dict(k=k[:1]), dict(k=torch.zeros(2, 30, 3, 64, dtype=bf)), dict(v=k[:, :20]), dict(out=q[:, :10]), dict(out=q.float()),
               dict(out=q.transpose(1, 2)), dict(q=torch.zeros(2, 6, 20, 32, dtype=bf).transpose(1, 2)), dict(q=q[0]), dict(lens=torch.zeros(3, dtype=i32)),
               dict(lens=torch.zeros(2)), dict(prefix=torch.zeros(2, dtype=torch.int64)), dict(slopes=torch.zeros(3)), dict(slopes=torch.zeros(6, dtype=bf)),
               dict(q_docs=torch.zeros(2, 30, dtype=i32)), dict(k_docs=torch.zeros(2, 20, dtype=i32)), dict(q_docs=torch.zeros(20, 2, dtype=i32).t())):
        with pytest.raises((bclib.BCError, TypeError)) as e:
            bclib.attention_masked(**dict(ok, **kw))
        assert getattr(e.value, "code", bclib.ERR_INVALID_ARG) == bclib.ERR_INVALID_ARG, kw
    with pytest.raises(bclib.BCError) as e:                                               # tensors of the host
        bclib.attention_masked(**ok)
    assert e.value.code == bclib.ERR_INVALID_ARG


def test_strides_whose_offsets_pass_64_bits_are_refused(bclib):
    for kw in (dict(B=1 << 14, q_batch=1 << 48), dict(B=1 << 14, k_batch=1 << 48), dict(B=1 << 14, v_batch=1 << 48), dict(B=256, q_batch=1 << 48)):
        assert _call(bclib, **kw) == bclib.ERR_INVALID_ARG, kw


def test_binding_refuses_numbers_past_their_types(bclib):
    q = torch.zeros(1, 2, 1, 32)
    for kw in (dict(window=1 << 40), dict(q_start=1 << 70)):
        with pytest.raises(bclib.BCError) as e:
            bclib.attention_masked(q, q.clone(), q.clone(), q.clone(), **kw)
        assert e.value.code == bclib.ERR_INVALID_ARG, kw


def test_oracle():
    """Against dense softmax with a mask; a cap above every score changes nothing; one visible key gives its value."""
    g = np.random.default_rng(0)
    q, k, v = g.standard_normal((9, 8)), g.standard_normal((12, 8)), g.standard_normal((12, 8))
    p = np.arange(9) + 3
    see = score.seen(p, 12, causal=True, window=4, prefix=2)
    want = np.array([[(j <= a and a - j < 4) or j < 2 for j in range(12)] for a in p])
    assert np.array_equal(see, want)
    both = score.seen(p, 12, window=3)
    assert np.array_equal(both, np.abs(p[:, None] - np.arange(12)) < 3)
    s = np.where(see, q @ k.T * 0.5 - 0.1 * np.abs(p[:, None] - np.arange(12)), -np.inf)
    w = np.exp(s - s.max(1, keepdims=True))
    assert np.allclose(score.attend(q, k, v, see, p, 0.5, slope=0.1)[0], (w / w.sum(1, keepdims=True)) @ v)
    assert np.allclose(score.attend(q, k, v, see, p, 0.5, cap=1e7)[0], score.attend(q, k, v, see, p, 0.5)[0])
    assert np.allclose(score.attend(q, k, v, np.eye(9, 12, dtype=bool), p, 0.5)[0], v[:9])
    docs = np.array([0, 0, 1, 1, -1, 2, 2, 2, 2])
    see = score.seen(np.arange(9), 9, q_docs=docs, k_docs=docs)
    assert see[4].sum() == 0 and see[2].tolist() == [False, False, True, True] + [False] * 5 and not score.attend(q, k[:9], v[:9], see, p, 1.0)[0][4].any()


# ---------------------------------------------------------------------------
# GPU
# ---------------------------------------------------------------------------
def _np(t):
    return t.double().cpu().numpy()


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _qkv(B, Hq, Hk, Tq, Tk, d, dt, seed=0, view=False):
    """view: rows of projections, the keys and values side by side, a gap behind each."""
    g = _gen(seed)
    mk = lambda *s: torch.empty(s, device=DEV).normal_(generator=g).to(TDT[dt])   # noqa: E731
    if not view:
        return mk(B, Tq, Hq, d), mk(B, Tk, Hk, d), mk(B, Tk, Hk, d)
    x, y = mk(B, Tq + 3, Hq * d + 8), mk(B, Tk + 1, 2 * Hk * d + 16)
    return (x[:, :Tq, 8:].unflatten(-1, (Hq, d)), y[:, :Tk, :Hk * d].unflatten(-1, (Hk, d)), y[:, :Tk, Hk * d:2 * Hk * d].unflatten(-1, (Hk, d)))


def _i32(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device=DEV)


def _run(bc, q, k, v, lens=None, docs=None, prefix=None, slopes=None, stream=None, **kw):
    B, Tq, Hq, d = q.shape
    Tk, Hk = k.shape[1:3]
    buf = torch.full((q.numel() + 64,), 7.0, device=DEV, dtype=q.dtype)
    out = buf[32:-32].view(B, Tq, Hq, d)
    n = bc.attention_masked_workspace_size(B, Hq, Hk, Tq, Tk, d, bc.dtype_code(q))
    ws = torch.full((n + 256,), 0xFF, dtype=torch.uint8, device=DEV)      # NaNs, were they read
    bc.attention_masked(q, k, v, out, lens=_i32(lens), prefix=_i32(prefix), slopes=slopes, q_docs=None if docs is None else _i32(docs[0]),
                        k_docs=None if docs is None else _i32(docs[1]), ws=ws[:n], **kw)
    torch.cuda.synchronize()
    assert bool((buf[:32] == 7).all()) and bool((buf[-32:] == 7).all()) and bool((ws[n:] == 0xFF).all())
    return out


def _check(bc, q, k, v, lens=None, docs=None, prefix=None, slopes=None, scale=None, cap=0.0, causal=False, window=0, q_start=None):
    out = _run(bc, q, k, v, lens, docs, prefix, slopes, scale=scale, cap=cap, causal=causal, window=window, q_start=q_start)
    B, Tq, Hq, d = q.shape
    Tk, Hk = k.shape[1:3]
    p = np.arange(Tq) + (Tk - Tq if q_start is None else q_start)
    qn, kn, vn, got = (_np(t) for t in (q, k, v, out))
    sl = None if slopes is None else _np(slopes)
    for b in range(B):
        n = Tk if lens is None else min(max(lens[b], 0), Tk)
        see = score.seen(p, n, causal, window, 0 if prefix is None else prefix[b], None if docs is None else np.array(docs[0][b]),
                         None if docs is None else np.array(docs[1][b]))
        for h in range(Hq):
            hk = h // (Hq // Hk)
            want, A, size, mag = score.attend(qn[b, :, h], kn[b, :n, hk], vn[b, :n, hk], see, p, d ** -0.5 if scale is None else scale, cap,
                                              0.0 if sl is None else sl[h])
            compare(got[b, :, h], want, tolerance(want, A, size, mag, d, Tk, cap, q.dtype == torch.bfloat16), A)
    return out


def _slopes(Hq):
    return 2.0 ** (-8.0 * torch.arange(1, Hq + 1, device=DEV, dtype=torch.float32) / Hq)


def _docs(B, T, n, seed, holes=True, mixed=False):
    """Documents of a packed row, in order (mixed: not), some tokens without one."""
    g = np.random.default_rng(seed)
    d = np.sort(g.integers(0, n, (B, T)), axis=1)
    if mixed:
        d = g.integers(0, n, (B, T))
    if holes:
        d[:, T - T // 10:] = -1
        d[g.random((B, T)) < 0.02] = -5
    return d.tolist()


SHAPES = [  # B, Hq, Hk, Tq, Tk, d
    (1, 1, 1, 1, 1, 32), (2, 4, 2, 1, 63, 64), (1, 8, 1, 2, 640, 128), (2, 3, 3, 16, 65, 72), (1, 2, 2, 17, 130, 64), (3, 2, 1, 40, 257, 32),
    (1, 2, 2, 129, 129, 128), (2, 2, 2, 200, 333, 72), (1, 5, 5, 300, 300, 64), (1, 6, 2, 100, 1000, 128), (1, 1, 1, 3, 4500, 64), (1, 2, 2, 70, 20, 32),
    (2, 16, 2, 5, 900, 72), (1, 32, 4, 2, 3000, 128)]
MASKS = ["none", "causal", "window", "causal window", "prefix", "lens", "docs", "docs causal", "mixed docs", "all"]


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("B,Hq,Hk,Tq,Tk,d", SHAPES)
def test_masks(bclib, B, Hq, Hk, Tq, Tk, d, mask, dt):
    seed = Tq * 7 + Tk
    q, k, v = _qkv(B, Hq, Hk, Tq, Tk, d, dt, seed, view=mask in ("causal", "docs", "all"))
    kw = {}
    if "causal" in mask or mask in ("prefix", "all"):
        kw["causal"] = True
    if "window" in mask or mask in ("prefix", "all"):
        kw["window"] = max(1, Tk // 5)
    if mask in ("prefix", "all"):
        kw["prefix"] = [(b * 37 + 1) % (Tk + 9) - 3 for b in range(B)]
    if mask in ("lens", "all"):
        kw["lens"] = [[Tk + 5, Tk - Tk // 3, 0, -2][b % 4] if mask == "lens" else max(1, Tk - 70 * b) for b in range(B)]
        for b, n in enumerate(kw["lens"]):                # behind a sample's keys
            k[b, max(n, 0):] = math.nan
            v[b, max(n, 0):] = math.inf
    if "docs" in mask:
        n = max(1, Tk // 50)
        kw["docs"] = (_docs(B, Tq, n, seed, mixed="mixed" in mask), _docs(B, Tk, n, seed + (Tq != Tk), mixed="mixed" in mask))
    if mask == "all":
        kw.update(docs=(_docs(B, Tq, 2, seed), _docs(B, Tk, 2, seed)), cap=20.0, slopes=_slopes(Hq), scale=0.3)
    _check(bclib, q, k, v, **kw)


@pytest.mark.gpu
@pytest.mark.parametrize("dt,B,Hq,Hk,T,d", [("bf16", 1, 16, 16, 4201, 32), ("bf16", 2, 20, 5, 1700, 72), ("f32", 3, 6, 6, 1950, 32)])
def test_documents_over_many_workgroups(bclib, dt, B, Hq, Hk, T, d):
    """More than one round of workgroups, which start by their documents' sizes."""
    q, k, v = _qkv(B, Hq, Hk, T, T, d, dt, seed=T)
    docs = _docs(B, T, 12, T)
    docs[0] = [0] * (T // 3) + [1 + i // 90 for i in range(T - T // 3)]
    _check(bclib, q, k, v, docs=(docs, docs), causal=d == 72, lens=[T - 100] * B if d == 72 else None)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("cap", [0.0, 0.5, 30.0, 999.0, 5000.0, 1e6])
@pytest.mark.parametrize("B,Hq,Hk,Tq,Tk,d", [(1, 4, 1, 2, 300, 64), (1, 2, 2, 50, 200, 128), (1, 2, 1, 150, 260, 72), (1, 2, 2, 200, 100, 32)])
def test_caps_and_distances(bclib, B, Hq, Hk, Tq, Tk, d, cap, dt):
    q, k, v = _qkv(B, Hq, Hk, Tq, Tk, d, dt, seed=d)
    q *= 6.0                                              # scores of tens
    _check(bclib, q, k, v, cap=cap)
    _check(bclib, q, k, v, cap=cap, slopes=_slopes(Hq))
    _check(bclib, q, k, v, cap=cap, slopes=-_slopes(Hq) / 8, q_start=17, causal=True)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_far_positions(bclib, dt):
    """Queries at the far end of the positions: everything, nothing, the prefix; distances of 2^24."""
    for Tq in (1, 100):
        q, k, v = _qkv(1, 2, 2, Tq, 150, 64, dt, seed=Tq)
        for start in ((1 << 24) - Tq, -(1 << 24), -50, 149):
            _check(bclib, q, k, v, q_start=start, causal=True)
            _check(bclib, q, k, v, q_start=start, window=60, prefix=[70])
            _check(bclib, q, k, v, q_start=start, window=1 << 24)
            _check(bclib, q, k, v, q_start=start, slopes=torch.tensor([1e-6, 0.0], device=DEV))


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("Tq,d,Hq", [(1, 64, 4), (9, 72, 2), (60, 32, 2), (150, 128, 2), (190, 72, 4), (200, 64, 2)])
def test_hidden_and_seen_values_that_are_not_finite(bclib, Tq, d, Hq, dt):
    """NaN and infinities in keys and values of other documents, later tokens and padding leave no trace; where they are seen, the formula's."""
    Tk = 200
    q, k, v = _qkv(1, Hq, Hq // 2, Tq, Tk, d, dt, seed=Tq)
    kd = np.repeat([0, 1, 2, 3, -1], [40, 50, 60, 45, 5])
    qd = kd[Tk - Tq:]
    bad_v = ((10, 1, math.inf), (95, d - 1, math.nan), (130, 3, math.inf), (131, 3, -math.inf), (132, 4, -math.inf), (198, 2, math.nan), (199, 5, math.inf))
    for j, c, x in bad_v:
        v[0, j, 0, c] = x
    k[0, 197] = math.nan
    docs = ([qd.tolist()], [kd.tolist()])
    _check(bclib, q, k, v, docs=docs)
    _check(bclib, q, k, v, docs=docs, causal=True, window=30)
    _check(bclib, q, k, v, causal=True, lens=[197])
    _check(bclib, q, k, v, lens=[90])
    got = _run(bclib, q, k, v, causal=True)               # the last rows see everything, the NaN key too
    assert bool(got[0, -1].isnan().all())
    q[0, 0, 0, 0] = math.nan                              # a query's own NaN stays in its row
    got = _run(bclib, q, k, v, docs=docs)
    assert bool(got[0, 0, 0].isnan().all()) or qd[0] < 0
    if Tq > 10:
        assert not bool(got[0, 10:, 1].isnan().all(-1).any())


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("Tq", [2, 60, 300])
def test_growing_scores(bclib, Tq, dt):
    """Scores of several hundred that grow from tile to tile, and fall: the references move at every one, or never after the first."""
    q, k, v = _qkv(1, 1, 1, Tq, 64 * 12, 64, dt, seed=Tq)
    k *= torch.arange(1, 64 * 12 + 1, device=DEV, dtype=torch.float32).div(40).view(1, -1, 1, 1).to(k.dtype)
    _check(bclib, q, k, v)
    _check(bclib, q, k.flip(1).contiguous(), v, causal=True)
    _check(bclib, q, k, v, scale=1e-6)


@pytest.mark.gpu
@pytest.mark.parametrize("dt,Hq,Tk", [("bf16", 16, 70_001), ("f32", 2, 9001)])
def test_few_queries_over_many_keys(bclib, dt, Hq, Tk):
    """In parts, past the caches' reach (bf16: 143 MB), with parts that see nothing."""
    q, k, v = _qkv(2, Hq, 4 if dt == "bf16" else 1, 2, Tk, 128, dt, seed=1)
    _check(bclib, q, k, v, lens=[Tk, 40_000 if dt == "bf16" else 130])
    _check(bclib, q, k, v, window=1000, causal=True, prefix=[70, 0])
    a = _run(bclib, q, k, v)
    assert torch.equal(a, _run(bclib, q, k, v))


@pytest.mark.gpu
def test_agrees_with_attention_without_masks(bclib):
    """Without options: bc_attention's results up to the order of the sums."""
    for dt, d in (("bf16", 128), ("bf16", 72), ("f32", 64)):
        q, k, v = _qkv(2, 3, 3, 700, 700, d, dt, seed=2)
        a, b = _run(bclib, q, k, v), torch.empty_like(q)
        bclib.attention(q, k, v, b)
        assert float((a.double() - b.double()).norm() / b.double().norm()) <= (4e-3 if dt == "bf16" else 2e-6)


@pytest.mark.gpu
@pytest.mark.parametrize("Tq", [1, 100])
def test_rows_beyond_32_bit_offsets(bclib, Tq):
    """Keys 2^25 values apart: the last start past 2^33 bytes."""
    Tk, row = 170, 1 << 25
    x = torch.empty(Tk * row, dtype=torch.bfloat16, device=DEV).view(1, Tk, row)
    q, k, v = _qkv(1, 2, 1, Tq, Tk, 64, "bf16", seed=5)
    k2, v2 = x[..., :64].unflatten(-1, (1, 64)), x[..., 64:128].unflatten(-1, (1, 64))
    k2.copy_(k)
    v2.copy_(v)
    assert torch.equal(_check(bclib, q, k2, v2, causal=True), _run(bclib, q, k, v, causal=True))


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("Tq", [1, 40, 150])
def test_prefixes_outside_the_keys(bclib, Tq, dt):
    """Held to the sample's keys: what is below shows nothing, what is above shows all."""
    q, k, v = _qkv(5, 2, 1, Tq, 200, 64, dt, seed=Tq)
    for kw in (dict(causal=True), dict(window=9), dict(causal=True, window=9)):
        out = _run(bclib, q, k, v, [200, 190, 0, 200, 130], None, [-2 ** 31, -1, 5, 2 ** 31 - 1, 131], **kw)
        want = _check(bclib, q, k, v, lens=[200, 190, 0, 200, 130], prefix=[0, 0, 0, 200, 130], **kw)
        assert torch.equal(out, want)


@pytest.mark.gpu
def test_streams_and_captured_graphs(bclib):
    """Two streams with workspaces of their own at once; two graphs replayed in turn on new lengths and documents."""
    q, k, v = _qkv(2, 4, 2, 33, 1000, 64, "bf16", seed=9)
    lens, docs = _i32([1000, 700]), _i32(_docs(2, 1000, 4, 3))
    n = bclib.attention_masked_workspace_size(2, 4, 2, 33, 1000, 64, bclib.BF16)
    runs = []
    for kw in (dict(causal=True, window=300), dict(cap=10.0)):
        s, out, ws = torch.cuda.Stream(), torch.empty_like(q), torch.empty(n, dtype=torch.uint8, device=DEV)
        qd = docs[:, -33:].contiguous()
        call = lambda o, w, kw=kw, qd=qd, **a: bclib.attention_masked(q, k, v, o, lens=lens, q_docs=qd, k_docs=docs, ws=w, **kw, **a)  # noqa: E731
        want, ws2 = torch.empty_like(q), torch.empty(n, dtype=torch.uint8, device=DEV)
        call(want, ws2)
        s.wait_stream(torch.cuda.current_stream())
        runs.append((s, out, ws, call, want, ws2))
    for s, out, ws, call, want, ws2 in runs:
        call(out, ws, stream=s)
    torch.cuda.synchronize()
    graphs = []
    for s, out, ws, call, want, ws2 in runs:
        assert torch.equal(out, want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(out, ws)
        graphs.append(graph)
    for step in range(3):
        lens -= 111
        for graph in graphs:
            graph.replay()
        for s, out, ws, call, want, ws2 in runs:
            call(want, ws2)
            torch.cuda.synchronize()
            assert torch.equal(out, want), step


def _check_hidden(bc, q, k, v, bad, lens=None, docs=None, prefix=None, slopes=None, cap=0.0, causal=False, window=0):
    """Keys `bad` = {key: value} are that value in their first columns of every head: rows that see one with a NaN are NaN, rows
    that see none of them are as without them."""
    (B, Tq, Hq, d), (Tk, Hk) = q.shape, k.shape[1:3]
    dirty = k.clone()
    for j, x in bad.items():
        dirty[:, j, :, :3] = x
    got = _np(_run(bc, q, dirty, v, lens, docs, prefix, slopes, cap=cap, causal=causal, window=window))
    qn, kn, vn = (_np(t) for t in (q, k, v))
    p, checked = np.arange(Tq) + Tk - Tq, 0
    for b in range(B):
        n = Tk if lens is None else lens[b]
        see = score.seen(p, n, causal, window, 0 if prefix is None else prefix[b], None if docs is None else np.array(docs[0][b]),
                         None if docs is None else np.array(docs[1][b]))
        nan = [j for j, x in bad.items() if math.isnan(x) and j < n]
        clean, ill = ~see[:, [j for j in bad if j < n]].any(1), see[:, nan].any(1)
        checked += int(clean.sum())
        for h in range(Hq):
            want, A, size, mag = score.attend(qn[b, :, h], kn[b, :n, h // (Hq // Hk)], vn[b, :n, h // (Hq // Hk)], see, p, d ** -0.5, cap,
                                              0.0 if slopes is None else float(slopes[h]))
            tol = tolerance(want, A, size, mag, d, Tk, cap, q.dtype == torch.bfloat16)
            compare(got[b, clean, h], want[clean], tol[clean], A[clean])
            assert np.isnan(got[b, ill, h]).all()
    assert checked


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("Tq", [4, 40, 150, 190])
@pytest.mark.parametrize("d", [32, 64, 72, 128])
def test_hidden_keys_next_to_seen_ones(bclib, d, Tq, dt):
    """NaN and infinities in the key after the last one that a row sees, and before its first: another document's, the next token's, one
    behind the window or the prefix, one past a sample's end."""
    Tk = 200
    q, k, v = _qkv(1, 4, 2, Tq, Tk, d, dt, seed=Tq + d)
    kd = np.repeat([0, 1, 2, 3, -1], [40, 50, 60, 45, 5])
    docs = ([kd[Tk - Tq:].tolist()], [kd.tolist()])
    more = dict(cap=20.0, slopes=_slopes(4))
    for bad in ({90: math.nan}, {150: math.nan, 195: math.inf}, {195: math.nan}, {39: math.nan, 89: -math.inf, 149: math.inf}, {196: math.inf, 197: math.nan}):
        for kw in (dict(), more):
            _check_hidden(bclib, q, k, v, bad, docs=docs, **kw)
    for j in (197, 198, Tk - Tq // 2):
        for kw in (dict(), more, dict(window=30)):
            _check_hidden(bclib, q, k, v, {j: math.nan}, causal=True, **kw)
        _check_hidden(bclib, q, k, v, {j: -math.inf, min(j + 1, Tk - 1): math.inf}, causal=True)
    _check_hidden(bclib, q, k, v, {150: math.nan}, window=max(2, Tq // 9))
    _check_hidden(bclib, q, k, v, {5: math.nan, 6: math.inf, 130: math.nan}, causal=True, window=max(2, Tq // 9), prefix=[5])
    _check_hidden(bclib, q, k, v, {197: math.nan}, lens=[197])


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("B,Hq,Hk,Tq,Tk,d", [(1, 2, 1, 1, 200, 64), (1, 4, 1, 1, 6000, 128), (1, 2, 2, 30, 190, 72), (1, 2, 1, 40, 5000, 64), (2, 3, 3, 150, 260, 72),
                                             (1, 2, 2, 200, 4000, 128), (1, 1, 1, 130, 64, 32), (1, 64, 8, 70, 2000, 32)])
def test_seen_values_of_small_weights_that_are_not_finite(bclib, B, Hq, Hk, Tq, Tk, d, dt):
    """A weight of 2^-230 is below fp32's least, and still more than nothing: an infinite value that is seen makes the output infinite, wherever
    the keys are cut; opposite ones make NaN, as NaN does."""
    q, k, v = _qkv(B, Hq, Hk, Tq, Tk, d, dt, seed=Tk)
    q[..., 0], k[..., 0] = 8.0, 0.0
    first, mid, last = 3, Tk // 2, Tk - 2
    k[:, [first, mid, last], :, 0] = -20.0                # 160 below the others
    v[:, first, :, 1] = math.inf
    v[:, last, :, 2] = -math.inf
    v[:, mid, :, 3] = math.nan
    v[:, first, :, 4], v[:, last, :, 4] = math.inf, -math.inf
    v[:, mid, :, d - 1] = math.inf
    v[:, mid + 1, :, 5] = math.inf                        # of an ordinary weight
    _check(bclib, q, k, v, scale=1.0)
    _check(bclib, q, k, v, scale=1.0, causal=True, lens=[last] * B)
    _check(bclib, q, k, v, scale=1.0, window=max(2, Tk // 3), prefix=[first] * B)
    _check(bclib, q, k, v, scale=1.0, slopes=torch.full((Hq,), 1e-3, device=DEV), cap=500.0)


@pytest.mark.gpu
@pytest.mark.parametrize("dt,Tq", [("bf16", 1), ("bf16", 40), ("bf16", 150), ("f32", 1), ("f32", 40)])
def test_prefix_and_window_share_the_parts(bclib, dt, Tq):
    """The keys between a prefix and a window, which nobody sees, are nobody's work: every part has some that are seen."""
    B, H, Tk, d = 1, 2, 16384, 64
    q, k, v = _qkv(B, H, H, Tq, Tk, d, dt, seed=Tq)
    size = bclib.attention_masked_workspace_size(B, H, H, Tq, Tk, d, bclib.dtype_code(q))
    parts = (size - 8 * (Tk // 64 + (Tq + 63) // 64)) // (Tq * H * (d + 2) * 4)       # (the rest is the documents')
    assert parts > 4
    ws = torch.zeros(size, dtype=torch.uint8, device=DEV)
    for prefix in (4, 200):
        ws.zero_()
        bclib.attention_masked(q, k, v, torch.empty_like(q), causal=True, window=4096, prefix=_i32([prefix]), ws=ws)
        sums = ws.view(torch.float32)[Tq * H * parts * d:][:Tq * H * parts * 2].view(Tq * H, parts, 2)[..., 1]
        assert bool((sums != 0).any(0).all()), (prefix, (sums != 0).any(0).tolist())


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hk,Tq,Tk", [(4, 1, 1, 3000), (2, 2, 3, 5000), (2, 1, 33, 3000), (2, 1, 300, 1500), (1, 1, 200, 700)])
def test_prefix_and_window_at_every_distance(bclib, Hq, Hk, Tq, Tk, dt):
    """A prefix that ends tiles before the window's first, beside it, in it, behind it; windows before all keys."""
    q, k, v = _qkv(2, Hq, Hk, Tq, Tk, 64, dt, seed=Tk)
    for window, prefix in ((1, [1, 64]), (70, [65, 128]), (300, [Tk - 500, Tk - 300]), (300, [Tk - 364, Tk - 100]), (Tk // 2, [Tk // 2 - 63, Tk // 2 + 1]),
                           (64, [Tk, 0]), (2 * Tk, [100, 3])):
        _check(bclib, q, k, v, window=window, prefix=prefix, causal=window % 4 != 0)
    _check(bclib, q, k, v, window=90, prefix=[500, 129], lens=[400, Tk - 130], causal=True)
    _check(bclib, q, k, v, window=90, prefix=[500, 1], q_start=-200, causal=True)
    _check(bclib, q, k, v, window=90, prefix=[77, 0], q_start=Tk + 80)
    docs = (_docs(2, Tq, 3, 1), _docs(2, Tk, 3, 1))
    _check(bclib, q, k, v, window=200, prefix=[70, 700], docs=docs)


@pytest.mark.gpu
@pytest.mark.parametrize("Tq", [2100, 4101])
def test_documents_over_very_many_rows(bclib, Tq):
    """525 workgroups of 64 rows a head, ordered by one thread each, and 1026, which are not ordered."""
    q, k, v = _qkv(1, 16, 1, Tq, Tq, 32, "f32", seed=Tq)
    docs = [[0] * 300 + [1 + i // 40 for i in range(Tq - 300)]]
    docs[0][77] = docs[0][Tq - 1] = -1
    _check(bclib, q, k, v, docs=(docs, docs))
