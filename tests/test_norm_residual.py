"""bc_norm_gate_residual: refusals on the CPU; on the GPU against float64.

Tolerances, with u = 2^-24.  A lane adds at most 64 values before ten further
additions, so a row's sum is off by at most 74 u of the sum of magnitudes: the
mean by 74 u mean|v|, the mean square by 76 u of itself plus what the mean's
error brings (second order), 1 / sqrt by half of that and three roundings.  N =
80 of them cover each of the two terms:
    norm:  80 u (|n| + mean|v| rstd), and an error e of the input gives 2 e rstd;
    x':    |g| times z's, and 3 u (|g z| + |a x|);
    h:     (1 + |scale|) times the norm's, and 4 u of its terms;
    bf16:  half a step, 2^-8, of h."""
import ctypes as C

import numpy as np
import pytest

torch = pytest.importorskip("torch")
DEV = "cuda:0"
TDT = {"f32": torch.float32, "bf16": torch.bfloat16}
KIND = {"none": 0, "rms": 1, "layer": 2}
U = 2.0 ** -24


def _desc(bc, **kw):
    d = bc.NormDesc()
    d.rows, d.D, d.rows_per_sample, d.dtype = 4, 64, 2, bc.F32
    d.y, d.x, d.x_out, d.h = 1 << 20, 2 << 20, 2 << 20, 3 << 20
    d.ldy = d.ldx = d.ldh = d.ld_gate = d.ld_mod = 64
    d.res_scale, d.eps = 1.0, 1e-6
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def test_refusals(bclib):
    fn = bclib.lib().bc_norm_gate_residual
    assert fn(None, None) == bclib.ERR_INVALID_ARG
    far = 8 << 20
    for kw in (dict(rows=-1), dict(D=0), dict(rows_per_sample=0), dict(dtype=2), dict(y=None), dict(x=None), dict(x_out=None),
               dict(post=3), dict(pre=-1), dict(post_w=far), dict(post=1, post_b=far), dict(post=1, post_w=far, post_b=far),
               dict(pre=2, pre_b=far), dict(shift=far), dict(scale=far), dict(h=None, pre=1), dict(h=None, shift=far, scale=far),
               dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(res_scale=float("nan")),
               dict(res_scale=float("inf")), dict(ldy=63), dict(ldx=63), dict(ldh=63), dict(gate=far, ld_gate=63),
               dict(shift=far, scale=far, ld_mod=63), dict(ldy=1 << 41),
               dict(x_out=(2 << 20) + 256), dict(h=2 << 20), dict(y=2 << 20), dict(h=(1 << 20) + 4), dict(h=1 << 20, ldh=65)):
        assert fn(C.byref(_desc(bclib, **kw)), None) == bclib.ERR_INVALID_ARG, kw
    far4 = dict(gate=far, shift=far + 4096, scale=far + 8192)
    for kw in (dict(y=(1 << 20) + 2), dict(x=(2 << 20) + 1, x_out=(2 << 20) + 1), dict(h=(3 << 20) + 2), dict(gate=far + 2),
               dict(far4, shift=far + 4097), dict(post=1, post_w=far + 2), dict(dtype=bclib.BF16, y=(1 << 20) + 1),           # not aligned to their elements
               dict(gate=(2 << 20) + 512), dict(gate=(3 << 20) - 4 * 64), dict(far4, scale=2 << 20), dict(far4, shift=(3 << 20) + 4),
               dict(post=1, post_w=(2 << 20) - 252), dict(pre=2, pre_w=far, pre_b=3 << 20), dict(ldy=(1 << 36) + 1)):
        assert fn(C.byref(_desc(bclib, **kw)), None) == bclib.ERR_INVALID_ARG, kw
    assert fn(C.byref(_desc(bclib, D=16385, ldy=16385, ldx=16385, ldh=16385)), None) == bclib.ERR_UNSUPPORTED
    assert fn(C.byref(_desc(bclib, rows=1 << 24)), None) == bclib.ERR_UNSUPPORTED
    assert fn(C.byref(_desc(bclib, rows=0)), None) == bclib.OK                 # nothing to do


def test_binding_refuses_tensors_that_do_not_fit(bclib):
    z = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt)
    y, x = z(4, 8), z(4, 8)
    for kw in (dict(h=z(4, 9)), dict(h=z(3, 8)), dict(h=z(4, 8, dt=torch.bfloat16)), dict(gate=z(1, 8)), dict(gate=z(2, 8, dt=torch.bfloat16)),
               dict(gate=z(2, 7)), dict(shift=z(2, 8), scale=z(2, 16)[:, ::2]), dict(shift=z(2, 8), scale=z(2, 16)[:, :8]),
               dict(post=1, post_w=z(7)), dict(post=1, post_w=z(8, dt=torch.bfloat16)), dict(post=1, post_w=z(16)[::2])):
        with pytest.raises(bclib.BCError) as e:
            bclib.norm_gate_residual(y, x, x, rows_per_sample=2, **kw)
        assert e.value.code == bclib.ERR_INVALID_ARG, kw
    with pytest.raises(bclib.BCError) as e:                                      # tensors of the host
        bclib.norm_gate_residual(y, x, z(4, 8))
    assert e.value.code == bclib.ERR_INVALID_ARG
    for a in ((y, z(4, 8, dt=torch.bfloat16), z(4, 8)), (y, x, z(3, 8)), (y, x, z(4, 16)[:, :8]), (z(4, 16)[:, ::2], x, x), (y, z(5, 8), z(5, 8))):
        with pytest.raises((bclib.BCError, TypeError)):
            bclib.norm_gate_residual(*a)


def _norm64(v, kind, w, b, eps):
    """(normed, rstd, mean |v|) in float64."""
    r = np.ones((v.shape[0], 1))
    n = v
    if kind == "layer":
        n = n - n.mean(1, keepdims=True)
    if kind != "none":
        r = 1.0 / np.sqrt((n * n).mean(1, keepdims=True) + eps)
        n = n * r
    if w is not None:
        n = n * w
    if b is not None:
        n = n + b
    return n, r, np.abs(v).mean(1, keepdims=True)


def _np(t):
    return None if t is None else t.double().cpu().numpy()


def _check(bc, y, x, x_out, h, rps, post, pre, a, vecs, mods, eps=1e-6):
    gate, shift, scale = mods
    x64, y64 = _np(x), _np(y)
    x0 = x64.copy()
    bc.norm_gate_residual(y, x, x_out, h, rows_per_sample=rps, post=KIND[post], post_w=vecs[0], post_b=vecs[1], gate=gate,
                          res_scale=a, pre=KIND[pre], pre_w=vecs[2], pre_b=vecs[3], shift=shift, scale=scale, eps=eps)
    s = np.arange(y64.shape[0]) // rps
    pw, pb, nw, nb = map(_np, vecs)
    one = np.ones_like
    absmax = lambda w: one(y64[:1]) if w is None else np.abs(w)[None]
    with np.errstate(invalid="ignore", over="ignore"):
        z, r, m = _norm64(y64, post, pw, pb, eps)
        ez = np.zeros_like(z) if post == "none" else 80 * U * (np.abs(z) + m * r * absmax(pw))
        g = one(z) if gate is None else _np(gate)[s]
        x2 = a * x0 + g * z
        ex = np.abs(g) * ez + 3 * U * (np.abs(g * z) + np.abs(a * x0))
        assert np.all((np.abs(_np(x_out) - x2) <= ex) | ~np.isfinite(x2)), float(np.nanmax(np.abs(_np(x_out) - x2) / ex))
        assert np.array_equal(np.isfinite(_np(x_out)), np.isfinite(x2))
        if h is None:
            return
        n, r, m = _norm64(x2, pre, nw, nb, eps)
        en = ex if pre == "none" else 2 * ex.max(1, keepdims=True) * r * absmax(nw) + 80 * U * (np.abs(n) + m * r * absmax(nw))
        sc, sh = (np.zeros_like(n), np.zeros_like(n)) if scale is None else (_np(scale)[s], _np(shift)[s])
        want = n * (1 + sc) + sh
        eh = en * (1 + np.abs(sc)) + 4 * U * (np.abs(n) * (1 + np.abs(sc)) + np.abs(sh))
        if h.dtype == torch.bfloat16:
            eh = eh + np.abs(want) * 2.0 ** -8 + 1e-30
        assert np.all((np.abs(_np(h) - want) <= eh) | ~np.isfinite(want)), float(np.nanmax(np.abs(_np(h) - want) / eh))
        assert np.array_equal(np.isfinite(_np(h)), np.isfinite(want))


def _make(rows, D, rps, dt, post, pre, gate, mod, affine, seed=0, wide=0):
    """Tensors of a call; wide > 0: views into buffers with `wide` more columns."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    rnd = lambda *s, dt=torch.float32: torch.empty(*s, device=DEV).normal_(generator=g).to(dt)
    t = TDT[dt]
    samples = -(-rows // rps)
    y, x, xo, h = (rnd(rows, D + wide, dt=k)[:, :D] for k in (t, torch.float32, torch.float32, t))
    mods = rnd(samples, 3 * D + wide) * 0.3
    vecs = []
    for kind in (post, pre):
        on = affine and kind != "none"
        vecs += [(1 + 0.1 * rnd(D)).to(t) if on else None, rnd(D, dt=t) if on and kind == "layer" else None]
    m = (mods[:, :D] if gate else None, mods[:, D:2 * D] if mod else None, mods[:, 2 * D:3 * D] if mod else None)
    return y, x * 2 + 0.5, xo, h, vecs, m


SHAPES = [(1, 1, 1), (1, 1152, 1), (5, 3, 2), (7, 64, 7), (9, 72, 4), (130, 100, 65), (37, 1152, 10), (3, 1154, 2), (6, 2050, 3),
          (5, 2048, 5), (5, 4096, 2), (3, 4100, 1), (2, 6144, 2), (2, 16384, 1), (2, 16383, 2), (1025, 256, 1000)]


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("post,pre,gate,mod,affine,a", [
    ("none", "layer", True, True, False, 1.0), ("rms", "rms", True, False, True, 1.0), ("layer", "none", False, True, True, 0.5),
    ("none", "none", True, False, False, 1.25), ("layer", "layer", True, True, True, 0.0), ("rms", "layer", False, False, False, -1.0)])
@pytest.mark.parametrize("rows,D,rps", SHAPES)
def test_against_float64(bclib, rows, D, rps, post, pre, gate, mod, affine, a, dt):
    y, x, xo, h, vecs, mods = _make(rows, D, rps, dt, post, pre, gate, mod, affine, seed=rows + D)
    _check(bclib, y, x, xo.contiguous(), h, rps, post, pre, a, vecs, mods)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,D,rps,dt", [(6002, 1152, 3001, "bf16"), (2100, 4096, 700, "bf16"), (1300, 4096, 1300, "f32"), (700, 64, 1, "bf16"),
                                           (700, 1156, 3, "f32"), (600, 4092, 2, "bf16"), (1030, 512, 1030, "f32"), (1030, 2048, 103, "bf16"),
                                           (1030, 3064, 515, "f32"), (1100, 2304, 9, "bf16"), (1025, 200, 1, "f32"), (1027, 640, 2, "bf16"), (1025, 500, 3, "f32"),
                                           (1026, 2040, 2, "bf16"), (1025, 3000, 1, "f32"), (1026, 4096, 2, "f32"), (1024, 4096, 1024, "bf16"), (1024, 256, 2, "f32")])
def test_many_rows(bclib, rows, D, rps, dt):
    """Launches past the caches' reach, and many samples of few rows."""
    y, x, xo, h, vecs, mods = _make(rows, D, rps, dt, "layer", "layer", True, True, True, seed=rows)
    _check(bclib, y, x, xo.contiguous(), h, rps, "layer", "layer", 1.0, vecs, mods)


@pytest.mark.gpu
@pytest.mark.parametrize("D,wide", [(64, 8), (64, 3), (1152, 36), (4100, 4), (33, 2)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_strided_rows_leave_the_rest_alone(bclib, D, wide, dt):
    y, x, xo, h, vecs, mods = _make(11, D, 4, dt, "rms", "layer", True, True, True, seed=D, wide=wide)
    xo = torch.full((11, D + wide), 5.0, device=DEV)
    xs = torch.zeros_like(xo)
    xs[:, :D] = x
    hb = torch.full((11, D + wide), 5.0, dtype=TDT[dt], device=DEV)
    _check(bclib, y, xs[:, :D], xo[:, :D], hb[:, :D], 4, "rms", "layer", 1.0, vecs, mods)
    assert bool((xo[:, D:] == 5.0).all()) and bool((hb[:, D:] == 5.0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("rows,rps", [(9, 9), (530, 5), (530, 3)])
@pytest.mark.parametrize("D,wide", [(1, 1), (2, 0), (3, 4), (5, 0), (255, 0), (257, 2), (258, 1), (259, 0), (777, 1), (2047, 0), (2049, 0), (4093, 0)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_widths_without_alignment(bclib, rows, rps, D, wide, dt):
    """Rows of a sample shared by a workgroup or not, at widths around the chunks'
    and the waves' ends; what lies between and behind the rows stays."""
    y, x, _, _, vecs, mods = _make(rows, D, rps, dt, "layer", "rms", True, True, True, seed=rows * D, wide=wide)
    n, ld = rows * (D + wide), D + wide
    xb = torch.full((n + 8,), 5.0, device=DEV)
    hb = torch.full((n + 8,), 5.0, dtype=TDT[dt], device=DEV)
    xs, hs = (b[:n].view(rows, ld) for b in (xb, hb))
    src = torch.zeros(rows, ld, device=DEV)
    src[:, :D] = x
    _check(bclib, y, src[:, :D], xs[:, :D], hs[:, :D], rps, "layer", "rms", 1.0, vecs, mods)
    for b, v in ((xb, xs), (hb, hs)):
        assert bool((v[:, D:] == 5.0).all()) and bool((b[n:] == 5.0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("D", [64, 1152, 4100, 1001])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_in_place_gives_the_same_bits(bclib, D, dt):
    y, x, xo, h, vecs, mods = _make(21, D, 7, dt, "layer", "layer", True, True, True, seed=D)
    args = dict(rows_per_sample=7, post=2, post_w=vecs[0], post_b=vecs[1], gate=mods[0], pre=2, pre_w=vecs[2], pre_b=vecs[3],
                shift=mods[1], scale=mods[2])
    xo, h = xo.contiguous(), h.contiguous()
    bclib.norm_gate_residual(y, x, xo, h, **args)
    x2, y2 = x.clone(), y.clone()
    bclib.norm_gate_residual(y2, x2, x2, y2, **args)
    assert torch.equal(x2, xo) and torch.equal(y2, h)
    # the unaligned path of the same rows, against float64
    if D % 4 == 0:
        buf = torch.empty(21 * D + 1, device=DEV)
        xu = buf[1:].view(21, D)
        xu.copy_(x)
        _check(bclib, y, xu, xu, h, 7, "layer", "layer", 1.0, vecs, mods)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("D", [128, 1152, 5000])
def test_rows_of_one_value_and_rows_that_are_not_finite(bclib, D, dt):
    y, x, xo, h, vecs, mods = _make(8, D, 8, dt, "layer", "layer", True, True, False, seed=D)
    y[1] = 3.0                      # a LayerNorm over equal values gives zeros
    x[2] = 1e4                      # a large common part
    y[2] = 0.0
    y[3, D // 2] = float("inf")
    x[4, 0] = float("nan")
    y[5] = 1e-20
    _check(bclib, y, x, xo.contiguous(), h.contiguous(), 8, "layer", "layer", 1.0, vecs, mods)
    x64 = (x[1].double()).cpu().numpy()
    out = torch.empty_like(x)
    bclib.norm_gate_residual(y, x, out, None, rows_per_sample=8, post=2, gate=mods[0])
    assert np.array_equal(out[1].double().cpu().numpy(), x64)


@pytest.mark.gpu
def test_captured_and_on_another_stream(bclib):
    y, x, xo, h, vecs, mods = _make(300, 1152, 100, "bf16", "rms", "layer", True, True, True)
    xo = xo.contiguous()
    args = dict(rows_per_sample=100, post=1, post_w=vecs[0], gate=mods[0], pre=2, pre_w=vecs[2], pre_b=vecs[3], shift=mods[1], scale=mods[2])
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        bclib.norm_gate_residual(y, x, xo, h, **args)
    for seed in range(3):
        y.normal_()
        x.normal_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        xe, he = torch.empty_like(xo), torch.empty_like(h.contiguous())
        bclib.norm_gate_residual(y, x, xe, he, **args)
        torch.cuda.synchronize()
        assert torch.equal(xe, xo) and torch.equal(he, h)


# Vectors that are infinite, NaN, or whose products leave fp32's range though the
# row's own values do not: what the formula gives, whatever the launch's form (few
# rows, rows that share a sample's vectors or do not, past the caches, any width).
FORMS = [(8, 256, 8), (1100, 256, 550), (1100, 256, 2), (8000, 1152, 4000), (600, 259, 300), (600, 259, 3), (1100, 640, 100), (6, 4100, 3),
         (1100, 4096, 1100)]


def _same_specials(got, want):
    assert np.array_equal(np.isnan(got), np.isnan(want))
    inf = np.isinf(want)
    assert np.array_equal(np.isinf(got), inf) and np.array_equal(got[inf], want[inf])


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("rows,D,rps", FORMS)
def test_gates_out_of_range(bclib, rows, D, rps, kind, dt):
    y, x, xo, _, vecs, (gate, _, _) = _make(rows, D, rps, dt, kind, "none", True, False, True, seed=D + rps)
    w, b = vecs[:2]
    gate = gate.clone()
    gate[:, 1], gate[:, 2], gate[:, 3], gate[0, 4], gate[:, D - 1] = np.inf, -np.inf, np.inf, np.nan, np.inf
    w[3] = 0.0                                            # only the bias is left (RMS: an infinite zero, NaN)
    if b is not None:
        b[2], b[3] = -b[2], 0.5
    if kind == "rms":
        w[6], gate[:, 6], y[:, 6] = 2.0 ** 100, 2.0 ** 30, 2.0 ** -20      # w gate overflows, gate (n w) does not
    xo = xo.contiguous()
    _check(bclib, y, x, xo, None, rps, kind, "none", 1.0, vecs, (gate, None, None))
    with np.errstate(invalid="ignore"):
        want = _np(x) + _np(gate)[np.arange(rows) // rps] * _norm64(_np(y), kind, _np(w), _np(b), 1e-6)[0]
    _same_specials(_np(xo), want)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["none", "rms", "layer"])
@pytest.mark.parametrize("rows,D,rps", FORMS)
def test_scales_and_shifts_out_of_range(bclib, rows, D, rps, kind, dt):
    y, x, xo, h, vecs, (_, shift, scale) = _make(rows, D, rps, dt, "none", kind, False, True, True, seed=D + rps)
    w, b = vecs[2:]
    shift, scale = shift.clone(), scale.clone()
    scale[:, 1], scale[:, 2], scale[:, 3], scale[0, 4], scale[:, D - 1] = np.inf, -np.inf, np.inf, np.nan, np.inf
    shift[:, 7], shift[:, 2] = -np.inf, 3.0
    if w is not None:
        w[3] = 0.0
    if b is not None:
        b[3] = 0.5
    if kind == "rms":
        w[6], scale[:, 6], x[:, 6], y[:, 6] = 2.0 ** 100, 2.0 ** 30, 2.0 ** -20, 0.0
    xo, h = xo.contiguous(), h.contiguous()
    _check(bclib, y, x, xo, h, rps, "none", kind, 1.0, vecs, (None, shift, scale))
    s = np.arange(rows) // rps
    with np.errstate(invalid="ignore"):
        want = _norm64(_np(x) + _np(y), kind, _np(w), _np(b), 1e-6)[0] * (1 + _np(scale)[s]) + _np(shift)[s]
    _same_specials(_np(h), want)


def test_no_rows_need_no_pointers(bclib):
    """An empty tensor has no address; scalars that no call takes are refused all the same."""
    fn = bclib.lib().bc_norm_gate_residual
    none = dict(rows=0, y=None, x=None, x_out=None, h=None)
    for kw in (dict(), dict(pre=2), dict(post=1, post_w=8 << 20), dict(pre=1, scale=8 << 20)):
        assert fn(C.byref(_desc(bclib, **none, **kw)), None) == bclib.OK, kw
    for kw in (dict(D=0), dict(dtype=2), dict(rows_per_sample=0), dict(post=3), dict(eps=0.0), dict(ldy=63)):
        assert fn(C.byref(_desc(bclib, **dict(none, **kw))), None) == bclib.ERR_INVALID_ARG, kw


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_empty_batch(bclib, dt):
    e = lambda n, k=torch.float32: torch.empty(n, 64, dtype=k, device=DEV)
    t, w = TDT[dt], torch.ones(64, dtype=TDT[dt], device=DEV)
    bclib.norm_gate_residual(e(0, t), e(0), e(0), e(0, t), rows_per_sample=7, post=1, post_w=w, gate=e(0), pre=2, pre_w=w, pre_b=w,
                             shift=e(0), scale=e(0))
    bclib.norm_gate_residual(e(0, t), e(0), e(0))
    bclib.norm_gate_residual(e(0, t), e(0), e(0), e(0, t), rows_per_sample=7, gate=e(2), pre=2, shift=e(1), scale=e(1))
    torch.cuda.synchronize()


BIG = [(27000, 252, 999, "bf16"), (13500, 508, 27, "bf16"), (8000, 1152, 1601, "f32"), (3500, 2048, 701, "bf16"), (2400, 2944, 481, "bf16"),
       (3500, 1500, 333, "f32"), (1800, 2944, 355, "f32"), (2600, 2944, 17, "bf16"), (1300, 4000, 650, "f32")]


@pytest.mark.gpu
@pytest.mark.parametrize("rows,D,rps,dt", BIG)
def test_launches_past_the_caches(bclib, rows, D, rps, dt):
    """80 MB of rows or more, samples of 16 rows or more: every count of a lane's
    chunks in that form (1, 2, 5, 8, 12 and 16 of 256 values), those of six to
    twelve by sixteen waves, several samples whose rows do not fill a workgroup's
    waves."""
    assert rows * D * (2 * (2 if dt == "bf16" else 4) + 8) >= 80e6 and rps >= 16 and rps % 16 and -(-rows // rps) > 1
    for post, pre, affine in (("layer", "layer", True), ("none", "rms", False)):
        y, x, xo, h, vecs, mods = _make(rows, D, rps, dt, post, pre, True, True, affine, seed=rows)
        _check(bclib, y, x, xo.contiguous(), h, rps, post, pre, 1.0, vecs, mods)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,rps,more", [(1000, 1000, 0), (1100, 275, 0), (1100, 1, 0), (1100, 1100, 1), (1100, 2, 1)])
def test_rows_beyond_32_bit_offsets(bclib, rows, rps, more):
    """Rows 2^22 values and a few apart: the last one's offset does not fit 32 bits."""
    D, ld = 64, (1 << 22) + 8 + more
    y, x, _, _, vecs, mods = _make(rows, D, rps, "bf16", "layer", "layer", True, True, True, seed=rows + rps)
    far = lambda dt: torch.empty(rows * ld, dtype=dt, device=DEV).as_strided((rows, D), (ld, 1))
    ys, xs, hs = far(torch.bfloat16), far(torch.float32), far(torch.bfloat16)
    ys.copy_(y)
    xs.copy_(x)
    _check(bclib, ys, xs, xs, hs, rps, "layer", "layer", 1.0, vecs, mods)
