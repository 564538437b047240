"""bc_rope and bc_rope_frequencies: refusals and frequencies on the CPU; on the GPU
every layout against float64.

Tolerance, u = 2^-24: sine and cosine are off by at most 4u (the reduced angle's
rounding at pi / 4, the sums and the amplitude), a product and the sum of two by u of
themselves each: 8u (|x_a| + |x_b|) m, and half a step of the output's type."""
import ctypes as C
import math

import numpy as np
import pytest

from oracle import rope as oracle

torch = pytest.importorskip("torch")
DEV = "cuda:0"
TDT = {"f32": torch.float32, "bf16": torch.bfloat16}
FAR = 1 << 24


# ---------------------------------------------------------------------------
# CPU
# ---------------------------------------------------------------------------
def _desc(bc, f, **kw):
    s = dict(B=2, T=5, Hq=4, Hk=2, d=16, dtype=1, q=FAR, k=2 * FAR, q_out=3 * FAR, k_out=4 * FAR, q_batch=5 * 64, q_row=64,
             k_batch=5 * 32, k_row=32, q_out_batch=5 * 64, q_out_row=64, k_out_batch=5 * 32, k_out_row=32, layout=0, axes=1,
             axis_dim=(C.c_int * 3)(16, 0, 0), freqs=f.ctypes.data, amplitude=1.0, inverse=0, pos=5 * FAR, pos_batch=5, start=0)
    s.update(kw)
    if not isinstance(s["axis_dim"], C.Array):
        s["axis_dim"] = (C.c_int * 3)(*s["axis_dim"])
    return bc.RopeDesc(**s)


def test_refusals(bclib):
    bad, no = bclib.ERR_INVALID_ARG, bclib.ERR_UNSUPPORTED
    f = np.ones(128)
    cases = [(dict(B=-1), bad), (dict(T=-1), bad), (dict(Hq=0), bad), (dict(Hk=-1), bad), (dict(d=0), bad), (dict(d=258), no),
             (dict(Hq=4096), no), (dict(dtype=2), bad), (dict(layout=2), bad), (dict(axes=0), bad), (dict(axes=4), bad),
             (dict(axis_dim=(15, 0, 0)), bad), (dict(axis_dim=(18, 0, 0)), bad), (dict(axis_dim=(0, 0, 0)), bad),
             (dict(axes=2, axis_dim=(8, 10, 0)), bad), (dict(axes=2, axis_dim=(8, 8, 0), pos=None), bad), (dict(freqs=None), bad),
             (dict(amplitude=math.nan), bad), (dict(amplitude=math.inf), bad), (dict(pos=5 * FAR + 2), bad), (dict(pos_batch=-1), bad),
             (dict(start=1 << 41), bad), (dict(q=None), bad), (dict(q_out=None), bad), (dict(k=None), bad), (dict(k_out=None), bad),
             (dict(q=FAR + 1), bad), (dict(k_out=4 * FAR + 1), bad), (dict(q_row=-64), bad), (dict(k_batch=-1), bad),
             (dict(q_out_row=63), bad), (dict(q_out_batch=4 * 64 + 63), bad),
             # an output on another operand, or on the positions
             (dict(q_out=FAR + 2), bad), (dict(q_out=2 * FAR), bad), (dict(k_out=3 * FAR + 64), bad), (dict(k_out=FAR), bad),
             (dict(k_out=5 * FAR), bad), (dict(q_out=FAR, q_out_row=128, q_out_batch=640), bad),
             # views of one projection's rows that meet: 64 + 32 columns of 96, the keys at column 60
             (dict(q_row=96, q_batch=480, k_row=96, k_batch=480, q_out=FAR, q_out_row=96, q_out_batch=480, k=FAR + 2 * 60, k_out=FAR + 2 * 60,
                   k_out_row=96, k_out_batch=480), bad)]
    for kw, want in cases:
        assert bclib.lib().bc_rope(C.byref(_desc(bclib, f, **kw)), None) == want, kw
    for x in (math.nan, math.inf, 1e7):
        g = np.ones(128)
        g[3] = x
        assert bclib.lib().bc_rope(C.byref(_desc(bclib, g)), None) == bad, x
    assert bclib.lib().bc_rope(None, None) == bad
    for kw in (dict(B=0), dict(T=0), dict(T=0, q=None, k=None, q_out=None, k_out=None)):
        assert bclib.lib().bc_rope(C.byref(_desc(bclib, f, **kw)), None) == bclib.OK, kw


def test_strides_whose_offsets_pass_64_bits_are_refused(bclib):
    f = np.ones(128)
    for kw in (dict(B=1 << 20, q_batch=1 << 48), dict(B=1 << 20, k_batch=1 << 48), dict(T=1 << 30, q_row=1 << 32), dict(B=1 << 20, q_out_batch=1 << 48),
               dict(pos_batch=1 << 62), dict(B=1 << 20, pos_batch=1 << 40)):
        assert bclib.lib().bc_rope(C.byref(_desc(bclib, f, **kw)), None) == bclib.ERR_INVALID_ARG, kw


def test_binding_refuses_what_are_no_numbers(bclib):
    q = torch.zeros(1, 5, 4, 16)
    for kw in (dict(freqs=3.0), dict(freqs=["a"] * 8), dict(freqs=None), dict(freqs=[1.0] * 8, start=1 << 70)):
        with pytest.raises(bclib.BCError) as e:
            bclib.rope(q, q.clone(), **kw)
        assert e.value.code == bclib.ERR_INVALID_ARG, kw


def test_frequencies(bclib):
    for n in (2, 4, 16, 56, 128, 256):
        for theta in (256.0, 10000.0, 1e6):
            for kw in (dict(), dict(scaling="linear", factor=8.0), dict(scaling="ntk", factor=4.0),
                       dict(scaling="parts", factor=16.0, original=4096), dict(scaling="parts", factor=2.0, original=100, beta_fast=8.0, beta_slow=2.0)):
                got, want = bclib.rope_frequencies(n, theta, **kw), oracle.frequencies(n, theta, **kw)
                assert np.all(np.abs(got - want) <= 1e-13 * want), (n, theta, kw)
    # By hand: 4 columns, theta 10000: 1 and 0.01; over 6283 positions 1000 and 10 turns, so the second pair keeps 9 / 31.
    got = bclib.rope_frequencies(4, 10000.0, scaling="parts", factor=4.0, original=6283)
    keep = (62.83 / (2 * math.pi) - 1) / 31
    assert got[0] == 1.0 and abs(got[1] - 0.01 * (keep + (1 - keep) / 4)) < 1e-15
    out = np.zeros(4)
    ok = (8, 100.0, 3, 2.0, 100, 32.0, 1.0, out.ctypes.data)
    fn = bclib.lib().bc_rope_frequencies
    assert fn(*ok) == bclib.OK
    for i, v in [(0, 7), (0, 0), (0, 258), (1, 0.0), (1, math.nan), (1, math.inf), (2, 4), (2, -1), (3, 0.5), (3, math.nan), (3, math.inf), (4, 0),
                 (5, 1.0), (5, math.nan), (6, -1.0), (7, None)]:
        assert fn(*[v if j == i else x for j, x in enumerate(ok)]) == bclib.ERR_INVALID_ARG, (i, v)


def test_binding_refuses_tensors_that_do_not_fit(bclib):
    q, k, f = torch.zeros(2, 5, 4, 16), torch.zeros(2, 5, 2, 16), np.ones(8)
    pos = torch.zeros(2, 5, dtype=torch.int32)
    ok = dict(q=q, q_out=q.clone(), freqs=f, k=k, k_out=k.clone(), pos=pos)
    for kw in (dict(q_out=q[:, :4]), dict(q_out=q.bfloat16()), dict(k=None), dict(k=k.bfloat16()), dict(k=k[:1]), dict(k=k[..., :8]),
               dict(q=q.transpose(1, 2)), dict(q=q[..., ::2]), dict(pos=pos.long()), dict(pos=pos[:, :4]), dict(pos=pos.t()), dict(axes=[8, 4]),
               dict(axes=[4, 4, 4, 4]), dict(axes=[]), dict(layout="whole"), dict(axes=[8, 8]), dict(freqs=np.ones((2, 4)))):
        with pytest.raises(bclib.BCError) as e:
            bclib.rope(**dict(ok, **kw))
        assert e.value.code == bclib.ERR_INVALID_ARG, kw
    with pytest.raises(bclib.BCError) as e:                                               # tensors of the host
        bclib.rope(**ok)
    assert e.value.code == bclib.ERR_INVALID_ARG
    with pytest.raises(bclib.BCError):
        bclib.rope_frequencies(8, scaling="other")


def test_packed_descriptors_lie_as_the_structures_do(bclib):
    """The binding packs descriptors as bytes: every field where the structure has it."""
    for cls, pack in ((bclib.RopeDesc, bclib._ROPE_PACK), (bclib.ScoreOpts, bclib._OPTS_PACK), (bclib.MaskedDesc, bclib._MASKED_PACK)):
        assert pack.size == C.sizeof(cls)

        def leaves(x):
            for name, kind in x._fields_:
                v = getattr(x, name)
                if isinstance(v, C.Structure):
                    yield from leaves(v)
                else:
                    yield from v if isinstance(v, C.Array) else (v,)

        n = len(list(leaves(cls())))
        assert list(leaves(cls.from_buffer_copy(pack.pack(*range(1, n + 1))))) == list(range(1, n + 1)), cls


def test_oracle():
    """Turning back gives the input; lengths are kept; a score depends on the distance alone."""
    g = np.random.default_rng(0)
    f = np.concatenate([oracle.frequencies(4, 100.0), oracle.frequencies(2, 256.0)])
    x, pos = g.standard_normal((1, 7, 2, 8)), g.integers(0, 50, (1, 7, 2))
    for layout in ("pairs", "halves"):
        y = oracle.turn(x, pos, [4, 2], f, layout)
        assert np.allclose(oracle.turn(y, pos, [4, 2], f, layout, inverse=True), x)
        assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1)) and np.array_equal(y[..., 6:], x[..., 6:])
        same = np.repeat(x[:, :1], 7, 1)
        at = np.arange(7)[None, :, None] * np.ones((1, 1, 2))
        a, b = oracle.turn(same, at, [4, 2], f, layout), oracle.turn(same, at + 3, [4, 2], f, layout)
        assert np.allclose((a[0, 0] * a[0, 5]).sum(), (b[0, 0] * b[0, 5]).sum())


# ---------------------------------------------------------------------------
# GPU
# ---------------------------------------------------------------------------
def _np(t):
    return t.double().cpu().numpy()


def _tol(x, want, axes, layout, m, dt):
    """Of every output: 8u (|x_a| + |x_b|) m for the turned columns, and half a step."""
    mag, col = np.zeros(x.shape), 0
    for n in axes:
        a = slice(col, col + n, 2) if layout == "pairs" else slice(col, col + n // 2)
        b = slice(col + 1, col + n, 2) if layout == "pairs" else slice(col + n // 2, col + n)
        mag[..., a] = mag[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
        col += n
    raw = 8 * 2.0 ** -24 * m * mag
    return raw + (2.0 ** -8 if dt == "bf16" else 2.0 ** -24) * (np.abs(want) + raw) * (mag > 0)


def _check(bc, B, T, Hq, Hk, d, axes, layout, dt, m=1.0, far=0, view=0, in_place=False, inverse=False, shared=False, seed=0):
    """view: 0 contiguous rows; else columns into a row of all heads and `view` - 1 values between rows (odd: unaligned)."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    width = (Hq + Hk) * d + (view - 1 if view else 0)
    buf = torch.empty(B * T * width, device=DEV).normal_(generator=g).to(TDT[dt])
    x = buf.view(B, T, width)
    q = x[..., :Hq * d].unflatten(-1, (Hq, d))
    k = x[..., Hq * d:(Hq + Hk) * d].unflatten(-1, (Hk, d)) if Hk else None
    if not view:
        q, k = q.contiguous(), k.contiguous() if Hk else None
    f = np.concatenate([oracle.frequencies(n, 256.0 if len(axes) > 1 else 10000.0) for n in axes])
    shape = (T, len(axes)) if shared else (B, T, len(axes))
    pos = torch.randint(0, 4000, shape, generator=g, device=DEV).to(torch.int32) + far
    qn, kn, pn = _np(q), _np(k) if Hk else None, np.broadcast_to(pos.cpu().numpy(), (B, T, len(axes)))
    before = buf.clone()
    if in_place:
        q_out, k_out, guard = q, k, None
    else:
        guard = torch.full((B * T * (Hq + Hk) * d + 64,), 9.0, device=DEV, dtype=TDT[dt])
        q_out = guard[32:32 + B * T * Hq * d].view(B, T, Hq, d)
        k_out = guard[32 + B * T * Hq * d:-32].view(B, T, Hk, d) if Hk else None
    bc.rope(q, q_out, f, k=k, k_out=k_out, pos=pos if len(axes) > 1 or shared else pos[..., 0].contiguous(), axes=axes, layout=layout, amplitude=m,
            inverse=inverse)
    torch.cuda.synchronize()
    for got, xn in ((q_out, qn), (k_out, kn)):
        if got is None:
            continue
        want = oracle.turn(xn, pn, axes, f, layout, m, inverse)
        err, tol = np.abs(_np(got) - want), _tol(xn, want, axes, layout, abs(m), dt)
        assert np.all(err <= tol), float((err - tol).max())
    if guard is not None:
        assert bool((guard[:32] == 9).all()) and bool((guard[-32:] == 9).all())
        assert torch.equal(buf, before)
    elif view > 1:
        assert torch.equal(buf.view(B, T, width)[..., (Hq + Hk) * d:], before.view(B, T, width)[..., (Hq + Hk) * d:])


ROPE = [  # B, T, Hq, Hk, d, axes, far
    (1, 1, 1, 0, 2, [2], 0), (1, 1, 16, 16, 72, [72], 100_000), (2, 7, 3, 1, 64, [64], 0), (3, 33, 4, 4, 64, [48], 10), (1, 129, 24, 24, 128, [16, 56, 56], 0),
    (2, 50, 5, 5, 96, [32, 32, 32], 0), (1, 700, 2, 1, 32, [16, 16], 3), (1, 3, 6, 2, 50, [50], 0), (2, 19, 3, 3, 66, [22, 44], 1 << 20),
    (4, 1, 32, 8, 128, [128], 2_000_000), (1, 2000, 1, 0, 8, [8], 0), (1, 40, 2, 2, 256, [256], 77), (2, 9, 3, 2, 7, [4], 0), (1, 11, 128, 8, 128, [64], 5)]


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["pairs", "halves"])
@pytest.mark.parametrize("B,T,Hq,Hk,d,axes,far", ROPE)
def test_rope(bclib, B, T, Hq, Hk, d, axes, far, layout, dt):
    _check(bclib, B, T, Hq, Hk, d, axes, layout, dt, far=far, seed=T + d)
    for view in (1, 2, 9):
        _check(bclib, B, T, Hq, Hk, d, axes, layout, dt, m=1.25, far=far, view=view, in_place=view != 2, inverse=view == 9, shared=view == 1, seed=T)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("d,axes", [(96, (24,)), (36, (24, 8)), (60, (20, 12)), (72, (16, 24, 24)), (50, (12, 28))])
@pytest.mark.parametrize("view", [0, 5, 3, 2])
def test_pieces_of_every_size(bclib, view, d, axes, layout, dt):
    """Halves, heads and rows that are multiples of 8, 4, 2 columns or of none."""
    _check(bclib, 2, 37, 3, 2, d, axes, layout, dt, m=1.25, view=view, in_place=view == 5, seed=d + view)


def test_binding_takes_shared_positions_whatever_the_batch(bclib):
    """[T, axes] and [T] are taken for every number of samples: what is left to refuse are the tensors of the host."""
    for n, B in ((1, 1), (1, 2), (1, 3), (2, 1), (2, 2), (2, 3), (3, 2), (3, 3)):
        for T in (1, 2, 3):
            q = torch.zeros(B, T, 2, 16)
            pos = torch.zeros(T, n, dtype=torch.int32)
            for p in (pos, pos.expand(B, T, n).contiguous(), *((pos[:, 0].contiguous(), pos[:, 0].expand(B, T).contiguous()) if n == 1 else ())):
                with pytest.raises(bclib.BCError) as e:
                    bclib.rope(q, q.clone(), np.ones(2 * n), pos=p, axes=[4] * n)
                assert "current device" in str(e.value), (n, B, T, p.shape)


@pytest.mark.gpu
@pytest.mark.parametrize("B,T,axes", [(2, 2, [8, 8]), (3, 3, [8, 4, 4]), (3, 3, [16]), (2, 3, [8, 4, 4]), (1, 1, [16]), (2, 1, [4, 8])])
def test_shared_positions(bclib, B, T, axes):
    """As many samples as tokens and axes, among others."""
    _check(bclib, B, T, 3, 2, 20, axes, "halves", "bf16", shared=True, seed=B)
    _check(bclib, B, T, 3, 2, 20, axes, "halves", "bf16", shared=False, seed=B)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_without_positions_tokens_run_from_start(bclib, dt):
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    q = torch.empty((2, 37, 3, 64), device=DEV).normal_(generator=g).to(TDT[dt])
    f = oracle.frequencies(64, 10000.0)
    a, b = torch.empty_like(q), torch.empty_like(q)
    for start in (0, 1000, -5, 3_000_000_000):
        bclib.rope(q, a, f, start=start)
        want = oracle.turn(_np(q), np.broadcast_to(np.arange(37)[None, :, None] + start, (2, 37, 1)), [64], f, "pairs")
        assert np.all(np.abs(_np(a) - want) <= _tol(_np(q), want, [64], "pairs", 1.0, dt)), start
    bclib.rope(q, a, f, start=1000)
    bclib.rope(q, b, f, pos=torch.arange(1000, 1037, dtype=torch.int32, device=DEV))
    assert torch.equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["pairs", "halves"])
def test_gradient(bclib, layout):
    """The gradient of sum(y w) is w turned back: against the formula's (autograd in 64 bits on the CPU) and differences."""
    g = torch.Generator(device=DEV)
    g.manual_seed(2)
    x, w = (torch.empty((1, 9, 2, 16), device=DEV).normal_(generator=g) for _ in range(2))
    f = oracle.frequencies(12, 100.0)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    bclib.rope(w, dx, f, layout=layout, amplitude=1.5, inverse=True)
    x64 = x.double().cpu().requires_grad_()
    phi = torch.arange(9, dtype=torch.float64)[None, :, None, None] * torch.from_numpy(f)
    a, b = (slice(0, 12, 2), slice(1, 12, 2)) if layout == "pairs" else (slice(0, 6), slice(6, 12))
    out = torch.zeros_like(x64) + torch.nn.functional.pad(x64[..., 12:], (12, 0))
    out[..., a] = 1.5 * (x64[..., a] * torch.cos(phi) - x64[..., b] * torch.sin(phi))
    out[..., b] = 1.5 * (x64[..., a] * torch.sin(phi) + x64[..., b] * torch.cos(phi))
    (out * w.double().cpu()).sum().backward()
    assert np.all(np.abs(_np(dx) - x64.grad.numpy()) <= _tol(_np(w), _np(dx), [12], layout, 1.5, "f32"))
    for at in ((0, 3, 1, 2), (0, 8, 0, 9), (0, 5, 1, 14)):
        d = torch.zeros_like(x)
        d[at] = 0.5                                       # linear: any step is exact but for rounding
        lo, hi = torch.empty_like(x), torch.empty_like(x)
        bclib.rope(x - d, lo, f, layout=layout, amplitude=1.5)
        bclib.rope(x + d, hi, f, layout=layout, amplitude=1.5)
        slope = float(((hi.double() - lo.double()) * w.double()).sum())
        assert abs(slope - float(dx[at])) <= 1e-5, at
    bclib.rope(x, y, f, layout=layout)
    bclib.rope(y, y, f, layout=layout, inverse=True)
    assert float((y - x).abs().max()) <= 32 * 2.0 ** -24 * float(x.abs().max())


@pytest.mark.gpu
def test_not_finite_values_stay_in_their_pair(bclib):
    for dt in TDT.values():
        q = torch.ones((1, 3, 2, 32), device=DEV, dtype=dt)
        q[0, 1, 0, 3], q[0, 1, 1, 30], q[0, 2, 1, 31] = math.nan, math.inf, math.nan
        out = torch.empty_like(q)
        bclib.rope(q, out, oracle.frequencies(28, 100.0), start=1)
        bad = ~torch.isfinite(out)
        assert bad[0, 1, 0, 2:4].all() and torch.equal(out[..., 28:].isnan(), q[..., 28:].isnan()) and math.isinf(float(out[0, 1, 1, 30]))
        assert int(bad.sum()) == 4


@pytest.mark.gpu
def test_rows_beyond_32_bit_offsets(bclib):
    """Rows of 2^27 values: the last one starts past 2^32 bytes."""
    T, row = 20, 1 << 27
    x = torch.empty(T * row, dtype=torch.bfloat16, device=DEV).view(1, T, row)
    q = x[..., :128].unflatten(-1, (2, 64))
    q.copy_(torch.randn(1, T, 2, 64, generator=torch.Generator().manual_seed(0)).to(DEV))
    want = oracle.turn(_np(q), np.arange(T)[None, :, None], [64], oracle.frequencies(64, 1e4), "halves")
    qn = _np(q)
    bclib.rope(q, q, oracle.frequencies(64, 1e4), layout="halves")
    assert np.all(np.abs(_np(q) - want) <= _tol(qn, want, [64], "halves", 1.0, "bf16"))


@pytest.mark.gpu
def test_other_streams_and_captured_graphs(bclib):
    q = torch.randn(2, 65, 4, 72, device=DEV).bfloat16()
    pos = torch.arange(130, dtype=torch.int32, device=DEV).view(2, 65)
    f = bclib.rope_frequencies(72)
    want, out = torch.empty_like(q), torch.empty_like(q)
    bclib.rope(q, want, f, pos=pos)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    bclib.rope(q, out, f, pos=pos, stream=s)
    s.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        bclib.rope(q, out, f, pos=pos)
    for step in range(3):                                 # positions are read when it runs
        f2 = f.copy()
        graph.replay()
        bclib.rope(q, want, f2, pos=pos)
        torch.cuda.synchronize()
        assert torch.equal(out, want), step
        pos += 1000
        f[:] = 0.0                                        # frequencies when it was recorded
        f = f2
