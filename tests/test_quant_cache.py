"""Quantised cache rings (bc_cache_create_quant): refusals on the CPU; on the
GPU the codes, the forecast from them, and sampling runs with such a ring,
against the float64 oracle.

Tolerances.  A value reads back as fl(code * s), one fp32 rounding of the
oracle's product.  A forecast rounds each weight to fp32, each weight times
scale, and each FMA once: at most (K + 2) half steps of 2^-24 of sum |w q s|
(doubled below for the oracle's own scale of the sum), and a bf16 output half a
step of 2^-8 more."""
import ctypes as C
import math

import numpy as np
import pytest

import synth
from oracle import bary, model as om, quant, sampler as osm

torch = pytest.importorskip("torch")
DEV = "cuda:0"
TDT = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------------------
# CPU: sizes and refusals (host metadata only; no address is followed)
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("n", [1, 63, 64, 65, 1000, 14310 * 1152])
def test_storage_size(bclib, n, bits):
    groups = -(-n // 64)
    up = lambda v: -(-v // 256) * 256
    for K in (1, 3, 8):
        assert bclib.quant_cache_bytes(K, n, bits) == K * (up(groups * 8 * bits) + up(groups * 4))


def _create(bclib, K=2, n=100, dtype=0, bits=8, storage=4096):
    h = C.c_void_p()
    rc = bclib.lib().bc_cache_create_quant(K, n, dtype, bits, storage, C.byref(h))
    return rc, h


def test_refusals_on_creation(bclib):
    bad = bclib.ERR_INVALID_ARG
    L = bclib.lib()
    for kw in (dict(K=0), dict(K=9), dict(n=0), dict(n=-5), dict(n=1 << 41), dict(dtype=2), dict(dtype=-1), dict(bits=0), dict(bits=5),
               dict(bits=16), dict(storage=None), dict(storage=4096 + 8)):
        rc, h = _create(bclib, **kw)
        assert rc == bad and not h.value, kw
    assert L.bc_cache_create_quant(2, 100, 0, 8, 4096, None) == bad
    n = C.c_size_t()
    for args in ((0, 10, 8), (9, 10, 8), (2, 0, 8), (2, 10, 3), (2, 1 << 41, 4)):
        assert L.bc_cache_quant_storage_size(*args, C.byref(n)) == bad
    assert L.bc_cache_quant_storage_size(2, 10, 8, None) == bad


def test_refusals_on_use(bclib):
    """Every call here is refused before anything is enqueued."""
    L = bclib.lib()
    rc, h = _create(bclib)
    assert rc == bclib.OK
    p = C.c_void_p()
    w = (C.c_double * 2)(1.0, 0.0)
    assert L.bc_cache_next_slot(h, C.byref(p)) == bclib.ERR_UNSUPPORTED
    assert L.bc_cache_push(h, None, 0.0, None) == bclib.ERR_INVALID_ARG
    assert L.bc_cache_push(h, 4096, math.nan, None) == bclib.ERR_INVALID_ARG
    assert L.bc_cache_read(h, 0, 4096, 0, None) == bclib.ERR_STATE        # empty
    assert L.bc_bary_extrapolate(h, w, 1, 4096, 0, None) == bclib.ERR_STATE
    for node, out, dt in ((-1, 4096, 0), (2, 4096, 0), (0, None, 0), (0, 4096, 7)):
        assert L.bc_cache_read(h, node, out, dt, None) == bclib.ERR_INVALID_ARG
    assert L.bc_cache_read(None, 0, 4096, 0, None) == bclib.ERR_INVALID_ARG
    for feat in (4096, 4096 + 400, 4096 - 396):                           # a feature that lies in the storage
        assert L.bc_cache_push(h, feat, 0.0, None) == bclib.ERR_INVALID_ARG
    for feat in ((1 << 20) + 1, (1 << 20) + 2):                           # not aligned to its elements
        assert L.bc_cache_push(h, feat, 0.0, None) == bclib.ERR_INVALID_ARG
    cnt = C.c_int(-1)
    assert L.bc_cache_state(h, C.byref(cnt), None, None, None) == bclib.OK and cnt.value == 0
    assert L.bc_cache_reset(h) == bclib.OK and L.bc_cache_destroy(h) == bclib.OK


def test_binding_refuses_tensors_that_do_not_fit(bclib):
    n = bclib.quant_cache_bytes(2, 100, 8)
    store = torch.empty(n + 64, dtype=torch.uint8)
    store = store[(-store.data_ptr()) % 16:][:n]
    ring = bclib.QuantCacheRing(2, 100, torch.float32, 8, store)
    for feat in (None, torch.zeros(99), torch.zeros(100, dtype=torch.bfloat16), torch.zeros(200)[::2]):
        with pytest.raises(bclib.BCError) as e:
            ring.push(feat, 0.0)
        assert e.value.code == bclib.ERR_INVALID_ARG
    for out in (torch.zeros(99), torch.zeros(200)[::2]):
        for call in (lambda: ring.read(0, out), lambda: bclib.bary_extrapolate(ring, [1.0], out)):
            with pytest.raises(bclib.BCError) as e:
                call()
            assert e.value.code == bclib.ERR_INVALID_ARG
    with pytest.raises(bclib.BCError) as e:                                              # a tensor of the host
        ring.push(torch.zeros(100), 0.0)
    assert e.value.code == bclib.ERR_INVALID_ARG and ring.state()[0] == 0
    for bad in (store[:n - 1], torch.empty(2 * n, dtype=torch.uint8)[::2]):
        with pytest.raises(bclib.BCError):
            bclib.QuantCacheRing(2, 100, torch.float32, 8, bad)
    with pytest.raises(bclib.BCError):
        bclib.QuantCacheRing(2, 100, torch.float16, 8, store)


def test_oracle_codes_by_hand():
    """A worked group: max 254 at 8 bits, so s = 2 and odd values are ties."""
    x = np.zeros(70, np.float32)
    x[:6] = [254.0, 1.0, 3.0, 5.0, -1.0, -3.0]
    x[64:] = [7.0, 0.5, 1.5, -0.5, -1.5, 0.0]
    assert list(quant.held(x, 8)[:6]) == [254.0, 0.0, 4.0, 4.0, 0.0, -4.0]
    assert list(quant.held(x, 4)[64:]) == [7.0, 0.0, 2.0, 0.0, -2.0, 0.0]


# ---------------------------------------------------------------------------
# GPU
# ---------------------------------------------------------------------------
def _feature(n, dt, seed, special=True):
    g = np.random.default_rng(seed)
    x = (g.standard_normal(n) * np.exp(g.standard_normal(n))).astype(np.float32)
    if special:
        for at in range(0, n, 64):
            k = (at // 64) % 8
            v = x[at:at + 64]
            if k == 1:
                v[:] = 0.0
            elif k == 2:                                  # every code and every tie at a scale of 2^-3
                v[:] = (np.arange(len(v)) * 2 - 63) * 2.0 ** -4
                v[0] = 127 * 2.0 ** -3
            elif k == 3:
                v[:] = v * np.float32(2.0 ** -118)        # near the smallest scale
            elif k == 4:
                v[:] = v * np.float32(1e30)
            elif k == 5:
                v[:] = 0.0
                v[len(v) // 2] = -3.0
    return synth.bf16_round(x) if dt == "bf16" else x


def _dev(x, dt):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV).to(TDT[dt])


def _qring(bc, K, n, dt, bits, guard=512):
    need = bc.quant_cache_bytes(K, n, bits)
    buf = torch.full((need + 2 * guard,), 0xA5, dtype=torch.uint8, device=DEV)
    return bc.QuantCacheRing(K, n, TDT[dt], bits, buf[guard:guard + need]), buf, guard


def _guards_kept(buf, guard):
    return bool((buf[:guard] == 0xA5).all()) and bool((buf[-guard:] == 0xA5).all())


NS = [1, 7, 63, 64, 65, 512, 513, 2047, 4096 + 72, 100003]


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n", NS)
def test_reads_back_what_the_definition_holds(bclib, n, dt, bits):
    x = _feature(n, dt, seed=n)
    ring, buf, guard = _qring(bclib, 2, n, dt, bits)
    first = _feature(n, dt, seed=n + 1)
    ring.push(_dev(first, dt), 0.0)
    ring.push(_dev(x, dt), 1.0)
    for node, src in ((0, x), (1, first)):
        out = torch.empty(n, device=DEV)
        ring.read(node, out)
        want = quant.held(src, bits)
        assert np.array_equal(out.cpu().numpy(), want.astype(np.float32))      # the codes exactly, one rounding of the product
        low = torch.empty(n, dtype=torch.bfloat16, device=DEV)
        ring.read(node, low)
        assert bool((low == out.bfloat16()).all())
        step = quant.codes(src, bits)[1].repeat(64)[:n]
        kept = step > 0
        assert np.all(np.abs(want - src)[kept] <= step[kept] * 0.5 * (1 + 1e-6))
    assert _guards_kept(buf, guard)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("bits", [8, 4])
def test_every_mantissa_against_every_largest_one(bclib, bits, dt):
    """All pairs of 8-bit mantissas down to quotients below a half, both signs: every
    tie, and every quotient next to one, that bf16 features can hold."""
    m = np.arange(128, 256, dtype=np.float64)
    x = (m[:, None] * 2.0 ** -np.arange(9 if bits == 8 else 5)).ravel()
    x = np.concatenate([x, -x])
    x = np.concatenate([x, np.zeros(-len(x) % 63)]).reshape(-1, 63)
    groups = []
    for k, a in enumerate(m):
        scale = 2.0 ** ((k % 5) * 20 - 40)
        g = np.concatenate([np.full((len(x), 1), a if k % 2 else -a), np.where(np.abs(x) <= a, x, 0.0)], axis=1)
        groups.append(np.roll(g, k, axis=1) * scale)
    feat = np.concatenate(groups).ravel().astype(np.float32)
    assert np.array_equal(feat, synth.bf16_round(feat))
    n, s = quant.codes(feat, bits)                        # the definition in exact integers times a power of two: 2|x| against (2k + 1) s
    a, q = np.abs(feat.astype(np.float64)).reshape(-1, 64), np.abs(n)
    assert np.all(2 * a <= (2 * q + 1) * s) and np.all(2 * a >= (2 * q - 1) * s)
    tie = (2 * a == (2 * q + 1) * s) | (2 * a == (2 * q - 1) * s)
    assert tie.any() and not (q[tie] % 2).any()
    ring, buf, guard = _qring(bclib, 1, feat.size, dt, bits)
    ring.push(_dev(feat, dt), 0.0)
    out = torch.empty(feat.size, device=DEV)
    ring.read(0, out)
    assert np.array_equal(out.cpu().numpy(), (n * s).ravel().astype(np.float32))
    assert _guards_kept(buf, guard)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [8, 4])
def test_long_features(bclib, bits):
    """Long bf16 features, whose writing and reading take their own paths, with a ragged end."""
    n, K = (16 << 20) + 77, 3
    ring, buf, guard = _qring(bclib, K, n, "bf16", bits)
    feats = [_feature(n, "bf16", seed=j, special=j == 0) for j in range(K)]
    for j in reversed(range(K)):
        ring.push(_dev(feats[j], "bf16"), float(-j))
    out = torch.empty(n, device=DEV)
    held = []
    for j in range(K):
        ring.read(j, out)
        held.append(quant.held(feats[j], bits).astype(np.float32))
        assert np.array_equal(out.cpu().numpy(), held[j]), j
    w = [1.75, -1.0, 0.25]
    low = torch.empty(n, dtype=torch.bfloat16, device=DEV)
    bclib.bary_extrapolate(ring, w, out)
    bclib.bary_extrapolate(ring, w, low)
    want = sum(a * h.astype(np.float64) for a, h in zip(w, held))
    tol = 2 * (K + 2) * 2.0 ** -24 * sum(abs(a) * np.abs(h.astype(np.float64)) for a, h in zip(w, held))
    assert np.all(np.abs(out.cpu().numpy() - want) <= tol)
    assert bool((low == out.bfloat16()).all())
    assert _guards_kept(buf, guard)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_unaligned_feature_and_output(bclib, dt, bits):
    n = 1000
    x = _feature(n, dt, seed=3)
    ring, buf, guard = _qring(bclib, 1, n, dt, bits)
    for off in (0, 1, 3):
        src = torch.zeros(n + 8, dtype=TDT[dt], device=DEV)
        src[off:off + n] = _dev(x, dt)
        src[off + n:] = float("nan")                       # behind the feature: not read
        ring.push(src[off:off + n], 0.0)
        for odt in ("f32", "bf16"):
            out = torch.full((n + 8,), 7.0, dtype=TDT[odt], device=DEV)
            ring.read(0, out[off:off + n])
            want = _dev(quant.held(x, bits).astype(np.float32), odt)
            assert bool((out[off:off + n] == want).all())
            assert bool((out[:off] == 7.0).all()) and bool((out[off + n:] == 7.0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [8, 4])
def test_values_that_are_not_finite_stay_visible(bclib, bits):
    n = 64 * 5 + 10
    x = _feature(n, "f32", seed=9, special=False)
    x[3] = np.inf
    x[64 + 63] = np.nan
    x[128 + 5] = -np.inf
    x[-1] = np.nan
    ring, _, _ = _qring(bclib, 1, n, "f32", bits)
    ring.push(_dev(x, "f32"), 0.0)
    out = torch.empty(n, device=DEV)
    ring.read(0, out)
    got, want = out.cpu().numpy(), quant.held(x, bits)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.isnan(got[:192]).all() and np.isnan(got[320:]).all() and np.isfinite(got[192:320]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("K", range(1, 9))
@pytest.mark.parametrize("dt,odt,n", [("f32", "f32", 5003), ("bf16", "bf16", 64 * 129), ("bf16", "f32", 777), ("f32", "bf16", 1)])
def test_forecast_from_codes(bclib, K, dt, odt, n, bits):
    feats = [_feature(n, dt, seed=10 * K + j, special=False) for j in range(K)]
    g = np.random.default_rng(K)
    w = g.standard_normal(K)
    w /= w.sum()
    ring, buf, guard = _qring(bclib, K, n, dt, bits)
    for j in reversed(range(K)):
        ring.push(_dev(feats[j], dt), float(-j))
    out = torch.empty(n, dtype=TDT[odt], device=DEV)
    bclib.bary_extrapolate(ring, w, out)
    held = [quant.held(f, bits) for f in feats]
    want = sum(a * f for a, f in zip(w, held))
    scale = sum(abs(a) * np.abs(f) for a, f in zip(w, held))
    tol = 2 * (K + 2) * 2.0 ** -24 * scale
    if odt == "bf16":
        tol = tol + np.abs(want) * 2.0 ** -8 * 1.01
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= tol)
    assert _guards_kept(buf, guard)


@pytest.mark.gpu
def test_ring_wraps_and_forecasts_fewer_nodes(bclib):
    n, K = 3000, 3
    ring, _, _ = _qring(bclib, K, n, "f32", 8)
    feats = [_feature(n, "f32", seed=j, special=False) for j in range(5)]
    for j in range(5):
        ring.push(_dev(feats[j], "f32"), float(j))
    cnt, head, tn, slots = ring.state()
    assert (cnt, head, list(tn), list(slots)) == (3, 1, [4.0, 3.0, 2.0], [1, 0, 2])
    out = torch.empty(n, device=DEV)
    for node in range(3):
        ring.read(node, out)
        assert np.array_equal(out.cpu().numpy(), quant.held(feats[4 - node], 8).astype(np.float32))
    bclib.bary_extrapolate(ring, [1.5, -0.5], out)
    want = 1.5 * quant.held(feats[4], 8) - 0.5 * quant.held(feats[3], 8)
    assert np.abs(out.cpu().numpy() - want).max() <= 1e-6 * np.abs(want).max()
    with pytest.raises(bclib.BCError):
        bclib.bary_extrapolate(ring, [0.25] * 4, out)
    ring.reset()
    with pytest.raises(bclib.BCError) as e:
        ring.read(0, out)
    assert e.value.code == bclib.ERR_STATE


@pytest.mark.gpu
def test_outputs_in_the_storage_are_refused(bclib):
    n = 256
    ring, buf, guard = _qring(bclib, 2, n, "f32", 8)
    ring.push(torch.ones(n, device=DEV), 0.0)
    before = buf.clone()
    inside = buf[guard:guard + 4 * n].view(torch.float32)
    for call in (lambda: ring.read(0, inside), lambda: bclib.bary_extrapolate(ring, [1.0], inside), lambda: ring.push(inside, 1.0)):
        with pytest.raises(bclib.BCError) as e:
            call()
        assert e.value.code == bclib.ERR_INVALID_ARG
    torch.cuda.synchronize()
    assert torch.equal(buf, before) and ring.state()[0] == 1


@pytest.mark.gpu
def test_plain_ring_reads_back(bclib):
    n = 1003
    for dt in ("f32", "bf16"):
        x = _dev(_feature(n, dt, seed=1), dt)
        ring = bclib.CacheRing(2, torch.zeros((2, n), dtype=TDT[dt], device=DEV))
        ring.push(x, 0.0)
        for odt in ("f32", "bf16"):
            out = torch.empty(n, dtype=TDT[odt], device=DEV)
            ring.read(0, out)
            assert bool((out == x.to(TDT[odt])).all())


@pytest.mark.gpu
def test_large_feature_on_another_stream_and_in_a_graph(bclib):
    """Push and forecast captured once; replays read new features from the same buffer."""
    n, K = 1 << 21, 2
    ring, buf, guard = _qring(bclib, K, n, "bf16", 4)
    feat = torch.empty(n, dtype=torch.bfloat16, device=DEV)
    out = torch.empty(n, dtype=torch.bfloat16, device=DEV)
    s = torch.cuda.Stream()
    feat.normal_()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        ring.push(feat, 0.0)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        ring.push(feat, 1.0)
        bclib.bary_extrapolate(ring, [1.5, -0.5], out)
    older = torch.empty(n, device=DEV)
    ring.read(1, older)
    for seed in range(3):
        torch.manual_seed(seed)
        feat.normal_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        h = torch.from_numpy(quant.held(feat.float().cpu().numpy(), 4).astype(np.float32)).to(DEV)
        want = (1.5 * h.double() - 0.5 * older.double())
        tol = 2 * 4 * 2.0 ** -24 * (1.5 * h.abs() + 0.5 * older.abs()).double() + want.abs() * 2.0 ** -8 * 1.01
        assert bool(((out.double() - want).abs() <= tol).all()), seed
    assert _guards_kept(buf, guard)


class _QuantRing(bary.Ring):
    """The oracle's ring, holding what the codes of a pushed feature stand for."""
    bits = 8

    def push(self, feat, k):
        held = None if feat is None else quant.held(np.asarray(feat, np.float64).astype(np.float32), self.bits)   # (None: the plan's ring)
        return super().push(held, k)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("name", ["tiny", "dit_cfg", "mmdit"])
def test_sampling_with_a_quantised_ring(bclib, monkeypatch, name, bits):
    """The fp32 runs against the oracle with a quantised ring.  A feature that is
    off by the run's own error of about 1e-6 of a step flips one code in 10^4 or
    fewer, by one step of at most 1/7 of its group: well within 2e-3 of the
    latents, and the run with a plain ring is further away than that error."""
    from paper_2608_28670_amd import loader
    cfg = synth.CONFIGS["tiny"]
    if name == "dit_cfg":
        cfg = synth.scaled(cfg, n_classes=5)
    if name == "mmdit":
        cfg = synth.scaled(synth.CONFIGS["hunyuan"], depth=1, depth_single=1, hidden=128, heads=4, head_dim=32, mlp=256,
                           latent=(16, 2, 8, 8), txt_tokens=9, steps=8, interval=3, batch=2, dtype="f32")
    P = synth.params(cfg)
    mask = bary.make_mask(cfg.steps, cfg.interval)
    xT = synth.latents(cfg)
    x = torch.from_numpy(np.ascontiguousarray(xT, dtype=np.float32)).to(DEV)
    dm = loader.DeviceModel(cfg, P)
    kw, okw = {}, {}
    if name == "mmdit":
        t = synth.text(cfg, batch=cfg.batch)
        kw["text"], okw["text"] = torch.from_numpy(t).to(DEV).to(loader.torch_dtype(cfg)), t
    monkeypatch.setattr(_QuantRing, "bits", bits)
    if name == "dit_cfg":
        lab = synth.labels(cfg, batch=cfg.batch)
        dm.sample_cfg(x, mask, torch.from_numpy(lab).to(DEV), 1.5, cache_bits=bits)
        okw.update(labels=lab, cfg_scale=1.5)
    else:
        dm.sample(x, mask, cache_bits=bits, **kw)
    got = x.double().cpu().numpy()
    model = om.Model(cfg, P)
    plain = osm.sample(model, xT.astype(np.float64), mask, cfg.K, **okw)
    monkeypatch.setattr(bary, "Ring", _QuantRing)
    want = osm.sample(model, xT.astype(np.float64), mask, cfg.K, **okw)
    rel = lambda a, b: float(np.linalg.norm(a - b) / np.linalg.norm(b))
    print(f"{name} {bits} bits: rel-L2 {rel(got, want):.2e}, plain ring differs by {rel(plain, want):.2e}")
    assert rel(got, want) <= min(2e-3, 0.2 * rel(plain, want))


def _blockwise_cfg(name):
    cfg = synth.CONFIGS["tiny"]
    if name == "odd":                                     # 25 tokens a sample
        cfg = synth.scaled(cfg, latent=(4, 5, 5))
    if name == "pixart":
        cfg = synth.scaled(synth.CONFIGS["pixart"], depth=2, hidden=128, heads=4, head_dim=32, mlp=256, latent=(4, 16, 16), batch=2,
                           steps=10, ctx_tokens=7, ctx_dim=64, dtype="f32", K=3)
    return cfg


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("name", ["tiny", "odd", "pixart"])
def test_blockwise_sampling_with_quantised_sites(bclib, monkeypatch, name, bits):
    """fp32 runs against the oracle whose sites hold what the codes stand for; the
    bound as for the stepwise runs.  The codes of the last full step's sites are
    read from the storage: [site][slot], each codes and then scales."""
    from paper_2608_28670_amd import loader
    cfg = _blockwise_cfg(name)
    P = synth.params(cfg)
    mask = bary.make_mask(cfg.steps, cfg.interval)
    xT = synth.latents(cfg)
    x = torch.from_numpy(np.ascontiguousarray(xT, dtype=np.float32)).to(DEV)
    dm = loader.DeviceModel(cfg, P)
    text = synth.text(cfg, batch=cfg.batch) if name == "pixart" else None
    store = dm.sample_blockwise(x, mask, text=torch.from_numpy(text).to(DEV) if text is not None else None, cache_bits=bits)
    torch.cuda.synchronize()
    got = x.double().cpu().numpy()
    model = om.Model(cfg, P)
    plain = osm.sample_blockwise(model, xT.astype(np.float64), mask, cfg.K, text=text)
    rings = []

    class SiteRing(bary.Ring):
        def __init__(self, K):
            super().__init__(K)
            rings.append(self)

        def push(self, sites, k):
            if sites is None:              # the plan's ring
                return super().push(None, k)
            self.raw = [np.asarray(v, np.float64).astype(np.float32) for v in sites]
            return super().push([quant.held(v, bits) for v in self.raw], k)

    monkeypatch.setattr(bary, "Ring", SiteRing)
    want = osm.sample_blockwise(model, xT.astype(np.float64), mask, cfg.K, text=text)
    rel = lambda a, b: float(np.linalg.norm(a - b) / np.linalg.norm(b))
    print(f"{name} {bits} bits: rel-L2 {rel(got, want):.2e}, plain sites differ by {rel(plain, want):.2e}")
    assert rel(got, want) <= min(2e-3, 0.2 * rel(plain, want))
    n = cfg.batch * cfg.tokens * cfg.hidden
    sites = len(rings[-1].raw)
    slot = bclib.quant_cache_bytes(1, n, bits)
    assert store.numel() == sites * cfg.K * slot
    raw = store.cpu().numpy().reshape(sites, cfg.K, slot)
    at = -(-(-(-n // 64) * 8 * bits) // 256) * 256
    for q in range(sites):
        s = np.frombuffer(raw[q, rings[-1].head].tobytes(), np.float32, count=n // 64, offset=at)
        assert np.abs(s / quant.codes(rings[-1].raw[q], bits)[1][:, 0] - 1).max() <= 1e-3


@pytest.mark.gpu
def test_quantised_blockwise_refusals_and_fused_final_step(bclib):
    from paper_2608_28670_amd import loader
    cfg = synth.scaled(synth.CONFIGS["dit_xl2"], depth=2, batch=2, steps=9, interval=4)
    dm = loader.DeviceModel(cfg, synth.params(cfg))
    lab = torch.from_numpy(synth.labels(cfg, batch=2)).to(DEV)
    xT = torch.from_numpy(np.ascontiguousarray(synth.latents(cfg), dtype=np.float32)).to(DEV)
    mask = bary.make_mask(9, 4)
    runs = {}
    for bits in (0, 8, 4):
        x = xT.clone()
        dm.sample_blockwise(x, mask, labels=lab, cache_bits=bits)
        runs[bits] = x.double()
    off = {b: float((runs[b] - runs[0]).norm() / runs[0].norm()) for b in (8, 4)}
    assert 0 < off[8] < off[4] < 0.1
    ws = dm.workspace(2, 9)
    need = dm.model.blockwise_quant_bytes(2, cfg.K, 8)
    store = torch.empty(need, dtype=torch.uint8, device=DEV)
    x = xT.clone()
    for bits, st in ((8, store[:need - 1]), (5, store), (0, store), (8, store[8:])):
        with pytest.raises(bclib.BCError) as e:
            bclib.sample_blockwise_quant(dm.model, 2, cfg.sampler, mask, cfg.K, bits, st, x, ws, labels=lab)
        assert e.value.code == bclib.ERR_INVALID_ARG
    for args in ((0, 3, 8), (65, 3, 8), (2, 0, 8), (2, 9, 8), (2, 3, 16)):
        with pytest.raises(bclib.BCError):
            dm.model.blockwise_quant_bytes(*args)
    numel = 2 * cfg.tokens * cfg.hidden                                                  # a ring in the workspace
    ring = bclib.QuantCacheRing(cfg.K, numel, torch.bfloat16, 4, ws[256:])
    with pytest.raises(bclib.BCError) as e:
        bclib.sample(dm.model, 2, cfg.sampler, mask, cfg.K, ring, x, ws, labels=lab)
    assert e.value.code == bclib.ERR_INVALID_ARG
    torch.cuda.synchronize()
    assert torch.equal(x, xT)


@pytest.mark.gpu
def test_graph_and_adaptive_runs_with_a_quantised_ring(bclib):
    """bf16 with the fused final step: the captured run and the adaptive run of
    the same mask give bc_sample's latents bit for bit."""
    from paper_2608_28670_amd import loader
    cfg = synth.scaled(synth.CONFIGS["dit_xl2"], depth=2, batch=2, steps=10)
    dm = loader.DeviceModel(cfg, synth.params(cfg))
    lab = torch.from_numpy(synth.labels(cfg, batch=2)).to(DEV)
    xT = torch.from_numpy(np.ascontiguousarray(synth.latents(cfg), dtype=np.float32)).to(DEV)
    mask = np.zeros(10, np.uint8)
    mask[[0, 9]] = 1
    a, b = xT.clone(), xT.clone()
    ring = dm.sample(a, mask, labels=lab, cache_bits=8)
    assert ring.bits == 8 and ring.state()[0] == 2
    _, realised, _ = dm.sample_adaptive(b, 10, math.inf, labels=lab, cache_bits=8)
    assert list(realised) == list(mask) and torch.equal(a, b)
    c = torch.empty_like(xT)
    g = dm.sample_graph(c, mask, labels=lab, cache_bits=8)
    for _ in range(3):
        c.copy_(xT)
        g.launch()
        torch.cuda.synchronize()
        assert torch.equal(a, c)
    d = xT.clone()
    dm.sample(d, mask, labels=lab)
    assert not torch.equal(a, d)
    # A ring of the other dtype or size is refused.
    n = cfg.tokens * cfg.hidden * 2
    for numel, dt in ((n, torch.float32), (n + 64, torch.bfloat16)):
        bad = bclib.QuantCacheRing(cfg.K, numel, dt, 8,
                                   torch.empty(bclib.quant_cache_bytes(cfg.K, numel, 8), dtype=torch.uint8, device=DEV))
        with pytest.raises(bclib.BCError) as e:
            bclib.sample(dm.model, 2, cfg.sampler, mask, cfg.K, bad, d, dm.workspace(2, 10), labels=lab)
        assert e.value.code == bclib.ERR_INVALID_ARG


def test_reads_into_a_plain_rings_storage_are_refused(bclib):
    """Refused before anything is enqueued; a node gets into the ring without a
    copy (the push of a slot that its producer wrote)."""
    L = bclib.lib()
    n, at = 100, 1 << 20
    for dtype, esz in ((0, 4), (1, 2)):
        h = C.c_void_p()
        assert L.bc_cache_create(2, n, dtype, at, C.byref(h)) == bclib.OK
        assert L.bc_cache_push(h, None, 0.0, None) == bclib.OK
        size = 2 * n * esz
        for odt, osz in ((0, 4), (1, 2)):
            for out in (at, at + 4, at + size - osz, at - n * osz + osz):            # inside, and by one element at either end
                assert L.bc_cache_read(h, 0, out, odt, None) == bclib.ERR_INVALID_ARG, (dtype, odt, out - at)
            assert L.bc_cache_read(h, 0, (2 << 20) + 1, odt, None) == bclib.ERR_INVALID_ARG      # not aligned to its elements
        assert L.bc_cache_destroy(h) == bclib.OK


@pytest.mark.gpu
def test_plain_ring_reads_beside_its_storage(bclib):
    n = 1003
    for dt in ("f32", "bf16"):
        buf = torch.zeros(4 * n, dtype=TDT[dt], device=DEV)
        x = _dev(_feature(n, dt, seed=2), dt)
        ring = bclib.CacheRing(2, buf[n:3 * n].view(2, n))
        ring.push(x, 0.0)
        for out in (buf[:n], buf[3 * n:]):
            ring.read(0, out)
            assert torch.equal(out, x)
        for out in (buf[1:n + 1], buf[n:2 * n], buf[3 * n - 1:4 * n - 1]):
            with pytest.raises(bclib.BCError) as e:
                ring.read(0, out)
            assert e.value.code == bclib.ERR_INVALID_ARG


def _host_model(name="tiny"):
    from paper_2608_28670_amd import loader
    cfg = _blockwise_cfg(name)
    return cfg, loader.DeviceModel(cfg, synth.params(cfg), device="cpu")


@pytest.mark.parametrize("name", ["tiny", "pixart"])
def test_site_storage_on_the_runs_own_buffers_is_refused(bclib, name):
    """The quantised sites in the workspace or on the latents: refused before anything is enqueued."""
    L = bclib.lib()
    cfg, dm = _host_model(name)
    mask = np.ascontiguousarray(bary.make_mask(cfg.steps, cfg.interval), dtype=np.uint8)
    ws, sites, lat, text = 1 << 30, 4 << 30, 8 << 30, 9 << 30
    ws_bytes = dm.model.workspace_size(cfg.batch, cfg.steps)
    x_bytes = 4 * int(np.prod(synth.latents(cfg).shape))
    for bits in (8, 4):
        need = dm.model.blockwise_quant_bytes(cfg.batch, cfg.K, bits)
        run = lambda at, size=need: L.bc_sample_blockwise_quant(dm.model.h, cfg.batch, bclib.SAMPLERS[cfg.sampler], len(mask), mask.ctypes.data,
                                                                cfg.K, None, bits, at, size, lat, None, text, ws, ws_bytes, None)
        for at in (ws, ws + 256, ws - need + 16, ws + ws_bytes - 512, lat, lat + x_bytes - 16, lat - need + 16):
            assert run(at) == bclib.ERR_INVALID_ARG, (bits, at)
        assert run(sites + 8, need + 8) == bclib.ERR_INVALID_ARG           # large enough: only its alignment is wrong
        assert run(sites, need - 1) == bclib.ERR_INVALID_ARG


@pytest.mark.parametrize("bits", [8, 4])
def test_quantised_ring_on_the_latents_is_refused(bclib, bits):
    L = bclib.lib()
    cfg, dm = _host_model()
    mask = np.ascontiguousarray(bary.make_mask(cfg.steps, cfg.interval), dtype=np.uint8)
    n = cfg.batch * cfg.tokens * cfg.hidden
    ws, store, ws_bytes = 1 << 30, 4 << 30, dm.model.workspace_size(cfg.batch, cfg.steps)
    size = bclib.quant_cache_bytes(cfg.K, n, bits)
    h = C.c_void_p()
    assert L.bc_cache_create_quant(cfg.K, n, bclib.F32, bits, store, C.byref(h)) == bclib.OK
    for lat in (store, store + size - 16):
        assert L.bc_sample(dm.model.h, cfg.batch, bclib.SAMPLERS[cfg.sampler], len(mask), mask.ctypes.data, cfg.K, None, h, lat, None, None,
                           ws, ws_bytes, None) == bclib.ERR_INVALID_ARG
    assert L.bc_cache_destroy(h) == bclib.OK


def test_blockwise_binding_refuses_tensors_of_the_host(bclib):
    cfg, dm = _host_model()
    mask = bary.make_mask(cfg.steps, cfg.interval)
    e = lambda n: torch.empty(n, dtype=torch.uint8)
    with pytest.raises(bclib.BCError) as err:
        bclib.sample_blockwise_quant(dm.model, cfg.batch, cfg.sampler, mask, cfg.K, 8, e(dm.model.blockwise_quant_bytes(cfg.batch, cfg.K, 8)),
                                     torch.zeros(synth.latents(cfg).shape), e(dm.model.workspace_size(cfg.batch, cfg.steps)))
    assert err.value.code == bclib.ERR_INVALID_ARG


@pytest.mark.gpu
def test_operands_and_streams_of_other_devices_are_refused(bclib):
    """A stream of another device, and a blockwise run with an operand on the host."""
    import types
    from paper_2608_28670_amd import loader
    n = 1000
    other = types.SimpleNamespace(cuda_stream=0, device_index=torch.cuda.current_device() + 1)
    ring, _, _ = _qring(bclib, 1, n, "f32", 8)
    x, out = torch.ones(n, device=DEV), torch.zeros(n, device=DEV)
    ring.push(x, 0.0)
    y = torch.ones(4, 64, device=DEV)
    q = torch.zeros(1, 128, 1, 64, device=DEV)
    blocks = torch.zeros(1, 1, 1, 1, dtype=torch.int32, device=DEV)
    ws = torch.empty(1 << 16, dtype=torch.uint8, device=DEV)
    calls = [lambda: ring.push(x, 1.0, stream=other), lambda: ring.read(0, out, stream=other), lambda: bclib.bary_extrapolate(ring, [1.0], out, stream=other),
             lambda: bclib.norm_gate_residual(y, y.clone(), y.clone(), stream=other), lambda: bclib.attention_select(q, q, blocks, ws=ws, stream=other),
             lambda: bclib.attention_sparse(q, q, q, blocks, torch.empty_like(q), ws=ws, stream=other)]
    cfg = _blockwise_cfg("tiny")
    dm = loader.DeviceModel(cfg, synth.params(cfg))
    mask = bary.make_mask(cfg.steps, cfg.interval)
    lat = torch.zeros(synth.latents(cfg).shape, device=DEV)
    sites = torch.empty(dm.model.blockwise_quant_bytes(cfg.batch, cfg.K, 8), dtype=torch.uint8, device=DEV)
    work = dm.workspace(cfg.batch, cfg.steps)
    run = lambda s, l, w, **kw: bclib.sample_blockwise_quant(dm.model, cfg.batch, cfg.sampler, mask, cfg.K, 8, s, l, w, **kw)
    calls += [lambda: run(sites.cpu(), lat, work), lambda: run(sites, lat, work.cpu()), lambda: run(sites, lat.cpu(), work),
              lambda: run(sites, lat, work, stream=other)]
    for i, call in enumerate(calls):
        with pytest.raises(bclib.BCError) as e:
            call()
        assert e.value.code == bclib.ERR_INVALID_ARG, i
    torch.cuda.synchronize()
    ring.read(0, out, stream=torch.cuda.Stream())
    torch.cuda.synchronize()
    assert torch.equal(out, x)


@pytest.mark.gpu
@pytest.mark.parametrize("bits,odt", [(8, "bf16"), (4, "bf16"), (4, "f32")])
def test_features_beyond_32_bit_offsets(bclib, bits, odt):
    """More than 2^32 values: what lies around 2^31, 2^32 and at the ragged end."""
    n = (1 << 32) + 64 * 5 + 7
    g = torch.Generator(device=DEV)
    g.manual_seed(bits)
    x = torch.empty(n, dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    ring = bclib.QuantCacheRing(1, n, torch.bfloat16, bits, torch.empty(bclib.quant_cache_bytes(1, n, bits), dtype=torch.uint8, device=DEV))
    ring.push(x, 0.0)
    out = torch.full((n + 8,), 7.0, dtype=TDT[odt], device=DEV)
    ring.read(0, out[:n])
    for at in (0, (1 << 31) - 640, (1 << 32) - 640):
        end = min(at + 1280, n)
        want = quant.held(x[at:end].float().cpu().numpy(), bits).astype(np.float32)
        assert torch.equal(out[at:end], _dev(want, odt)), at
    assert bool((out[n:] == 7.0).all())
