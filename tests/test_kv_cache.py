"""The key-value cache in 8 bits: refusals on the CPU; on the GPU what it holds,
exactly, and its attention against float64 over those values."""
import ctypes as C
import math

import numpy as np
import pytest

from oracle import kv as oracle
from oracle import score
from score_checks import compare, tolerance

torch = pytest.importorskip("torch")
DEV = "cuda:0"
TDT = {"f32": torch.float32, "bf16": torch.bfloat16}
FAR = 1 << 24


# ---------------------------------------------------------------------------
# CPU
# ---------------------------------------------------------------------------
def _cache(bc, **kw):
    s = dict(B=1, H=2, d=64, capacity=1000, storage=FAR)
    s.update(kw)
    return C.byref(bc.KVCacheDesc(**s))


def _push(bc, T=20, k=2 * FAR, v=3 * FAR, lens=4 * FAR, counts=None, dtype=1, strides=(20 * 128, 128), **kw):
    return bc.lib().bc_kv_push(_cache(bc, **kw), T, k, *strides, v, *strides, lens, counts, dtype, None)


def _read(bc, first=0, n=20, lens=4 * FAR, k=2 * FAR, v=3 * FAR, dtype=1, **kw):
    return bc.lib().bc_kv_read(_cache(bc, **kw), first, n, lens, k, v, dtype, None)


def _attend(bc, Hq=2, Tq=300, q=2 * FAR, strides=(300 * 128, 128), lens=4 * FAR, counts=None, opts=None, out=5 * FAR, dtype=1, ws=None, ws_bytes=0, **kw):
    o = C.byref(bc.ScoreOpts(**opts)) if opts is not None else None
    return bc.lib().bc_kv_attention(_cache(bc, **kw), Hq, Tq, q, *strides, lens, counts, o, out, dtype, ws, ws_bytes, None)


def test_refusals(bclib):
    bad, no = bclib.ERR_INVALID_ARG, bclib.ERR_UNSUPPORTED
    lim = 1 << 24
    for kw, want in [(dict(B=0), bad), (dict(H=0), bad), (dict(d=0), bad), (dict(capacity=0), bad), (dict(d=48), no), (dict(capacity=lim), no),
                     (dict(B=1 << 21), no), (dict(storage=None), bad), (dict(storage=FAR + 128), bad), (dict(dtype=2), bad), (dict(lens=None), bad),
                     (dict(lens=4 * FAR + 2), bad)]:
        for call in (_push, _read, _attend):
            if call is _attend and kw.get("H") or kw.get("B") == 1 << 21 and call is _attend:
                continue
            assert call(bclib, **kw) == want, (call.__name__, kw)
    size = C.c_size_t()
    assert bclib.lib().bc_kv_cache_size(1, 2, 64, 1000, None) == bad and bclib.lib().bc_kv_cache_size(1, 2, 40, 1000, C.byref(size)) == no
    assert bclib.lib().bc_kv_cache_size(1, 2, 72, 1000, C.byref(size)) == bclib.OK and size.value == 2 * 16 * (128 * 72 + 8)
    bytes64 = bclib.kv_cache_bytes(1, 2, 64, 1000)
    for kw in (dict(T=0), dict(T=-1), dict(k=None), dict(v=None), dict(k=2 * FAR + 8), dict(v=3 * FAR + 2), dict(strides=(20 * 128, 132)), dict(strides=(-1, 128)),
               dict(counts=5 * FAR + 1), dict(k=FAR + bytes64 - 16), dict(v=FAR), dict(lens=FAR + 64), dict(counts=FAR + 64)):
        assert _push(bclib, **kw) == bad, kw
    for kw in (dict(first=-1), dict(n=0), dict(first=990), dict(k=None), dict(v=None), dict(k=2 * FAR + 1), dict(k=FAR + bytes64 - 8), dict(v=FAR), dict(v=2 * FAR + 64),
               dict(k=4 * FAR - 100), dict(first=2_147_483_647)):
        assert _read(bclib, **kw) == bad, kw
    for kw in (dict(Hq=3), dict(Hq=0), dict(Tq=0), dict(q=None), dict(q=2 * FAR + 8), dict(strides=(300 * 128, 100)), dict(counts=6 * FAR + 2), dict(out=None),
               dict(out=5 * FAR + 1), dict(opts=dict(cap=-1.0)), dict(opts=dict(window=-1)), dict(opts=dict(scale=math.nan)), dict(out=FAR), dict(out=2 * FAR + 4096),
               dict(out=4 * FAR), dict(out=6 * FAR, counts=6 * FAR), dict(out=7 * FAR, opts=dict(slopes=7 * FAR)), dict(out=7 * FAR, opts=dict(prefix=7 * FAR))):
        assert _attend(bclib, **kw) == bad, kw
    split = dict(Tq=1, capacity=100_000, storage=16 * FAR)                                # in parts, which need a workspace
    n = C.c_size_t()
    assert bclib.lib().bc_kv_attention_workspace_size(_cache(bclib, capacity=100_000), 2, 1, 1, C.byref(n)) == bclib.OK and n.value > 0
    for kw in (dict(), dict(ws=64 * FAR, ws_bytes=n.value - 1), dict(ws=64 * FAR + 64, ws_bytes=n.value), dict(ws=16 * FAR, ws_bytes=n.value),
               dict(ws=2 * FAR, ws_bytes=n.value), dict(ws=4 * FAR, ws_bytes=n.value), dict(ws=5 * FAR, ws_bytes=n.value)):
        assert _attend(bclib, **split, **kw) == bad, kw
    assert bclib.lib().bc_kv_attention_workspace_size(_cache(bclib), 3, 1, 1, C.byref(n)) == bad
    assert bclib.lib().bc_kv_push(None, 1, FAR, 1, 1, FAR, 1, 1, FAR, None, 1, None) == bad


def test_strides_whose_offsets_pass_64_bits_are_refused(bclib):
    for call in (_push, _attend):
        assert call(bclib, B=1 << 13, capacity=64, storage=1 << 44, strides=(1 << 48, 128)) == bclib.ERR_INVALID_ARG


def test_binding_refuses_tensors_that_do_not_fit(bclib):
    bf, i32 = torch.bfloat16, torch.int32
    n = bclib.kv_cache_bytes(2, 3, 32, 100)
    store = torch.zeros(n + 256, dtype=torch.uint8)
    store = store[-store.data_ptr() % 256:][:n]
    with pytest.raises(bclib.BCError):
        bclib.KVCache(2, 3, 32, 100, store[:-1])
    c = bclib.KVCache(2, 3, 32, 100, store)
    k, lens = torch.zeros(2, 5, 3, 32, dtype=bf), torch.zeros(2, dtype=i32)
    for kw in (dict(k=k[:1]), dict(v=k.float()), dict(v=k[:, :4]), dict(k=k[0]), dict(lens=lens.long()), dict(lens=lens[:1]), dict(counts=lens.float()), dict(lens=None), dict()):
        with pytest.raises(bclib.BCError) as e:                                           # (the last: tensors of the host)
            c.push(**dict(dict(k=k, v=k.clone(), lens=lens), **kw))
        assert e.value.code == bclib.ERR_INVALID_ARG, kw
    for kw in (dict(k_out=k[:1]), dict(v_out=k.float()), dict(v_out=k[:, :4]), dict(k_out=k.transpose(1, 2)), dict(lens=None), dict()):
        with pytest.raises(bclib.BCError) as e:
            c.read(**dict(dict(k_out=k, v_out=k.clone(), lens=lens), **kw))
        assert e.value.code == bclib.ERR_INVALID_ARG, kw
    q = torch.zeros(2, 5, 6, 32, dtype=bf)
    for kw in (dict(q=q[:1]), dict(out=q[:, :4]), dict(out=q.float()), dict(slopes=torch.zeros(3)), dict(prefix=lens.long()), dict(lens=None), dict()):
        with pytest.raises(bclib.BCError) as e:
            c.attention(**dict(dict(q=q, out=q.clone(), lens=lens), **kw))
        assert e.value.code == bclib.ERR_INVALID_ARG, kw


def test_oracle():
    """e4m3 as torch rounds to it; scales by hand; a growing scale."""
    x = np.concatenate([np.linspace(-450, 450, 9001), 2.0 ** np.linspace(-14, 8, 4001), [0.0, 448.0, 2.0 ** -10, 3 * 2.0 ** -10]]).astype(np.float32)
    x = x[np.abs(x) <= 448]
    assert np.array_equal(oracle.round8(x), torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy())
    for top, s in ((448.0, 1.0), (448.1, 2.0), (1.0, 2.0 ** -8), (1.75, 2.0 ** -8), (1.76, 2.0 ** -7), (0.0, 2.0 ** -100), (1e-35, 2.0 ** -100), (3e38, 2.0 ** 120)):
        assert oracle.scale_of(np.array([top, -top / 3, np.inf, np.nan])) == s, top
    c = oracle.Cache(1, 1, 2, 130)
    c.push(np.full((1, 70, 1, 2), 0.013), [70], [70])
    c.push(np.full((1, 3, 1, 2), 400.0), [73], [3])
    # 0.013 * 2^15 = 425.98, steps of 32: 416; 416 * 2^-15 = 6.5 / 512: to the even 6.  400 = 12.5 * 32: to the even 12.
    assert c.scale[0, 0].tolist() == [2.0 ** -15, 1.0, 0.0] and c.val[0, 0, 69, 0] == 6 / 512 and c.val[0, 0, 70, 1] == 384.0
    c.push(np.full((1, 200, 1, 2), 1.0), [150], [200])                                    # held to the capacity; the first lie before position 0
    assert (c.val[0, 0] == 1.0).all()


# ---------------------------------------------------------------------------
# GPU
# ---------------------------------------------------------------------------
def _np(t):
    return t.double().cpu().numpy()


def _i32(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device=DEV)


class Both:
    """The library's cache beside the oracle's; the storage starts as NaN codes, margins around it."""

    def __init__(self, bc, B, H, d, capacity, dt):
        self.bc, self.dt, n = bc, TDT[dt], bc.kv_cache_bytes(B, H, d, capacity)
        self.buf = torch.full((n + 512,), 0x7F, dtype=torch.uint8, device=DEV)
        self.cache = bc.KVCache(B, H, d, capacity, self.buf[256:256 + n])
        self.k, self.v = oracle.Cache(B, H, d, capacity), oracle.Cache(B, H, d, capacity)
        self.lens = [0] * B

    def push(self, x, y, lens, counts=None):
        self.cache.push(x, y, _i32(lens), counts=_i32(counts))
        counts = [x.shape[1]] * x.shape[0] if counts is None else counts
        self.k.push(_np(x), lens, counts)
        self.v.push(_np(y), lens, counts)
        self.lens = lens
        torch.cuda.synchronize()
        assert bool((self.buf[:256] == 0x7F).all()) and bool((self.buf[-256:] == 0x7F).all())

    def check(self, first=0, n=None):
        c = self.cache
        n = c.capacity - first if n is None else n
        guard = torch.full((2, c.B * n * c.H * c.d + 64), 3.0, dtype=self.dt, device=DEV)
        outs = [g[32:-32].view(c.B, n, c.H, c.d) for g in guard]
        c.read(*outs, _i32(self.lens), first=first)
        torch.cuda.synchronize()
        assert bool((guard[:, :32] == 3).all()) and bool((guard[:, -32:] == 3).all())
        for got, want in zip(outs, (self.k, self.v)):
            want = want.val[:, :, first:first + n].transpose(0, 2, 1, 3).copy()
            for b, m in enumerate(self.lens):
                want[b, max(0, m - first):] = 0.0
            assert np.array_equal(_np(got), want, equal_nan=True)

    def attend(self, q, lens=None, counts=None, prefix=None, slopes=None, scale=None, cap=0.0, causal=False, window=0):
        c, (B, Tq, Hq, d) = self.cache, q.shape
        lens = self.lens if lens is None else lens
        buf = torch.full((q.numel() + 64,), 7.0, device=DEV, dtype=q.dtype)
        out = buf[32:-32].view(q.shape)
        n = c.attention_workspace_size(Hq, Tq, self.bc.dtype_code(q))
        ws = torch.full((n + 256,), 0xFF, dtype=torch.uint8, device=DEV)
        c.attention(q, out, _i32(lens), counts=_i32(counts), scale=scale, cap=cap, slopes=slopes, causal=causal, window=window, prefix=_i32(prefix), ws=ws[:n])
        torch.cuda.synchronize()
        assert bool((buf[:32] == 7).all()) and bool((buf[-32:] == 7).all()) and bool((ws[n:] == 0xFF).all())
        qn, got, sl = _np(q), _np(out), None if slopes is None else _np(slopes)
        for b in range(B):
            m = min(max(lens[b], 0), c.capacity)
            rows = Tq if counts is None else min(max(counts[b], 0), Tq)
            p = m - rows + np.arange(rows)
            see = score.seen(p, m, causal, window, 0 if prefix is None else prefix[b])
            assert not got[b, rows:].any()
            for h in range(Hq):
                hk = h // (Hq // c.H)
                want, A, size, mag = score.attend(qn[b, :rows, h], self.k.val[b, hk, :m], self.v.val[b, hk, :m], see, p,
                                                  d ** -0.5 if scale is None else scale, cap, 0.0 if sl is None else sl[h])
                compare(got[b, :rows, h], want, tolerance(want, A, size, mag, d, c.capacity, cap, q.dtype == torch.bfloat16), A)
        return out


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _randn(g, *shape, dt="bf16", scale=1.0):
    return torch.empty(shape, device=DEV).normal_(0.0, scale, generator=g).to(TDT[dt])


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 72, 128])
def test_what_pushes_leave(bclib, d, dt):
    """Pushes of many tokens and of one, into tiles that hold some, with scales that grow and that stay; ragged samples; views."""
    B, H, cap = 3, 2, 400
    c, g = Both(bclib, B, H, d, cap, dt), _gen(d)
    c.check()
    lens = [0] * B
    for T, counts, size in ((5, [5, 3, 0], 1.0), (1, None, 3.0), (130, [130, 64, 58], 0.1), (1, [1, 0, 1], 100.0), (64, None, 0.01), (63, [0, 63, 1], 1.0), (2, None, 1e-4)):
        x = _randn(g, B, T + 1, 2 * H * d + 8, dt=dt, scale=size)
        x[:, :, :H * d] *= torch.exp(_randn(g, 1, 1, H * d, dt="f32", scale=2.0)).to(x.dtype)
        counts = counts or [T] * B
        lens = [n + m for n, m in zip(lens, counts)]
        c.push(x[:, :T, :H * d].unflatten(-1, (H, d)), x[:, :T, H * d:2 * H * d].unflatten(-1, (H, d)), lens, counts)
        c.check()
    c.check(first=100, n=77)
    c.check(first=64, n=1)
    back = [n - 70 for n in lens]                                                         # going back, and on from there
    x, y = _randn(g, B, 10, H, d, dt=dt), _randn(g, B, 10, H, d, dt=dt)
    c.push(x, y, [n + 10 for n in back])
    c.check()


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_pushes_at_the_edges(bclib, dt):
    """Lengths beyond the capacity and below zero, tokens before position 0, counts out of range; the last token of a capacity that ends inside a tile."""
    c, g = Both(bclib, 4, 1, 64, 150, dt), _gen(0)
    x, y = _randn(g, 4, 200, 1, 64, dt=dt), _randn(g, 4, 200, 1, 64, dt=dt)
    c.push(x, y, [150, 500, 70, -3])
    c.lens = [150, 150, 70, 0]
    c.check()
    c.push(x[:, :3], y[:, :3], [150, 149, 64, 2], [3, 9, -1, 2])
    c.check()


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_codes_of_special_values(bclib, dt):
    """Ties, subnormal codes, zeros, the largest values, values that are not finite."""
    c = Both(bclib, 1, 1, 128, 640, dt)
    x = torch.zeros(640, 128, device=DEV)
    x[0:64, :] = (torch.arange(64 * 128, device=DEV).float() - 4096).view(64, 128) / 128             # every half step of small codes
    x[64:128] = (torch.arange(64 * 128, device=DEV).float() * 2.0 ** -14).view(64, 128)
    x[64, 0] = 448.0
    x[128, 3], x[129, 4], x[130, 5], x[131] = math.inf, -math.inf, math.nan, 5.0
    x[192:256] = 3e38
    x[256:320] = 1e-38
    x[320:384] = 2.0 ** -126
    x[384:448, ::2] = 1e-30
    x[384:448, 1] = 1e-32
    x[448] = -448.0
    x[449] = 447.0
    x[512:576] = math.nan
    x = x.to(TDT[dt]).view(1, 640, 1, 128)
    c.push(x, x.flip(3).contiguous(), [640])
    c.check()
    y = torch.full((1, 1, 1, 128), 1e4, device=DEV, dtype=TDT[dt])
    for n in (513, 385, 321, 200, 130):                                                   # going back, a large token behind them moves what stands
        c.push(y, y, [n])
        c.check()


ATTEND = [  # B, H, G, Tq, capacity, lens, counts, d
    (1, 1, 1, 1, 1, [1], None, 32), (2, 2, 2, 1, 300, [300, 7], None, 64), (3, 2, 4, 1, 5000, [5000, 0, 63], None, 128), (2, 3, 1, 3, 700, [650, 2], [3, 2], 72),
    (1, 2, 8, 2, 9000, [8999], None, 64), (2, 1, 2, 40, 500, [400, 64], [40, 11], 128), (1, 2, 1, 150, 150, [150], None, 72), (2, 2, 1, 130, 1000, [1000, 129], [130, 0], 32),
    (1, 3, 2, 100, 2000, [1900], None, 64), (2, 2, 1, 300, 400, [120, 390], None, 128), (1, 1, 1, 60, 6000, [6000], None, 72), (1, 4, 4, 1, 40_000, [39_000], None, 128)]


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("form", ["plain", "causal", "all"])
@pytest.mark.parametrize("B,H,G,Tq,capacity,lens,counts,d", ATTEND)
def test_attention(bclib, B, H, G, Tq, capacity, lens, counts, d, form, dt):
    c, g = Both(bclib, B, H, d, capacity, dt), _gen(capacity)
    c.push(_randn(g, B, max(lens), H, d, dt=dt), _randn(g, B, max(lens), H, d, dt=dt), lens, lens)
    x = _randn(g, B, Tq + 1, H * G * d + 16, dt=dt)
    q = x[:, 1:, 16:].unflatten(-1, (H * G, d))
    kw = {}
    if form != "plain":
        kw["causal"] = True
    if form == "all":
        kw.update(window=max(1, capacity // 6), prefix=[min(70, capacity) - 3 * b for b in range(B)], cap=15.0, scale=0.25,
                  slopes=2.0 ** -torch.arange(1, H * G + 1, device=DEV, dtype=torch.float32))
    a = c.attend(q, counts=counts, **kw)
    assert torch.equal(a, c.attend(q, counts=counts, **kw))


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_piece_by_piece(bclib, dt):
    """A sample made in pieces and single tokens with turned queries and keys, as a program does it, ends with the attention over all of it at once (causal), to the cache's rounding."""
    B, H, G, d, T = 2, 2, 2, 64, 200
    g = _gen(3)
    q, k, v = _randn(g, B, T, H * G, d, dt=dt), _randn(g, B, T, H, d, dt=dt), _randn(g, B, T, H, d, dt=dt)
    f = bclib.rope_frequencies(d)
    c = Both(bclib, B, H, d, T, dt)
    outs, at = [], 0
    for n in (90, 1, 1, 64, 3, 41):
        piece = [x[:, at:at + n].contiguous() for x in (q, k)]
        bclib.rope(piece[0], piece[0], f, k=piece[1], k_out=piece[1], start=at)
        at += n
        c.push(piece[1], v[:, at - n:at], [at] * B)
        outs.append(c.attend(piece[0], causal=True))
    assert at == T
    qt, kt, want = torch.empty_like(q), torch.empty_like(k), torch.empty_like(q)
    bclib.rope(q, qt, f, k=k, k_out=kt)
    ws = torch.empty(bclib.attention_masked_workspace_size(B, H * G, H, T, T, d, bclib.dtype_code(q)), dtype=torch.uint8, device=DEV)
    bclib.attention_masked(qt, kt, v, want, causal=True, ws=ws)
    got = torch.cat(outs, 1)
    # Keys and values off by 2^-4 of themselves at most, about 2^-4 / sqrt(3) / 2 of it in the mean of their squares.
    assert float((got.double() - want.double()).norm() / want.double().norm()) <= 2.0 ** -4


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("Tq,d", [(1, 128), (6, 72), (40, 64), (180, 32), (180, 72)])
def test_values_that_are_not_finite(bclib, Tq, d, dt):
    """NaN (infinities are held as NaN) where no query sees them leave no trace; where some do, those are NaN."""
    c, g = Both(bclib, 1, 2, d, 300, dt), _gen(d)
    x, y = _randn(g, 1, 260, 2, d, dt=dt), _randn(g, 1, 260, 2, d, dt=dt)
    y[0, 30, 0, 1], y[0, 100, 1, d - 1], y[0, 250, 0, 7], x[0, 255, 1, 0] = math.inf, -math.inf, math.nan, math.nan
    c.push(x, y, [260])
    q = _randn(g, 1, Tq, 4, d, dt=dt)
    c.attend(q, lens=[240], window=60, causal=True)
    c.attend(q, lens=[240], causal=True)
    c.attend(q, causal=True)
    c.attend(q, lens=[25])


@pytest.mark.gpu
def test_tokens_beyond_32_bit_offsets(bclib):
    """5 million tokens a head: codes past 2^33 bytes, positions past 2^22."""
    H, d, cap = 8, 128, 5_000_000
    store = torch.empty(bclib.kv_cache_bytes(1, H, d, cap), dtype=torch.uint8, device=DEV)
    c, g = bclib.KVCache(1, H, d, cap, store), _gen(1)
    k, v, q = _randn(g, 1, 200, H, d), _randn(g, 1, 200, H, d), _randn(g, 1, 100, H, d)
    lens = _i32([cap - 5])
    c.push(k, v, lens)
    k2, v2 = torch.empty(1, 190, H, d, device=DEV), torch.empty(1, 190, H, d, device=DEV)
    c.read(k2, v2, lens, first=cap - 5 - 190)
    small = Both(bclib, 1, H, d, 256, "bf16")
    at = (cap - 5 - 200) % 64                             # the same places in their tiles
    small.push(torch.cat([k[:, :at] * 0, k], 1), torch.cat([v[:, :at] * 0, v], 1), [at + 200])
    assert np.array_equal(_np(k2), small.k.val[:, :, at + 10:at + 200].transpose(0, 2, 1, 3))
    assert np.array_equal(_np(v2), small.v.val[:, :, at + 10:at + 200].transpose(0, 2, 1, 3))
    for Tq in (1, 100):
        out = torch.empty_like(q[:, :Tq])
        ws = torch.empty(max(256, c.attention_workspace_size(H, Tq, bclib.BF16)), dtype=torch.uint8, device=DEV)
        c.attention(q[:, :Tq].contiguous(), out, lens, causal=True, window=90, ws=ws)
        want = small.attend(q[:, :Tq].contiguous(), causal=True, window=90)
        assert float((out.double() - want.double()).abs().max()) <= 2.0 ** -6 * float(want.double().abs().max())


@pytest.mark.gpu
def test_captured_graph_goes_on(bclib):
    """A step of push and attention recorded once: each replay takes up where the sample is; another stream's cache works beside it."""
    B, H, G, d, cap = 2, 2, 2, 64, 500
    c, g = Both(bclib, B, H, d, cap, "bf16"), _gen(4)
    c.push(_randn(g, B, 120, H, d), _randn(g, B, 120, H, d), [120, 60], [120, 60])
    k, v, q = _randn(g, B, 3, H, d), _randn(g, B, 3, H, d), _randn(g, B, 3, H * G, d)
    lens, counts = _i32([120, 60]), _i32([3, 3])
    out = torch.empty_like(q)
    ws = torch.empty(max(256, c.cache.attention_workspace_size(H * G, 3, bclib.BF16)), dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lens.add_(counts)
        c.cache.push(k, v, lens, counts=counts)
        c.cache.attention(q, out, lens, counts=counts, causal=True, ws=ws)
    lens.copy_(_i32([120, 60]))
    other, s = Both(bclib, 1, 1, 32, 100, "f32"), torch.cuda.Stream()
    x = _randn(g, 1, 1, 1, 32, dt="f32")
    for step in range(4):
        for t, size in ((k, 1.0 + step), (v, 0.5), (q, 1.0)):
            t.copy_(_randn(g, *t.shape, scale=size))
        counts.copy_(_i32([3, step]))
        s.wait_stream(torch.cuda.current_stream())
        graph.replay()
        other.cache.push(x, x, _i32([step + 1]), stream=s)
        torch.cuda.synchronize()
        now, m = lens.tolist(), counts.tolist()
        c.k.push(_np(k), now, m)
        c.v.push(_np(v), now, m)
        c.lens = now
        c.check()
        assert torch.equal(out, c.attend(q, counts=m, causal=True)), step


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("Tq,n,d", [(1, 200, 64), (1, 6000, 128), (30, 190, 72), (40, 3000, 64), (180, 260, 72), (150, 3000, 32)])
def test_seen_values_of_small_weights_that_are_not_finite(bclib, Tq, n, d, dt):
    """Weights of 2^-230, below fp32's least: a NaN that is seen makes the output NaN, wherever the keys are cut."""
    c, g = Both(bclib, 1, 2, d, n, dt), _gen(n)
    q, x, y = _randn(g, 1, Tq, 4, d, dt=dt), _randn(g, 1, n, 2, d, dt=dt), _randn(g, 1, n, 2, d, dt=dt)
    q[..., 0], x[..., 0] = 8.0, 0.0
    x[:, [3, n // 2, n - 2], :, 0] = -20.0
    y[:, 3, :, 1], y[:, n // 2, :, 2], y[:, n - 2, :, d - 1] = math.nan, math.inf, math.nan
    c.push(x, y, [n])
    c.attend(q, scale=1.0)
    c.attend(q, scale=1.0, causal=True, lens=[n - 2])
    c.attend(q, scale=1.0, window=max(2, n // 3), prefix=[3])


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("Tq", [1, 4, 40, 150])
def test_a_kept_prefix_and_a_window(bclib, Tq, dt):
    """The first tokens and the last ones of a long sample, in parts."""
    c, g = Both(bclib, 2, 1, 64, 4000, dt), _gen(Tq)
    c.push(_randn(g, 2, 4000, 1, 64, dt=dt), _randn(g, 2, 4000, 1, 64, dt=dt), [4000, 2111], [4000, 2111])
    q = _randn(g, 2, Tq, 2, 64, dt=dt)
    for window, prefix in ((500, [4, 64]), (64, [65, 1]), (1000, [2900, 1200]), (1000, [2999, 0]), (9, [4000, 2110])):
        c.attend(q, window=window, prefix=prefix, causal=True)
        c.attend(q, window=window, prefix=prefix)
