"""bc_attention_select and bc_attention_sparse: refusals on the CPU; on the GPU
the lists exactly, the attention against float64.

Tolerances of the attention, with A = sum p |v| per output.  bf16: the
probabilities are rounded to bf16 for the second product (2^-8 of A), their row
sums are those of the rounded ones (2^-8 of A again), the output is rounded
(2^-8 of itself); fp32 sums and the exponential are below 2 % of that.  fp32,
u = 2^-24: a score is off by at most (d + 3) u sum |q k| scale, a probability by
twice the largest of these (itself and the sum) and a sum of n terms by n u."""
import ctypes as C
import math

import numpy as np
import pytest

from oracle import sparse

torch = pytest.importorskip("torch")
DEV = "cuda:0"
TDT = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------------------
# CPU
# ---------------------------------------------------------------------------
SHAPE = dict(B=1, H=2, Tq=200, Tk=300, d=64)
FAR = 1 << 20


def _select(bc, q=FAR, k=2 * FAR, lens=None, keep=2, last=0, blocks=4 * FAR, dtype=1, ws=5 * FAR, ws_bytes=FAR, **kw):
    s = dict(SHAPE, **kw)
    return bc.lib().bc_attention_select(s["B"], s["H"], s["Tq"], s["Tk"], s["d"], q, k, lens, keep, last, blocks, dtype, ws, ws_bytes, None)


def _sparse(bc, q=FAR, k=2 * FAR, v=3 * FAR, lens=None, blocks=4 * FAR, keep=2, out=5 * FAR, pre=0, dtype=1, ws=None, ws_bytes=0, **kw):
    s = dict(SHAPE, **kw)
    return bc.lib().bc_attention_sparse(s["B"], s["H"], s["Tq"], s["Tk"], s["d"], q, k, v, lens, blocks, keep, out, pre, dtype, ws, ws_bytes, None)


def test_refusals(bclib):
    bad, no = bclib.ERR_INVALID_ARG, bclib.ERR_UNSUPPORTED
    shapes = [(dict(B=0), bad), (dict(H=0), bad), (dict(Tq=0), bad), (dict(Tk=0), bad), (dict(d=0), bad), (dict(keep=0), bad),
              (dict(d=40), no), (dict(d=256), no), (dict(d=72, dtype=0), no), (dict(d=128, dtype=0), no), (dict(dtype=2), bad),
              (dict(Tk=64 * 4096 + 1), no), (dict(keep=4097), no), (dict(B=1 << 13, H=1 << 13), no), (dict(q=FAR + 8), bad), (dict(k=FAR + 2), bad)]
    for kw, want in shapes + [(dict(q=None), bad), (dict(k=None), bad), (dict(blocks=None), bad), (dict(ws=None), bad),
                              (dict(ws=FAR + 16), bad), (dict(ws_bytes=100), bad), (dict(last=-1), bad), (dict(last=3), bad)]:
        assert _select(bclib, **kw) == want, kw
    for kw, want in shapes + [(dict(q=None), bad), (dict(k=None), bad), (dict(v=None), bad), (dict(blocks=None), bad),
                              (dict(out=None), bad), (dict(v=FAR + 8), bad), (dict(pre=1, dtype=0), no)]:
        assert _sparse(bclib, **kw) == want, kw
    for at in (FAR, FAR + 4096, 2 * FAR, 3 * FAR, 4 * FAR - 2, 6 * FAR):                  # an output on another operand
        assert _sparse(bclib, out=at, lens=6 * FAR) == bad, at
    for at in (FAR, 2 * FAR + 4, 5 * FAR, 6 * FAR):
        assert _select(bclib, blocks=at, lens=6 * FAR) == bad, at
    for kw in (dict(lens=6 * FAR + 2), dict(blocks=4 * FAR + 1)):                          # not aligned to their elements
        assert _sparse(bclib, **kw) == bad and _select(bclib, **kw) == bad, kw
    assert _sparse(bclib, out=5 * FAR + 1) == bad and _sparse(bclib, out=5 * FAR + 2, dtype=0) == bad
    for at in (FAR, 2 * FAR, 4 * FAR, 6 * FAR):                                            # the workspace on another operand
        assert _select(bclib, ws=at, lens=6 * FAR) == bad, at
    n = C.c_size_t()
    split = dict(Tq=1, Tk=6400, keep=64, k=16 * FAR, v=32 * FAR)                  # few queries, long lists: in parts, which need a workspace
    assert bclib.lib().bc_attention_sparse_workspace_size(1, 2, 1, 6400, 64, 64, 1, C.byref(n)) == bclib.OK and n.value > 0
    for kw in (dict(), dict(ws=64 * FAR, ws_bytes=n.value - 1), dict(ws=64 * FAR + 128, ws_bytes=n.value)):
        assert _sparse(bclib, **split, **kw) == bad, kw
    for at in (FAR, 16 * FAR, 32 * FAR, 4 * FAR, 5 * FAR, 6 * FAR):
        assert _sparse(bclib, **split, ws=at, ws_bytes=n.value, lens=6 * FAR) == bad, at
    for fn in (bclib.lib().bc_attention_select_workspace_size, bclib.lib().bc_attention_sparse_workspace_size):
        assert fn(1, 2, 200, 300, 64, 2, 1, None) == bad
        assert fn(1, 2, 200, 300, 40, 2, 1, C.byref(n)) == no
        assert fn(1, 0, 200, 300, 64, 2, 1, C.byref(n)) == bad
        assert fn(1, 2, 200, 300, 64, 2, 1, C.byref(n)) == bclib.OK


def test_binding_refuses_tensors_that_do_not_fit(bclib):
    bf = torch.bfloat16
    q, k, blocks = torch.zeros(2, 200, 3, 32, dtype=bf), torch.zeros(2, 100, 3, 32, dtype=bf), torch.zeros(2, 3, 2, 5, dtype=torch.int32)
    ok = dict(q=q, k=k, blocks=blocks, lens=None)
    bad = [dict(k=torch.zeros(2, 100, 3, 64, dtype=bf)), dict(k=k.float()), dict(k=torch.zeros(1, 100, 3, 32, dtype=bf)),
           dict(q=q.transpose(1, 2)), dict(blocks=blocks.long()), dict(blocks=blocks[:, :, :1]), dict(blocks=blocks[..., ::2]),
           dict(lens=torch.zeros(3, dtype=torch.int32)), dict(lens=torch.zeros(2, dtype=torch.int64))]
    for kw in bad:
        a = dict(ok, **kw)
        with pytest.raises(bclib.BCError) as e:
            bclib.attention_select(a["q"], a["k"], a["blocks"], lens=a["lens"])
        assert e.value.code == bclib.ERR_INVALID_ARG, kw
        with pytest.raises(bclib.BCError):
            bclib.attention_sparse(a["q"], a["k"], k, a["blocks"], q, lens=a["lens"])
    for call in (lambda: bclib.attention_select(q, k, blocks), lambda: bclib.attention_sparse(q, k, k, blocks, q.clone())):
        with pytest.raises(bclib.BCError) as e:                                           # tensors of the host
            call()
        assert e.value.code == bclib.ERR_INVALID_ARG
    for v, out in ((k[:, :50], q), (k.float(), q), (k, q.float()), (k, q[:, :100])):
        with pytest.raises(bclib.BCError) as e:
            bclib.attention_sparse(q, k, v, blocks, out)
        assert e.value.code == bclib.ERR_INVALID_ARG


def test_oracle_against_dense_attention():
    """All blocks listed, the attention is the plain one; one block, that block's."""
    g = np.random.default_rng(0)
    q, k, v = g.standard_normal((150, 8)), g.standard_normal((100, 8)), g.standard_normal((100, 8))
    s = q @ k.T / math.sqrt(8)
    p = np.exp(s)
    dense = (p / p.sum(1, keepdims=True)) @ v
    assert np.allclose(sparse.attend(q, k, v, np.array([[0, 1], [0, 1]]))[0], dense)
    got = sparse.attend(q, k, v, np.array([[1, -1], [-1, 0]]))[0]
    one = np.exp(s[:128, 64:])
    assert np.allclose(got[:128], (one / one.sum(1, keepdims=True)) @ v[64:]) and not got[128:].any()
    assert sparse.list_of([0, 2, 2, 3], 9) == [0, 2] and sparse.list_of([3, 1], 9) == [3] and sparse.list_of([9], 9) == []


# ---------------------------------------------------------------------------
# GPU
# ---------------------------------------------------------------------------
def _qkv(B, H, Tq, Tk, d, dt, seed=0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    mk = lambda T: torch.empty((B, T, H, d), device=DEV).normal_(generator=g).to(TDT[dt])
    q, k, v = mk(Tq), mk(Tk), mk(Tk)
    k += (torch.empty((B, -(-Tk // 64), H, d), device=DEV).normal_(generator=g).repeat_interleave(64, 1)[:, :Tk]).to(TDT[dt])
    return q, k, v


def _np(t):
    return t.double().cpu().numpy()


def _lens(lens, B):
    return None if lens is None else torch.tensor(lens, dtype=torch.int32, device=DEV)


def _run_select(bc, q, k, keep, lens=None, last=0):
    B, Tq, H, d = q.shape
    Tk = k.shape[1]
    nq = -(-Tq // 128)
    buf = torch.full((B * H * nq * keep + 64,), -7, dtype=torch.int32, device=DEV)
    blocks = buf[32:-32].view(B, H, nq, keep)
    n = bc.attention_select_workspace_size(B, H, Tq, Tk, d, keep, bc.dtype_code(q))
    ws = torch.full((n + 256,), 0xFF, dtype=torch.uint8, device=DEV)      # NaNs, were they read
    bc.attention_select(q, k, blocks, lens=_lens(lens, B), keep_last=last, ws=ws[:n])
    torch.cuda.synchronize()
    assert bool((buf[:32] == -7).all()) and bool((buf[-32:] == -7).all()) and bool((ws[n:] == 0xFF).all())
    return blocks


def _want_select(q, k, keep, lens=None, last=0):
    B, Tq, H, d = q.shape
    Tk = k.shape[1]
    q, k = _np(q), _np(k)
    n = [Tk] * B if lens is None else [min(max(x, 0), Tk) for x in lens]
    return np.stack([np.stack([sparse.select(q[b, :, h], k[b, :n[b], h], keep, last) for h in range(H)]) for b in range(B)])


SELECT = [  # B, H, Tq, Tk, d, keep, lens, last
    (1, 1, 1, 1, 32, 1, None, 0), (2, 3, 128, 64, 64, 3, None, 0), (1, 2, 129, 65, 72, 1, None, 1), (2, 2, 300, 1000, 128, 5, None, 2),
    (3, 2, 500, 640, 64, 4, [640, 0, 129], 1), (2, 1, 257, 4096, 72, 13, [5000, -3], 0), (1, 4, 1000, 8256, 32, 20, None, 0),
    (1, 3, 2100, 4161, 64, 64, None, 3), (1, 2, 640, 16384, 32, 70, [16321], 5), (1, 1, 130, 70001, 64, 33, None, 0),
    (1, 1, 5, 70001, 128, 1024, [69999], 0), (2, 5, 700, 777, 32, 50, [777, 64], 50), (2, 1, 140, 66000, 72, 40, [66000, 65601], 1),
    (1, 2, 900, 66000, 32, 9, [130], 2), (2, 1, 2049, 1025, 128, 17, None, 0)]


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,Tq,Tk,d,keep,lens,last", SELECT)
def test_select_lists(bclib, B, H, Tq, Tk, d, keep, lens, last, dt):
    if dt == "f32" and d > 64:
        d = 64
    q, k, _ = _qkv(B, H, Tq, Tk, d, dt, seed=Tq + Tk)
    if lens is not None:
        for b, n in enumerate(lens):
            k[b, max(n, 0):] = float("nan")               # behind a sample's keys: not read
    got = _run_select(bclib, q, k, keep, lens, last).cpu().numpy()
    want = _want_select(q, k, keep, lens, last)
    assert np.array_equal(got, want)


@pytest.mark.gpu
def test_select_ties_and_scores_that_are_not_finite(bclib):
    q, k, _ = _qkv(1, 2, 256, 64 * 200, 64, "bf16", seed=5)
    k = k.view(1, 200, 64, 2, 64)
    k[:, 3::7] = k[:, 3:4]                                # equal blocks: equal scores
    k[:, 150:] = 0.0                                      # and scores of zero
    k[:, 9, 5] = float("nan")
    k[:, 11, 6, :, 0] = float("inf")
    k[:, 12, 6, :, 0] = -float("inf")
    k = k.reshape(1, 64 * 200, 2, 64)
    for keep in (1, 5, 30, 110, 199, 200, 201):
        got = _run_select(bclib, q, k, keep).cpu().numpy()
        assert np.array_equal(got, _want_select(q, k, keep)), keep
    z = torch.zeros_like(q)
    got = _run_select(bclib, z, torch.zeros_like(k), 6).cpu().numpy()
    assert (got == np.arange(6)).all()                    # all equal: the lowest


def _lists(B, H, Tq, Tk, keep, seed, kind="mixed"):
    """Random ascending lists; mixed: full, short, empty and malformed ones."""
    g = np.random.default_rng(seed)
    nq, nk = -(-Tq // 128), -(-Tk // 64)
    out = np.full((B, H, nq, keep), -1, np.int32)
    for n, at in enumerate(np.ndindex(B, H, nq)):
        m = min(keep, nk)
        e = np.sort(g.choice(nk, m, replace=False))
        how = n % 6 if kind == "mixed" else 0
        if how == 1:
            e = e[:len(e) // 2]
        elif how == 2:
            e = e[:0]
        elif how == 3 and len(e) > 1:
            e[1] = e[0]                                   # the same block twice: ends there
        elif how == 4 and len(e) > 2:
            e[2] = [nk, 2 ** 31 - 1, -2 ** 31][n % 3]     # past the end, or far out: ends there
        out[at][:len(e)] = e
    return out


def _check_attend(bc, q, k, v, lists, lens=None, prescaled=False, keep_bits=None):
    B, Tq, H, d = q.shape
    Tk = k.shape[1]
    blocks = torch.from_numpy(np.ascontiguousarray(lists)).to(DEV)
    n = bc.attention_sparse_workspace_size(B, H, Tq, Tk, d, lists.shape[3], bc.dtype_code(q))
    ws = torch.full((n + 512,), 0xFF, dtype=torch.uint8, device=DEV)
    buf = torch.full((q.numel() + 64,), 7.0, dtype=q.dtype, device=DEV)
    out = buf[32:-32].view(q.shape)
    bc.attention_sparse(q, k, v, blocks, out, lens=_lens(lens, B), ws=ws[:n], prescaled=prescaled)
    torch.cuda.synchronize()
    assert bool((buf[:32] == 7.0).all()) and bool((buf[-32:] == 7.0).all()) and bool((ws[n:] == 0xFF).all())
    qn, kn, vn, got = (_np(t) for t in (q, k, v, out))
    for b in range(B):
        m = Tk if lens is None else min(max(lens[b], 0), Tk)
        for h in range(H):
            want, A, top = sparse.attend(qn[b, :, h], kn[b, :m, h], vn[b, :m, h], lists[b, h],
                                         math.log(2.0) if prescaled else None)
            if q.dtype == torch.bfloat16:
                tol = 2.0 ** -8 * 1.02 * (2 * A + np.abs(want)) + 1e-30
            else:
                u = 2.0 ** -24
                tol = A * (2 * (d + 3) * u * top + (lists.shape[3] * 64 + 20) * u) + 1e-30
            err = np.abs(got[b, :, h] - want)
            assert np.all(err <= tol), (b, h, float((err / tol).max()))
            assert not got[b, :, h][(A == 0).all(axis=1)].any()
    return out


ATTEND = [  # B, H, Tq, Tk, d, keep, lens
    (1, 1, 1, 1, 32, 1, None), (1, 2, 1, 700, 64, 4, None), (2, 2, 128, 64, 72, 2, None), (1, 3, 129, 65, 128, 2, None),
    (2, 3, 513, 1000, 64, 7, None), (3, 2, 400, 640, 72, 5, [640, 0, 129]), (2, 2, 1024, 1024, 128, 9, [1, 1023]),
    (2, 1, 300, 300, 32, 5, [900, -1]), (1, 2, 2000, 2111, 128, 33, None), (1, 1, 3, 20000, 64, 200, [19999]),
    (1, 4, 1, 40000, 128, 500, None), (1, 2, 130, 9000, 72, 100, None), (2, 2, 128, 6400, 32, 100, [6400, 3000]),
    (1, 3, 17, 900, 72, 9, None), (2, 2, 64, 6400, 128, 60, [6400, 2000]), (1, 2, 33, 4480, 32, 70, None), (1, 2, 16, 5000, 64, 79, [4999]),
    (1, 2, 600, 3000, 64, 20, None)]


@pytest.mark.gpu
@pytest.mark.parametrize("form", ["bf16", "prescaled", "f32"])
@pytest.mark.parametrize("kind", ["full", "mixed"])
@pytest.mark.parametrize("B,H,Tq,Tk,d,keep,lens", ATTEND)
def test_attention_over_lists(bclib, B, H, Tq, Tk, d, keep, lens, kind, form):
    if form == "f32":
        d = min(d, 64)
        d = 64 if d == 72 else d
    q, k, v = _qkv(B, H, Tq, Tk, d, "f32" if form == "f32" else "bf16", seed=Tq * 3 + Tk)
    if form == "prescaled":
        q = (q.float() * (math.log2(math.e) / math.sqrt(d))).bfloat16()
    if lens is not None:                                  # what lies behind a sample's keys is not read
        for b, n in enumerate(lens):
            k[b, max(n, 0):] = float("nan")
            v[b, max(n, 0):] = float("inf")
    _check_attend(bclib, q, k, v, _lists(B, H, Tq, Tk, keep, seed=Tk + keep, kind=kind), lens, prescaled=form == "prescaled")


@pytest.mark.gpu
@pytest.mark.parametrize("d", [32, 64, 72, 128])
def test_blocks_outside_the_lists_are_not_read(bclib, d):
    """Keys and values of unlisted blocks are NaN; a list longer than a wave's 64 lanes."""
    B, H, Tq, Tk, keep = 1, 2, 260, 64 * 150 - 9, 70
    q, k, v = _qkv(B, H, Tq, Tk, d, "bf16", seed=d)
    lists = np.tile(np.sort(np.random.default_rng(d).choice(150, keep, replace=False)).astype(np.int32), (B, H, 3, 1))
    for j in set(range(150)) - set(lists[0, 0, 0].tolist()):
        k[:, 64 * j:64 * j + 64] = float("nan")
        v[:, 64 * j:64 * j + 64] = float("nan")
    _check_attend(bclib, q, k, v, lists)


@pytest.mark.gpu
def test_large_scores(bclib):
    """Scores of several hundred that grow from block to block: the running maximum moves at every one."""
    q, k, v = _qkv(1, 1, 200, 64 * 12, 64, "bf16", seed=8)
    k *= torch.arange(1, 64 * 12 + 1, device=DEV, dtype=torch.float32).div(40).view(1, -1, 1, 1).bfloat16()
    lists = np.tile(np.arange(12, dtype=np.int32), (1, 1, 2, 1))
    _check_attend(bclib, q, k, v, lists)
    _check_attend(bclib, q, k.flip(1), v, lists)


@pytest.mark.gpu
@pytest.mark.parametrize("prescaled", [False, True])
@pytest.mark.parametrize("d,H,Tq", [(32, 32, 1), (64, 16, 3), (72, 14, 16), (128, 8, 1)])
def test_single_tokens_over_long_lists(bclib, d, H, Tq, prescaled):
    """81 MB of listed keys and values: past the caches' reach."""
    B, Tk = 4, 5005
    q, k, v = _qkv(B, H, Tq, Tk, d, "bf16", seed=d)
    if prescaled:
        q = (q.float() * (math.log2(math.e) / math.sqrt(d))).bfloat16()
    lists = np.tile(np.arange(79, dtype=np.int32), (B, H, 1, 1))
    lists[1, :, :, 5:] = -1
    lists[3, 0] = -1
    _check_attend(bclib, q, k, v, lists, [5005, 5000, 4801, 64], prescaled)


@pytest.mark.gpu
@pytest.mark.parametrize("Tq,d", [(1, 32), (1, 64), (70, 64), (200, 32)])
def test_fp32_lists_in_parts(bclib, Tq, d):
    """One to three blocks a part, scores that grow from block to block, parts
    beyond a short list's end, and NaN in every block that no list names."""
    Tk = 64 * 40 - 17
    q, k, v = _qkv(1, 2, Tq, Tk, d, "f32", seed=d + Tq)
    k *= torch.arange(1, Tk + 1, device=DEV, dtype=torch.float32).div(200).view(1, -1, 1, 1)
    lists = np.full((1, 2, -(-Tq // 128), 30), -1, np.int32)
    lists[0, 0, :, :30] = np.arange(9, 39)
    lists[0, 1, :, :3] = [11, 20, 39]
    for j in (0, 3, 8):
        k[:, 64 * j:64 * j + 64] = float("nan")
        v[:, 64 * j:64 * j + 64] = float("nan")
    a = _check_attend(bclib, q, k, v, lists)
    assert torch.equal(a, _check_attend(bclib, q, k, v, lists))


@pytest.mark.gpu
def test_all_blocks_agree_with_dense_attention(bclib):
    """Listing every block gives bc_attention's result up to the order of the sums."""
    q, k, v = _qkv(2, 3, 700, 700, 128, "bf16", seed=2)
    lists = np.tile(np.arange(11, dtype=np.int32), (2, 3, 6, 1))
    got = _check_attend(bclib, q, k, v, lists)
    dense = torch.empty_like(q)
    bclib.attention(q, k, v, dense)
    assert float((got.float() - dense.float()).abs().max()) <= 2.0 ** -6


@pytest.mark.gpu
def test_select_then_attend_captured(bclib):
    """Both calls in one graph on another stream, replayed with new inputs."""
    B, H, Tq, Tk, d, keep = 2, 4, 700, 1500, 64, 6
    q, k, v = _qkv(B, H, Tq, Tk, d, "bf16")
    lens = torch.tensor([1500, 900], dtype=torch.int32, device=DEV)
    blocks = torch.zeros((B, H, 6, keep), dtype=torch.int32, device=DEV)
    out = torch.empty_like(q)
    code = bclib.BF16
    ws = torch.empty(max(bclib.attention_select_workspace_size(B, H, Tq, Tk, d, keep, code),
                         bclib.attention_sparse_workspace_size(B, H, Tq, Tk, d, keep, code)), dtype=torch.uint8, device=DEV)

    def call(blk, o):
        bclib.attention_select(q, k, blk, lens=lens, keep_last=1, ws=ws)
        bclib.attention_sparse(q, k, v, blk, o, lens=lens, ws=ws)

    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        call(blocks, out)
    for seed in range(3):
        for t in (q, k, v):
            t.normal_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        b2, o2 = torch.empty_like(blocks), torch.empty_like(out)
        call(b2, o2)
        torch.cuda.synchronize()
        assert torch.equal(b2, blocks) and torch.equal(o2, out)
        assert np.array_equal(blocks.cpu().numpy(), _want_select(q, k, keep, [1500, 900], 1))


@pytest.mark.gpu
@pytest.mark.parametrize("Tq", [1, 3, 16, 17, 100])
@pytest.mark.parametrize("d", [32, 64, 72, 128])
@pytest.mark.parametrize("Tk", [64 * 5, 64 * 100])
def test_a_value_that_all_keys_share_comes_back(bclib, Tk, d, Tq):
    """The weights of a row add up to one whatever the probabilities' rounding: one
    key of every block scores 0 and all others -255/256 (log2 units), whose
    probability 0.5014 is rounded to 0.5, 0.27 % lower; over a sum of the unrounded
    ones an output would be 0.9974 of the value, which bf16 tells from a power of two."""
    q, k, v = (torch.zeros(1, T, 1, d, dtype=torch.bfloat16, device=DEV) for T in (Tq, Tk, Tk))
    q[..., 0] = 1.0
    k[..., 0] = -255.0 / 256.0
    k[:, ::64, :, 0] = 0.0
    v[:] = torch.arange(1, d + 1, device=DEV).bfloat16()
    lists = np.tile(np.arange(-(-Tk // 64), dtype=np.int32), (1, 1, 1, 1))
    out = _check_attend(bclib, q, k, v, lists, prescaled=True)
    assert torch.equal(out, v[:, :1].expand_as(out))


SELECT_LONG = [  # 257 to 1024 key blocks: B, H, Tq, Tk, d, keep, lens, last
    (1, 2, 300, 16385, 32, 70, None, 0), (3, 1, 129, 20011, 64, 300, [16384, 20011, 16385], 2), (2, 2, 2049, 40000, 72, 33, [32768 + 187, 32768], 1),
    (1, 1, 257, 65536, 128, 1024, None, 0), (2, 1, 200, 65536, 128, 100, [49153, 65535], 5), (1, 1, 16, 65473, 64, 1, None, 0),
    (1, 2, 17, 33000, 32, 516, [33000], 500), (1, 1, 1, 16400, 72, 256, None, 256)]


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,Tq,Tk,d,keep,lens,last", SELECT_LONG)
def test_select_lists_of_long_samples(bclib, B, H, Tq, Tk, d, keep, lens, last, dt):
    """A wave takes several tiles of 16 key blocks, the workgroup 256 a round; samples end inside a round and just behind one."""
    test_select_lists(bclib, B, H, Tq, Tk, d, keep, lens, last, dt)


@pytest.mark.gpu
def test_select_ties_of_long_samples(bclib):
    q, k, _ = _qkv(1, 1, 140, 64 * 1000, 64, "bf16", seed=6)
    k = k.view(1, 1000, 64, 1, 64)
    k[:, 3::7] = k[:, 3:4]                                # equal blocks in every round
    k[:, 900:] = 0.0
    k[:, 300, 5] = float("nan")
    k[:, 511, 6, :, 0] = float("inf")
    k = k.reshape(1, 64 * 1000, 1, 64)
    for keep in (1, 30, 143, 300, 600, 999, 1000, 1001):
        got = _run_select(bclib, q, k, keep).cpu().numpy()
        assert np.array_equal(got, _want_select(q, k, keep)), keep
    got = _run_select(bclib, torch.zeros_like(q), torch.zeros_like(k), 300).cpu().numpy()
    assert (got == np.arange(300)).all()


@pytest.mark.gpu
@pytest.mark.parametrize("Tq", [1, 16, 17, 64, 300])
@pytest.mark.parametrize("d,dt", [(32, "bf16"), (64, "bf16"), (72, "bf16"), (128, "bf16"), (32, "f32"), (64, "f32")])
@pytest.mark.parametrize("lens", [None, [700, 129, 64, 1]])
def test_infinite_values_of_a_last_key(bclib, lens, d, dt, Tq):
    """A sample's keys end inside a block: its last key's values reach the output
    once, as infinity of their sign, whatever stands in for the keys behind it."""
    B, H, Tk, keep = 4, 2, 777, 6
    q, k, v = _qkv(B, H, Tq, Tk, d, dt, seed=d + Tq)
    n = lens or [Tk] * B
    for b in range(B):
        v[b, n[b] - 1, :, 1], v[b, n[b] - 1, :, 3], v[b, n[b] - 1, :, d - 1] = math.inf, -math.inf, math.nan
    lists = np.full((B, H, -(-Tq // 128), keep), -1, np.int32)
    for b in range(B):
        last = -(-n[b] // 64) - 1
        own = sorted({0, last // 2, last})
        lists[b, :, :, :len(own)] = own
    blocks = torch.from_numpy(lists).to(DEV)
    size = bclib.attention_sparse_workspace_size(B, H, Tq, Tk, d, keep, bclib.dtype_code(q))
    ws = torch.full((size + 256,), 0xFF, dtype=torch.uint8, device=DEV)
    out = torch.empty_like(q)
    bclib.attention_sparse(q, k, v, blocks, out, lens=_lens(lens, B), ws=ws)
    got = _np(out)
    assert (got[..., 1] == math.inf).all() and (got[..., 3] == -math.inf).all() and np.isnan(got[..., d - 1]).all()
    got[..., [1, 3, d - 1]] = 0.0
    assert np.isfinite(got).all()


@pytest.mark.gpu
@pytest.mark.parametrize("Tq,d,dt", [(1, 128, "bf16"), (40, 128, "bf16"), (200, 72, "bf16"), (70, 64, "f32")])
def test_keys_beyond_32_bit_offsets(bclib, Tq, d, dt):
    """262 144 keys of enough heads that the last ones' offsets do not fit 32 bits: lists and outputs of the outer heads."""
    Tk, keep = 262144, 5
    H = -(-((1 << 31) + (1 << 28)) // (Tk * d))
    g = torch.Generator(device=DEV)
    g.manual_seed(Tq)
    mk = lambda T: torch.empty((1, T, H, d), dtype=TDT[dt], device=DEV).normal_(generator=g)
    q, k, v = mk(Tq), mk(Tk), mk(Tk)
    assert k.numel() > 1 << 31
    got = _run_select(bclib, q, k, keep, last=1)
    lists = np.tile(np.array([0, 2047, 3500, 4094, 4095], np.int32), (1, H, -(-Tq // 128), 1))
    blocks = torch.from_numpy(lists).to(DEV)
    n = bclib.attention_sparse_workspace_size(1, H, Tq, Tk, d, keep, bclib.dtype_code(q))
    ws = torch.empty(max(n, 256), dtype=torch.uint8, device=DEV)
    out = torch.empty_like(q)
    bclib.attention_sparse(q, k, v, blocks, out, ws=ws)
    for h in (0, H - 1):
        qn, kn, vn, on = (_np(t[0, :, h]) for t in (q, k, v, out))
        assert np.array_equal(got[0, h].cpu().numpy(), sparse.select(qn, kn, keep, 1))
        want, A, top = sparse.attend(qn, kn, vn, lists[0, h])
        u = 2.0 ** -24
        tol = 2.0 ** -8 * 1.02 * (2 * A + np.abs(want)) if dt == "bf16" else A * (2 * (d + 3) * u * top + (keep * 64 + 20) * u)
        assert np.all(np.abs(on - want) <= tol + 1e-30), h
