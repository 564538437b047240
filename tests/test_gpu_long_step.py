"""The operators for long samples run together, as a program that drives its own
blocks uses them: attention over selected blocks, module outputs normed, gated
and added, the stepwise feature into a quantised ring, and forecasts from it.

Each stage is checked against float64 on the inputs it got, within its own
bound (tests/test_sparse_attention.py, test_norm_residual.py,
test_quant_cache.py), and the whole step against a float64 step that is given
the selected blocks: every stage rounds its output to bf16 once (2^-8), as do
the probabilities, eight roundings on the way to the stream, whose update is the
smaller part of it; 8 x 2^-8 of the update bounds the stream's error."""
import math

import numpy as np
import pytest

from oracle import quant, sparse

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
B, T, H, D_HEAD, MLP = 2, 900, 4, 64, 512
D = H * D_HEAD
KEEP, K = 5, 3
LENS = [900, 650]
BF = torch.bfloat16


class Step:
    """Buffers and weights of one block; run() enqueues a full step."""

    def __init__(self, bc, bits):
        g = torch.Generator(device=DEV)
        g.manual_seed(3)
        rnd = lambda *s, scale=1.0: torch.empty(*s, device=DEV).normal_(0, scale, generator=g)
        self.bc = bc
        self.w = {n: rnd(*s, scale=1.5 / math.sqrt(s[-1])).to(BF) for n, s in
                  dict(q=(D, D), k=(D, D), v=(D, D), o=(D, D), up=(MLP, D), down=(D, MLP)).items()}
        self.mods = rnd(B, 6 * D, scale=0.3)
        self.post = [(1 + rnd(D, scale=0.1)).to(BF) for _ in range(2)]
        self.x = rnd(B * T, D)
        self.lens = torch.tensor(LENS, dtype=torch.int32, device=DEV)
        e = lambda *s, dt=BF: torch.zeros(*s, dtype=dt, device=DEV)
        self.h, self.h2, self.y, self.y2, self.attn = (e(B * T, D) for _ in range(5))
        self.q, self.k, self.v = (e(B, T, H, D_HEAD) for _ in range(3))
        self.mlp = e(B * T, MLP)
        self.x1, self.x2, self.out = (e(B * T, D, dt=torch.float32) for _ in range(3))
        self.zero = e(B * T, D)
        self.blocks = torch.zeros((B, H, -(-T // 128), KEEP), dtype=torch.int32, device=DEV)
        n = max(bc.attention_select_workspace_size(B, H, T, T, D_HEAD, KEEP, bc.BF16),
                bc.attention_sparse_workspace_size(B, H, T, T, D_HEAD, KEEP, bc.BF16), 256)
        self.ws = torch.empty(n, dtype=torch.uint8, device=DEV)
        store = torch.empty(bc.quant_cache_bytes(K, B * T * D, bits), dtype=torch.uint8, device=DEV)
        self.ring = bc.QuantCacheRing(K, B * T * D, torch.float32, bits, store)

    def mod(self, i):
        return self.mods[:, i * D:(i + 1) * D]

    def run(self, t):
        bc, w = self.bc, self.w
        # The block's first norm: nothing to add yet.
        bc.norm_gate_residual(self.zero, self.x, self.x1, self.h, rows_per_sample=T, pre=bc.NORM_LAYER,
                              shift=self.mod(0), scale=self.mod(1))
        for n in "qkv":
            bc.linear(self.h, w[n], None, getattr(self, n).view(B * T, D))
        bc.attention_select(self.q, self.k, self.blocks, lens=self.lens, keep_last=1, ws=self.ws)
        bc.attention_sparse(self.q, self.k, self.v, self.blocks, self.attn.view(B, T, H, D_HEAD), lens=self.lens, ws=self.ws)
        bc.linear(self.attn, w["o"], None, self.y)
        bc.norm_gate_residual(self.y, self.x, self.x1, self.h2, rows_per_sample=T, post=bc.NORM_RMS, post_w=self.post[0],
                              gate=self.mod(2), pre=bc.NORM_LAYER, shift=self.mod(3), scale=self.mod(4))
        bc.linear(self.h2, w["up"], None, self.mlp, bc.EPI_BIAS_GELU)
        bc.linear(self.mlp, w["down"], None, self.y2)
        bc.norm_gate_residual(self.y2, self.x1, self.x2, rows_per_sample=T, post=bc.NORM_RMS, post_w=self.post[1], gate=self.mod(5))
        self.ring.push(self.x2, t)


def _np(t):
    return t.double().cpu().numpy()


def _layer(v, shift, scale):
    n = (v - v.mean(1, keepdims=True)) / np.sqrt(v.var(1, keepdims=True) + 1e-6)
    return n * (1 + scale) + shift


def _rms(v, w):
    return v / np.sqrt((v * v).mean(1, keepdims=True) + 1e-6) * w


def _gelu(v):
    return 0.5 * v * (1 + np.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3)))


def _heads(v):
    return v.reshape(B, T, H, D_HEAD)


def _float64_step(s, blocks):
    """The step in float64 (weights and stream as the GPU has them) over the given blocks."""
    w = {n: _np(t) for n, t in s.w.items()}
    m = [np.repeat(_np(s.mod(i)), T, 0) for i in range(6)]
    x = _np(s.x)
    h = _layer(x, m[0], m[1])
    q, k, v = (_heads(h @ w[n].T) for n in "qkv")
    o = np.zeros_like(q)
    for b in range(B):
        for i in range(H):
            o[b, :, i] = sparse.attend(q[b, :, i], k[b, :LENS[b], i], v[b, :LENS[b], i], blocks[b, i])[0]
    x1 = x + m[2] * _rms(o.reshape(B * T, D) @ w["o"].T, _np(s.post[0]))
    h2 = _layer(x1, m[3], m[4])
    return x1 + m[5] * _rms(_gelu(h2 @ w["up"].T) @ w["down"].T, _np(s.post[1]))


def _check_step(s):
    """Every stage on the inputs it got, and the whole."""
    q, k, v, blocks = _np(s.q), _np(s.k), _np(s.v), s.blocks.cpu().numpy()
    at = _heads(_np(s.attn))
    for b in range(B):
        for i in range(H):
            assert np.array_equal(blocks[b, i], sparse.select(q[b, :, i], k[b, :LENS[b], i], KEEP, 1))
            want, A, _ = sparse.attend(q[b, :, i], k[b, :LENS[b], i], v[b, :LENS[b], i], blocks[b, i])
            assert np.all(np.abs(at[b, :, i] - want) <= 2.0 ** -8 * 1.02 * (2 * A + np.abs(want)))
    m = [np.repeat(_np(s.mod(i)), T, 0) for i in range(6)]
    x1 = _np(s.x) + m[2] * _rms(_np(s.y), _np(s.post[0]))
    assert np.abs(_np(s.x1) - x1).max() <= 1e-5 * np.abs(x1).max()
    h2 = _layer(_np(s.x1), m[3], m[4])
    assert np.all(np.abs(_np(s.h2) - h2) <= 2.0 ** -8 * np.abs(h2) + 1e-4)
    x2 = _np(s.x1) + m[5] * _rms(_np(s.y2), _np(s.post[1]))
    assert np.abs(_np(s.x2) - x2).max() <= 1e-5 * np.abs(x2).max()
    want = _float64_step(s, blocks)
    err = np.linalg.norm(_np(s.x2) - want) / np.linalg.norm(want - _np(s.x))
    print(f"step error {err:.2e} of its update")
    assert err <= 8 * 2.0 ** -8


@pytest.mark.parametrize("bits", [8, 4])
def test_full_steps_and_forecasts(bclib, bits):
    s = Step(bclib, bits)
    stored, times = [], [0.0, 4.0, 8.0, 12.0]
    for t in times:
        s.run(t)
        torch.cuda.synchronize()
        _check_step(s)
        stored.insert(0, quant.held(_np(s.x2).astype(np.float32), bits))
        if len(stored) >= 2:
            n = min(K, len(stored))
            w = bclib.bary_weights([float(v) for v in reversed(times[:len(stored)])][:n], t + 2.0)
            bclib.bary_extrapolate(s.ring, w, s.out)
            want = sum(a * f for a, f in zip(w, stored))
            tol = 2 * (n + 2) * 2.0 ** -24 * sum(abs(a) * np.abs(f) for a, f in zip(w, stored))
            assert np.all(np.abs(_np(s.out) - want) <= tol)
        s.x.add_(torch.randn_like(s.x), alpha=0.3)      # the next full step's stream
    s.ring.read(K - 1, s.out)
    assert np.array_equal(s.out.cpu().numpy(), stored[K - 1].astype(np.float32))


def test_step_captured_and_replayed(bclib):
    """One full step and a forecast in a graph; replays, with the program's own
    eager work between them, give the eager bits."""
    s = Step(bclib, 8)
    s.run(0.0)
    torch.cuda.synchronize()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        s.run(1.0)
        bclib.bary_extrapolate(s.ring, [1.5, -0.5], s.out)
    for seed in range(3):
        torch.manual_seed(seed)
        s.x.normal_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        x2, out = s.x2.clone(), s.out.clone()
        first = Step(bclib, 8)
        first.run(0.0)
        first.x.copy_(s.x)
        first.run(1.0)
        bclib.bary_extrapolate(first.ring, [1.5, -0.5], first.out)
        torch.cuda.synchronize()
        assert torch.equal(first.x2, x2) and torch.equal(first.out, out)
