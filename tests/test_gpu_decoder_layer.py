"""The 4-bit decoder operators together, as a decoder layer uses them: prompts of different lengths, then single tokens from a captured graph."""
import math

import numpy as np
import pytest
import torch

import lvx_synth as S
from oracle import decoder_oracle as O
from oracle.lvx_oracle import gelu_tanh
from test_gpu_fp8 import e4m3_decode

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
H, KV, D, FFN, SEQS, LAYERS, MAX = 6, 2, 64, 512, 3, 2, 150
DM = H * D
QKV = (H + 2 * KV) * D


def model(lvx):
    layers = []
    for l in range(LAYERS):
        w = {}
        for name, n, k in (("qkv", QKV, DM), ("o", DM, DM), ("up", FFN, DM), ("down", DM, FFN)):
            w[name] = lvx.lvx_fp4_quantize(S.randn_bf16((n, k), S.seed_of("layer", name, l), 1 / math.sqrt(k), device=DEV))
        for name in ("g1", "g2"):
            w[name] = 1 + 0.1 * S.randn_f32((DM,), S.seed_of("layer", name, l), 1.0, device=DEV)
        layers.append(w)
    return layers


class Buffers:
    def __init__(self, lvx, cache, n, most):
        e = lambda *s, dtype=torch.bfloat16: torch.empty(*s, dtype=dtype, device=DEV)
        self.x8, self.s8, self.qkv, self.att = e(n, DM, dtype=torch.uint8), e(n, dtype=torch.float32), e(n, QKV), e(n, DM)
        self.up, self.most = e(n, FFN), most
        self.ws = e(lvx.lvx_kv4_attention_workspace_bytes(cache, H, most), dtype=torch.uint8)


def forward(lvx, layers, cache, h, counts, starts, b, look=lambda *a: None):
    """h: fp32 residual stream [n][DM], updated in place.  `look` is told of every operator and what it took and gave."""
    for l, w in enumerate(layers):
        lvx.lvx_rmsnorm_residual_fp8(None, h, w["g1"], 1e-6, b.x8, b.s8)
        look("norm", h, w["g1"], b.x8, b.s8)
        lvx.lvx_linear_fp8_fp4(b.x8, b.s8, *w["qkv"], b.qkv)
        look("linear8", b.x8, b.s8, w["qkv"], b.qkv, lambda x: x)
        q, k, v = b.qkv[:, :DM], b.qkv[:, DM:DM + KV * D], b.qkv[:, DM + KV * D:]
        lvx.lvx_kv4_append(cache, l, k, v, counts, starts=starts, max_tokens=b.most)
        lvx.lvx_kv4_attention(cache, l, q, H, 1 / math.sqrt(D), counts, b.att, b.ws, starts=starts, max_tokens=b.most)
        look("attention", l, q, k, v, b.att)
        before = h.clone() if look.__name__ != "<lambda>" else None
        lvx.lvx_linear_fp4(b.att, *w["o"], h, lvx.EPI_RESID_GATE_F32, resid=h)
        look("linear16", b.att, w["o"], before, h)
        lvx.lvx_rmsnorm_residual_fp8(None, h, w["g2"], 1e-6, b.x8, b.s8)
        look("norm", h, w["g2"], b.x8, b.s8)
        lvx.lvx_linear_fp8_fp4(b.x8, b.s8, *w["up"], b.up, lvx.EPI_GELU_TANH)
        look("linear8", b.x8, b.s8, w["up"], b.up, gelu_tanh)
        before = h.clone() if look.__name__ != "<lambda>" else None
        lvx.lvx_linear_fp4(b.up, *w["down"], h, lvx.EPI_RESID_GATE_F32, resid=h)
        look("linear16", b.up, w["down"], before, h)


def weight64(q, s):
    q = q.cpu().numpy()
    codes = np.stack([q & 15, q >> 4], -1).reshape(q.shape[0], -1)
    return (O.e2m1_value(codes).reshape(len(q), -1, 32) * np.exp2(s.cpu().numpy().astype(np.float64) - 127)[..., None]).reshape(codes.shape)


class Follow:
    """Every operator against 64 bits on the numbers that it was given; the tolerances are those of the operators' own tests."""
    __name__ = "follow"

    def __init__(self):
        self.kv = [[(np.zeros((0, KV, D)),) * 2 for _ in range(SEQS)] for _ in range(LAYERS)]
        self.new = None

    def __call__(self, what, *a):
        getattr(self, what)(*a)

    def norm(self, h, g, q, s):
        _, ref = O.rmsnorm_residual(None, S.to_f64(h), S.to_f64(g), 1e-6)
        s64, e32 = S.to_f64(s)[:, None], (DM / 2 + 8) * 2.0 ** -24
        assert np.all(np.abs(e4m3_decode(q.cpu().numpy()) * s64 - ref) <= (2.0 ** -4 + 4 * e32 + 2.0 ** -20) * np.abs(ref) + 2.0 ** -10 * s64)

    def linear8(self, q, s, w, out, act):
        a, w64 = e4m3_decode(q.cpu().numpy()) * S.to_f64(s)[:, None], weight64(*w)
        x, off = a @ w64.T, (a.shape[1] + 8) * 2.0 ** -24 * (np.abs(a) @ np.abs(w64).T)
        assert np.all(np.abs(S.to_f64(out) - act(x)) <= 2.0 ** -8 * np.abs(act(x)) + 2 * off + 2.0 ** -18 * np.abs(x))

    def linear16(self, a, w, before, out):
        a, w64 = S.to_f64(a), weight64(*w)
        want, off = S.to_f64(before) + a @ w64.T, (a.shape[1] + 8) * 2.0 ** -24 * (np.abs(a) @ np.abs(w64).T)
        assert np.all(np.abs(S.to_f64(out) - want) <= 2.0 ** -24 * np.abs(want) + 2 * off)

    def attention(self, l, q, k, v, out):
        q, k, v, got, at = S.to_f64(q), S.to_f64(k), S.to_f64(v), S.to_f64(out), 0
        for s, n in enumerate(self.new):
            new = O.quantise_groups(k[at:at + n])[2].reshape(n, KV, D), O.quantise_vectors(v[at:at + n].reshape(n, KV, D))[2]
            self.kv[l][s] = tuple(np.concatenate(x) for x in zip(self.kv[l][s], new))
            c = len(self.kv[l][s][0])
            ref, spread, size = O.attention(q[at:at + n].reshape(n, H, D), *self.kv[l][s], 1 / math.sqrt(D), [c - (n - 1 - i) for i in range(n)])
            tol = 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 2.0 ** -16 + 2 * (D + 4) * 2.0 ** -24 * size[..., None]) * spread
            assert np.all(np.abs(got[at:at + n].reshape(n, H, D) - ref) <= tol)
            at += n


def stream(n, *tag):
    return S.randn_f32((n, DM), S.seed_of("layer_h", *tag), 1.0, device=DEV)


def test_prompts_then_single_tokens(lvx):
    """Prompts of different lengths, single tokens, an idle sequence, a second prompt behind the first."""
    layers, follow = model(lvx), Follow()
    cache = lvx.KV4Cache(lvx.kv4_desc(LAYERS, SEQS, KV, D, MAX), DEV)
    cache.storage.fill_(0xff)
    lengths = np.zeros(SEQS, int)
    for step, new in enumerate([(70, 3, 31), (1, 1, 1), (1, 1, 1), (0, 40, 1), (1, 1, 1)]):
        lengths, follow.new = lengths + np.array(new), new
        forward(lvx, layers, cache, stream(sum(new), step), torch.tensor(lengths, dtype=torch.int32, device=DEV),
                torch.tensor([0, *np.cumsum(new)], dtype=torch.int32, device=DEV), Buffers(lvx, cache, sum(new), max(new)), follow)


def test_captured_steps_replay_with_other_lengths(lvx):
    """One captured step of single tokens, replayed while the lengths grow on the device, against the same steps run eagerly, bit for bit."""
    layers = model(lvx)
    steps = 6

    def start(cache):
        cache.storage.fill_(0xff)
        h = stream(60, "prompt")
        counts = torch.tensor([30, 10, 20], dtype=torch.int32, device=DEV)
        forward(lvx, layers, cache, h, counts, torch.tensor([0, 30, 40, 60], dtype=torch.int32, device=DEV), Buffers(lvx, cache, 60, 30))
        return counts

    eager = lvx.KV4Cache(lvx.kv4_desc(LAYERS, SEQS, KV, D, MAX), DEV)
    counts, want = start(eager), []
    b = Buffers(lvx, eager, SEQS, 1)
    for i in range(steps):
        counts += 1
        h = stream(SEQS, "tok", i)
        forward(lvx, layers, eager, h, counts, None, b)
        want.append(h)

    cache = lvx.KV4Cache(lvx.kv4_desc(LAYERS, SEQS, KV, D, MAX), DEV)
    counts = start(cache)
    h, given = torch.empty(SEQS, DM, device=DEV), torch.empty(SEQS, DM, device=DEV)
    own = Buffers(lvx, cache, SEQS, 1)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        counts.add_(1)
        h.copy_(given)
        forward(lvx, layers, cache, h, counts, None, own)
    for i in range(steps):
        given.copy_(stream(SEQS, "tok", i))
        graph.replay()
        assert torch.equal(h, want[i]), i
        torch.cuda.synchronize()
