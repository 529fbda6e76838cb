"""The 4-bit cache: appended rows bit for bit, attention against the 64-bit oracle on the decoded cache.

Tolerance of an attention output: the probability is rounded to bf16 once (2^-8 of itself, times |v| summed: 2^-8 * sum p|v|), the output once (2^-8 of
itself); a score is off by at most (D + 4) * 2^-24 of scale * sum |q||k| (D products added in fp32, the scale's two roundings), which moves a probability
by twice that, and the exponential and the sums add less than 2^-16."""
import math

import numpy as np
import pytest
import torch

import lvx_synth as S
from oracle import decoder_oracle as O

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def rows(n, width, *tag):
    return S.randn_bf16((n, width), S.seed_of(*tag), 1.0, device=DEV)


def gathered(lvx, cache, layer, counts, n_keys, first=0):
    d = cache.desc
    k = torch.full((d.n_seqs, n_keys, d.n_kv_heads * d.head_dim + 8), 7.0, dtype=torch.bfloat16, device=DEV)
    v = k.clone()
    w = d.n_kv_heads * d.head_dim
    lvx.lvx_kv4_gather(cache, layer, counts, k[:, :, :w], v[:, :, :w], first_key=first)
    assert bool((k[:, :, w:] == 7).all()) and bool((v[:, :, w:] == 7).all())
    return (S.to_f64(t[:, :, :w]).reshape(d.n_seqs, n_keys, d.n_kv_heads, d.head_dim) for t in (k, v))


def decoded(k, KV, D):
    return O.quantise_groups(S.to_f64(k))[2].reshape(-1, KV, D)


def decoded_v(v, KV, D):
    return O.quantise_vectors(S.to_f64(v).reshape(-1, KV, D))[2]


@pytest.mark.parametrize("KV,D", [(1, 64), (3, 64), (2, 128), (5, 128)])
def test_append_in_pieces(lvx, KV, D):
    """Prompts and steps of ragged lengths: every piece lands where its keys belong and leaves its neighbours as they were."""
    S_, L, n_layers = 4, 203, 2
    cache = lvx.KV4Cache(lvx.kv4_desc(n_layers, S_, KV, D, L), DEV)
    cache.storage.fill_(0xff)
    want = [[(np.zeros((0, KV, D)), np.zeros((0, KV, D))) for _ in range(S_)] for _ in range(n_layers)]
    lengths = [0] * S_
    for step, new in enumerate([(5, 0, 64, 1), (1, 1, 1, 1), (70, 3, 9, 0), (0, 8, 1, 130), (1, 1, 1, 1), (100, 2, 7, 64)]):
        lengths = [a + b for a, b in zip(lengths, new)]
        starts, counts = i32([0] + list(np.cumsum(new))), i32(lengths)
        for l in range(n_layers):
            ld = 2 * KV * D + 8
            kv = rows(sum(new) + 1, ld, "app", KV, D, step, l)
            k, v = kv[:sum(new), :KV * D], kv[:sum(new), KV * D:2 * KV * D]
            lvx.lvx_kv4_append(cache, l, k, v, counts, starts=starts, max_tokens=max(new))
            dk, dv, at = decoded(k, KV, D), decoded_v(v, KV, D), 0
            for s in range(S_):
                a, b = want[l][s]
                want[l][s] = (np.concatenate([a, dk[at:at + new[s]]]), np.concatenate([b, dv[at:at + new[s]]]))
                at += new[s]
    for l in range(n_layers):
        k, v = gathered(lvx, cache, l, i32(lengths), L)
        for s in range(S_):
            n = lengths[s]
            assert np.array_equal(k[s, :n], want[l][s][0]) and np.array_equal(v[s, :n], O.bf16(want[l][s][1]))
            assert not k[s, n:].any() and not v[s, n:].any()
        k2, v2 = gathered(lvx, cache, l, i32(lengths), 60, first=70)
        assert np.array_equal(k2, k[:, 70:130]) and np.array_equal(v2, v[:, 70:130])


def test_append_outside_the_slot(lvx):
    """Tokens in front of the first and behind the last place are dropped; ranges that leave the rows are cut."""
    KV, D, L = 2, 64, 40
    cache = lvx.KV4Cache(lvx.kv4_desc(1, 3, KV, D, L), DEV)
    cache.storage.zero_()
    k, v = rows(30, KV * D, "out_k"), rows(30, KV * D, "out_v")
    lvx.lvx_kv4_append(cache, 0, k, v, i32([4, 45, -3]), starts=i32([0, 10, 20, 30]), max_tokens=10)
    gk, gv = gathered(lvx, cache, 0, i32([40, 99, 40]), L)
    dk, dv = decoded(k, KV, D), O.bf16(decoded_v(v, KV, D))
    assert np.array_equal(gk[0, :4], dk[6:10]) and np.array_equal(gv[0, :4], dv[6:10]) and not gk[0, 4:].any()
    assert np.array_equal(gk[1, 35:], dk[10:15]) and np.array_equal(gv[1, 35:], dv[10:15]) and not gk[1, :35].any()
    assert not gk[2].any() and not gv[2].any()
    cache.storage.zero_()
    lvx.lvx_kv4_append(cache, 0, k, v, i32([4, 4, 4]), starts=i32([-5, 3, 27, 99]), max_tokens=4, n_tokens=12)
    gk, _ = gathered(lvx, cache, 0, i32([4, 4, 4]), L)
    assert np.array_equal(gk[0, 1:4], dk[:3]) and not gk[0, 0].any()      # rows 0 .. 2 of the range [-5, 3)
    assert np.array_equal(gk[1, :4], dk[3:7])                              # four of [3, 12): no more than max_tokens
    assert not gk[2].any()                                                 # [27, 99) lies behind the last row


def test_non_finite_keys_and_values(lvx):
    KV, D = 1, 128
    cache = lvx.KV4Cache(lvx.kv4_desc(1, 1, KV, D, 64), DEV)
    k, v = rows(20, D, "nf_k").clone(), rows(20, D, "nf_v").clone()
    k[3, 40], v[5, 7], v[6, 0] = float("nan"), float("inf"), float("nan")
    lvx.lvx_kv4_append(cache, 0, k, v, i32([20]), max_tokens=20)
    gk, gv = gathered(lvx, cache, 0, i32([20]), 20)
    assert np.isnan(gk[0, 3, 0, 32:64]).all() and np.isfinite(gk[0, 3, 0, :32]).all() and np.isfinite(gk[0, 3, 0, 64:]).all()
    assert not np.isfinite(gv[0, 5]).any() and np.isnan(gv[0, 6]).all() and np.isfinite(gv[0, [0, 4, 7, 19]]).all()
    q = rows(20, D, "nf_q")
    ws = torch.empty(lvx.lvx_kv4_attention_workspace_bytes(cache, 1, 20), dtype=torch.uint8, device=DEV)
    out = torch.empty_like(q)
    lvx.lvx_kv4_attention(cache, 0, q, 1, 0.1, i32([20]), out, ws, max_tokens=20)
    # what a token does not see does not reach it
    assert bool(torch.isfinite(out[:3]).all()) and bool(torch.isnan(out[3:]).all())


def make(lvx, S_, KV, D, L, counts, tag, fill=0xff):
    """A cache whose slots hold other keys (or whatever the memory held) behind their sequences."""
    cache = lvx.KV4Cache(lvx.kv4_desc(2, S_, KV, D, L), DEV)
    cache.storage.fill_(fill)
    wide = torch.exp(S.randn_f32((KV * D,), S.seed_of(tag, "wide"), 0.7, device=DEV))
    k = (rows(S_ * L, KV * D, tag, "k").float() * wide).to(torch.bfloat16)
    v = rows(S_ * L, KV * D, tag, "v")
    if fill == 0xff:
        starts = [0] + list(np.cumsum([max(0, min(c, L)) for c in counts]))
        lvx.lvx_kv4_append(cache, 1, k, v, i32([max(0, min(c, L)) for c in counts]), starts=i32(starts), max_tokens=L)
        return cache, [(decoded(k[a:b], KV, D), decoded_v(v[a:b], KV, D)) for a, b in zip(starts, starts[1:])]
    lvx.lvx_kv4_append(cache, 1, k, v, i32([L] * S_), max_tokens=L)
    return cache, [(decoded(k[s * L:(s + 1) * L], KV, D), decoded_v(v[s * L:(s + 1) * L], KV, D)) for s in range(S_)]


def check(lvx, cache, kv, q, H, scale, counts, new, causal, starts=None, out=None):
    D, T = cache.desc.head_dim, sum(new)
    out = torch.full((q.shape[0] + 1, H * D + 8), 7.0, dtype=torch.bfloat16, device=DEV) if out is None else out
    ws = torch.empty(lvx.lvx_kv4_attention_workspace_bytes(cache, H, max(new)), dtype=torch.uint8, device=DEV).fill_(0xff)
    st = None if starts is None else i32(starts)
    lvx.lvx_kv4_attention(cache, 1, q, H, scale, i32(counts), out[:q.shape[0], :H * D], ws, starts=st, max_tokens=max(new), causal=causal, n_tokens=q.shape[0] if starts is None else T)
    got, qn, at = S.to_f64(out), S.to_f64(q), 0
    for s, n in enumerate(new):
        k, v = kv[s]
        c = min(counts[s], cache.desc.max_keys)
        seen = [c - (n - 1 - i) if causal else c for i in range(n)]
        ref, spread, size = O.attention(qn[at:at + n].reshape(n, H, D), k, v, scale, seen)
        tol = 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 2.0 ** -16 + 2 * (D + 4) * 2.0 ** -24 * size[..., None]) * spread
        err = np.abs(got[at:at + n, :H * D].reshape(n, H, D) - ref)
        assert np.all(err <= tol), (s, float((err - tol).max()), np.argwhere(err > tol)[:4].tolist())
        at += n
    assert bool((out[T:] == 7).all()) and bool((out[:, H * D:] == 7).all())   # rows behind the last sequence, columns behind the last head
    return out


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("KV,group,n,L,causal", [(1, 1, 1, 1, True), (2, 1, 1, 63, True), (2, 4, 1, 65, True), (1, 5, 3, 200, True), (3, 8, 2, 129, False),
                                                 (2, 7, 5, 640, True), (1, 16, 1, 1500, True), (4, 3, 1, 1100, False), (1, 1, 40, 333, True),
                                                 (2, 2, 130, 131, True), (1, 6, 50, 90, False), (2, 1, 300, 700, True)])
def test_attention(lvx, D, KV, group, n, L, causal):
    """Batches of one length: single tokens, a few, prompts, with every number of heads to a kv head."""
    S_, H = 3, KV * group
    tag = "att%d_%d_%d_%d_%d" % (D, KV, group, n, L)
    counts = [L, max(n // 2, 1), max(1, L // 2)]
    cache, kv = make(lvx, S_, KV, D, L, counts, tag)
    q = rows(S_ * n, H * D + 16, tag, "q")[:, :H * D]
    a = check(lvx, cache, kv, q, H, 1 / math.sqrt(D), counts, [n] * S_, causal)
    b = check(lvx, cache, kv, q, H, 1 / math.sqrt(D), counts, [n] * S_, causal)
    assert torch.equal(a, b)


@pytest.mark.parametrize("fill", [0xff, 0])
@pytest.mark.parametrize("KV,group,D,L,new,counts,causal", [
    (2, 5, 128, 300, (1, 0, 7, 1, 33), (300, 120, 7, 0, 64), True),         # an idle slot, one without keys, a whole prompt
    (2, 5, 128, 300, (1, 0, 7, 1, 33), (300, 120, 3, -5, 20), True),        # tokens in front of the first key see nothing
    (1, 3, 64, 2600, (2, 1, 1, 9, 0), (2600, 2500, 64, 65, 5), False),
    (4, 2, 64, 1030, (64, 1, 200, 3, 1), (1030, 4000, 200, 3, 1), True),    # a count beyond the slot
    (8, 5, 128, 4000, (1, 1, 1, 1, 1), (4000, 3999, 1, 63, 2049), True),
])
def test_attention_ragged(lvx, fill, KV, group, D, L, new, counts, causal):
    tag = "rag%d_%d_%d_%d" % (KV, group, D, L)
    H = KV * group
    cache, kv = make(lvx, len(new), KV, D, L, counts, tag, fill)
    starts = [0] + list(np.cumsum(new))
    q = rows(sum(new) + 5, H * D, tag, "q")
    check(lvx, cache, kv, q, H, 1 / math.sqrt(D), counts, new, causal, starts=starts)


@pytest.mark.parametrize("scale", [1e-3, 1.0, -0.2])
def test_attention_scales(lvx, scale):
    """Near-uniform, very peaked and negative scales."""
    counts = [900, 17]
    cache, kv = make(lvx, 2, 2, 128, 900, counts, "scales")
    q = rows(2 * 3, 4 * 128, "scales_q")
    check(lvx, cache, kv, q, 4, scale, counts, [3, 3], True)


def test_attention_growing_scores(lvx):
    """Scores that grow along the keys: the softmax reference moves in every tile."""
    KV, D, L = 1, 128, 1200
    cache = lvx.KV4Cache(lvx.kv4_desc(2, 1, KV, D, L), DEV)
    q = rows(2, D, "grow_q")
    k = (q[:1].float() * torch.linspace(-6, 6, L, device=DEV)[:, None]).to(torch.bfloat16)
    v = rows(L, D, "grow_v")
    lvx.lvx_kv4_append(cache, 1, k, v, i32([L]), max_tokens=L)
    check(lvx, cache, [(decoded(k, KV, D), decoded_v(v, KV, D))], q, 1, 0.2, [L], [2], True)


def test_attention_in_place_and_another_stream(lvx):
    counts = [700, 300, 12]
    cache, kv = make(lvx, 3, 2, 128, 700, counts, "inplace")
    q = rows(3 * 2, 6 * 128, "inplace_q")
    want = check(lvx, cache, kv, q, 6, 0.09, counts, [2, 2, 2], True)[:6, :6 * 128]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both = q.clone()
        ws = torch.empty(lvx.lvx_kv4_attention_workspace_bytes(cache, 6, 2), dtype=torch.uint8, device=DEV)
        lvx.lvx_kv4_attention(cache, 1, both, 6, 0.09, i32(counts), both, ws, max_tokens=2)
    side.synchronize()
    assert torch.equal(both, want)


def test_offsets_beyond_32_bits(lvx):
    """The last sequence of the last layer of a cache of 5 GB: all keys and values zero but the last ones."""
    KV, D, L, S_, n = 8, 128, 131072, 12, 70
    cache = lvx.KV4Cache(lvx.kv4_desc(3, S_, KV, D, L), DEV)
    assert cache.storage.numel() > 1 << 32
    cache.storage.zero_()
    k, v = rows(n, KV * D, "far_k"), rows(n, KV * D, "far_v")
    starts, counts = i32([0] * S_ + [n]), i32([0] * (S_ - 1) + [L])
    lvx.lvx_kv4_append(cache, 2, k, v, counts, starts=starts, max_tokens=n)
    k_out = torch.empty(S_, n, KV * D, dtype=torch.bfloat16, device=DEV)
    v_out = torch.empty_like(k_out)
    lvx.lvx_kv4_gather(cache, 2, counts, k_out, v_out, first_key=L - n)
    dk, dv = decoded(k, KV, D), decoded_v(v, KV, D)
    assert np.array_equal(S.to_f64(k_out[-1]), dk.reshape(n, -1))
    assert np.array_equal(S.to_f64(v_out[-1]), O.bf16(dv).reshape(n, -1)) and not bool(k_out[:-1].any())
    q = rows(1, KV * D, "far_q")
    out = torch.empty_like(q)
    ws = torch.empty(lvx.lvx_kv4_attention_workspace_bytes(cache, KV, 1), dtype=torch.uint8, device=DEV)
    lvx.lvx_kv4_attention(cache, 2, q, KV, 1.0, counts, out, ws, starts=i32([0] * S_ + [1]))
    x = np.einsum("hd,jhd->jh", S.to_f64(q).reshape(KV, D), dk)
    p = np.exp(x) / (np.exp(x).sum(0) + L - n)
    ref, spread = np.einsum("jh,jhd->hd", p, dv), np.einsum("jh,jhd->hd", p, np.abs(dv))
    size = np.einsum("hd,jhd->jh", np.abs(S.to_f64(q).reshape(KV, D)), np.abs(dk)).max()
    assert np.all(np.abs(S.to_f64(out).reshape(KV, D) - ref) <= 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 2.0 ** -16 + 2 * (D + 4) * 2.0 ** -24 * size) * spread)


@pytest.mark.parametrize("group,n,count", [(1, 10, 75), (1, 40, 90), (8, 30, 1000), (2, 9, 2 ** 31 - 1)])
def test_counts_beyond_the_slot(lvx, group, n, count):
    """A count that passes the slot: every token sees the keys up to its own place, as append stored them, or all there are."""
    KV, D, L = 2, 64, 70
    tag = "over%d_%d_%d" % (group, n, count)
    cache = lvx.KV4Cache(lvx.kv4_desc(1, 1, KV, D, L), DEV)
    k, v, q = rows(L, KV * D, tag, "k"), rows(L, KV * D, tag, "v"), rows(n, KV * group * D, tag, "q")
    lvx.lvx_kv4_append(cache, 0, k, v, i32([L]), max_tokens=L)
    ws = torch.empty(lvx.lvx_kv4_attention_workspace_bytes(cache, KV * group, n), dtype=torch.uint8, device=DEV)
    out, each = torch.empty_like(q), torch.empty_like(q)
    lvx.lvx_kv4_attention(cache, 0, q, KV * group, 0.125, i32([count]), out, ws, max_tokens=n)
    lvx.lvx_kv4_attention(cache, 0, q, KV * group, 0.125, i32([L]), each, ws, max_tokens=n, causal=False)
    seen = [min(count - (n - 1 - i), L) for i in range(n)]
    ref, spread, size = O.attention(S.to_f64(q).reshape(n, -1, D), decoded(k, KV, D), decoded_v(v, KV, D), 0.125, seen)
    tol = 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 2.0 ** -16 + 2 * (D + 4) * 2.0 ** -24 * size[..., None]) * spread
    assert np.all(np.abs(S.to_f64(out).reshape(ref.shape) - ref) <= tol)
    if min(seen) == L:
        assert torch.equal(out, each)


@pytest.mark.parametrize("H,n,L", [(1, 20, 64), (4, 20, 20), (8, 20, 90)])
def test_unlikely_values_that_are_not_finite(lvx, H, n, L):
    """A value that is no number reaches the tokens that see it though its probability underflows to zero, wherever its key lies in a tile."""
    D = 128
    cache = lvx.KV4Cache(lvx.kv4_desc(1, 1, 1, D, L), DEV)
    q = rows(1, D, "unlikely").expand(n, D).repeat(1, H).contiguous()
    k, v = rows(L, D, "unlikely_k", L).clone(), rows(L, D, "unlikely_v", L).clone()
    k[L - 10] = (-10 * q[0, :D].float()).to(torch.bfloat16)      # a score near -10 * 128
    v[L - 10] = float("nan")
    lvx.lvx_kv4_append(cache, 0, k, v, i32([L]), max_tokens=L)
    ws = torch.empty(lvx.lvx_kv4_attention_workspace_bytes(cache, H, n), dtype=torch.uint8, device=DEV)
    out = torch.empty_like(q)
    lvx.lvx_kv4_attention(cache, 0, q, H, 1.0, i32([L]), out, ws, max_tokens=n)
    assert bool(torch.isfinite(out[:n - 10]).all()) and bool(torch.isnan(out[n - 10:]).all())


# sequences, kv heads, heads of a group, tokens, keys; rows of a workgroup, whether the keys are split (tests/test_kv4_rules.py holds the rule to them)
FORMS = [(3, 1, 3, 5, 129, 16, False), (1, 1, 1, 1, 3000, 16, True), (1, 2, 3, 700, 3000, 32, False), (1, 1, 3, 700, 9000, 32, True),
         (1, 8, 8, 130, 130, 64, False), (1, 2, 3, 1500, 9000, 64, True), (16, 8, 5, 64, 130, 128, False), (2, 8, 8, 130, 9000, 128, True)]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("S_,KV,group,n,L,rows_,splits", FORMS)
def test_every_form(lvx, D, S_, KV, group, n, L, rows_, splits):
    """Every form of the kernel with one range of keys and with several, on ragged tokens and lengths; some tokens of each sequence against the oracle."""
    tag, H = "form%d_%d_%d_%d_%d" % (D, KV, group, n, L), KV * group
    new = [max(1, n - 5 * s) for s in range(S_)]
    counts = [max(1, L - 40 * s) if s % 3 < 2 else new[s] // 2 for s in range(S_)]
    cache, kv = make(lvx, S_, KV, D, L, counts, tag)
    starts = [0] + list(np.cumsum(new))
    q = rows(sum(new), H * D, tag, "q")
    for causal in (True, False):
        out = torch.full((sum(new) + 1, H * D), 7.0, dtype=torch.bfloat16, device=DEV)
        ws = torch.empty(lvx.lvx_kv4_attention_workspace_bytes(cache, H, n) + 64, dtype=torch.uint8, device=DEV).fill_(0xff)
        for _ in range(2):
            lvx.lvx_kv4_attention(cache, 1, q, H, 1 / math.sqrt(D), i32(counts), out, ws[:-64], starts=i32(starts), max_tokens=n, causal=causal)
        assert bool((ws[-64:] == 0xff).all()) and bool((out[-1] == 7).all()) and bool(torch.isfinite(out).all())
        for s in range(S_):
            at = sorted({0, 1, new[s] // 3, new[s] // 2, new[s] - 1} & set(range(new[s])))
            sel = [starts[s] + i for i in at]
            seen = [counts[s] - (new[s] - 1 - i) if causal else counts[s] for i in at]
            ref, spread, size = O.attention(S.to_f64(q[sel]).reshape(-1, H, D), *kv[s], 1 / math.sqrt(D), seen)
            tol = 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 2.0 ** -16 + 2 * (D + 4) * 2.0 ** -24 * size[..., None]) * spread
            err = np.abs(S.to_f64(out[sel]).reshape(ref.shape) - ref)
            assert np.all(err <= tol), (s, causal, float((err - tol).max()))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("S_,KV,group,n,L,rows_,splits", FORMS)
def test_keys_whose_scores_overflow(lvx, D, S_, KV, group, n, L, rows_, splits):
    """The first keys' scores pass fp32 below (-infinity: probability zero), those behind them are finite and negative: they alone make the output."""
    H, hidden = KV * group, L // 2 // 64 * 64 + 10
    cache = lvx.KV4Cache(lvx.kv4_desc(1, S_, KV, D, L), DEV)
    q = torch.full((S_ * n, H * D), 2.0 ** 60, dtype=torch.bfloat16, device=DEV)
    k = (-(2.0 ** -60) * (1 + 0.3 * rows(S_ * L, KV * D, "over_k", L).float().tanh())).to(torch.bfloat16).view(S_, L, KV * D)
    k[:, :hidden] = -(2.0 ** 70)
    v = rows(S_ * L, KV * D, "over_v", L)
    counts = i32([L] * S_)
    lvx.lvx_kv4_append(cache, 0, k.flatten(0, 1), v, counts, max_tokens=L)
    ws = torch.empty(lvx.lvx_kv4_attention_workspace_bytes(cache, H, n), dtype=torch.uint8, device=DEV)
    out = torch.empty_like(q)
    lvx.lvx_kv4_attention(cache, 0, q, H, 0.1, counts, out, ws, max_tokens=n, causal=False)
    dk, dv = decoded(k[0, hidden:], KV, D), decoded_v(v[hidden:L], KV, D)
    ref, spread, size = O.attention(S.to_f64(q[:1]).reshape(1, H, D), dk, dv, 0.1, [L - hidden])
    tol = 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 2.0 ** -16 + 2 * (D + 4) * 2.0 ** -24 * size[..., None]) * spread
    assert np.all(np.abs(S.to_f64(out[:n]).reshape(n, H, D) - ref) <= tol)


# sequences, kv heads, heads of a group, tokens, keys; rows of a workgroup: in the last block of rows fewer than a token's heads are left
IN_PLACE = [(1, 6, 5, 141, 200, 16), (1, 2, 3, 715, 3000, 32), (4, 6, 5, 205, 300, 64), (1, 8, 5, 1549, 1560, 64), (16, 8, 5, 77, 130, 128), (16, 6, 5, 77, 130, 128)]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("S_,KV,group,n,L,rows_", IN_PLACE)
def test_in_place(lvx, D, S_, KV, group, n, L, rows_):
    """Outputs over the queries are the bits of outputs elsewhere: no workgroup reads a query that another may have stored over."""
    tag, H = "place%d_%d_%d" % (KV, n, L), KV * group
    cache = lvx.KV4Cache(lvx.kv4_desc(1, S_, KV, D, L), DEV)
    counts = i32([L - s for s in range(S_)])
    lvx.lvx_kv4_append(cache, 0, rows(S_ * L, KV * D, tag, "k"), rows(S_ * L, KV * D, tag, "v"), i32([L] * S_), max_tokens=L)
    q = rows(S_ * n, H * D, tag, "q")
    ws = torch.empty(lvx.lvx_kv4_attention_workspace_bytes(cache, H, n), dtype=torch.uint8, device=DEV)
    out = torch.empty_like(q)
    lvx.lvx_kv4_attention(cache, 0, q, H, 1.0, counts, out, ws, max_tokens=n)
    for _ in range(4):
        both = q.clone()
        lvx.lvx_kv4_attention(cache, 0, both, H, 1.0, counts, both, ws, max_tokens=n)
        assert torch.equal(both, out)
