"""4-bit quantisation (bit for bit) and the linears with 4-bit weights against the 64-bit oracle.

Tolerance of a product: every term is exact in fp32 or its operands are, and K terms are added in fp32 in some order, so the sum is off by at most
(K + 8) * 2^-24 * sum_k |a w|; a bf16 output by half a step (2^-8 of itself) more.  Many 8-bit rows with bf16 outputs may go through the matrix cores' mixed
8-bit x 4-bit product, which lines four neighbouring channels' products up with the largest of them and cuts what lies 12 binary places below its leading bit: at most
2^-12 of that largest for each of the three others, so 3 * 2^-12 * sum over the fours of max |a| max |w| for an output (test_mixed_products_lose_no_more_than_that
holds the instruction to it).  GELU is 1.13-Lipschitz and its own fp32 evaluation is off by at most
2^-18 of |x| (its exponential's argument reaches tens)."""
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


def unpack(q):
    q = q.cpu().numpy()
    return np.stack([q & 15, q >> 4], -1).reshape(q.shape[0], -1)


@pytest.mark.parametrize("rows,cols,std", [(5, 32, 1.0), (37, 96, 0.02), (1, 4096, 30.0), (130, 160, 1e-3)])
def test_quantize_codes_and_scales(lvx, rows, cols, std):
    x = S.randn_bf16((rows, cols + 8), S.seed_of("fp4q", rows, cols), std, device=DEV)[:, :cols].clone()
    pad = torch.empty(rows, cols + 8, dtype=torch.bfloat16, device=DEV)
    x[0, :32] = 0
    x[rows // 2, 3] = 7.0 * 2.0 ** 20                       # exactly at the border of a scale
    x[rows - 1, 1] = 7.0625
    x[0, cols - 1] = -0.0
    pad[:, :cols] = x
    q = torch.full((rows + 1, -(-(cols // 2) // 16) * 16 + 16), 0x5a, dtype=torch.uint8, device=DEV)
    s = torch.full((rows + 1, cols // 32 + 3), 0x5a, dtype=torch.uint8, device=DEV)
    lvx.lvx_fp4_quantize(pad[:, :cols], q[:rows, :cols // 2], s[:rows, :cols // 32])
    code, e, _ = O.quantise_groups(S.to_f64(x))
    got = unpack(q[:rows, :cols // 2])
    zero = O.LEVELS[code & 7] == 0                           # the sign of a zero is kept, too
    assert np.array_equal(got, code) and zero.any()
    assert np.array_equal(s[:rows, :cols // 32].cpu().numpy().astype(np.int64) - 127, e)
    assert bool((q[rows] == 0x5a).all()) and bool((q[:, cols // 2:] == 0x5a).all()) and bool((s[rows] == 0x5a).all()) and bool((s[:, cols // 32:] == 0x5a).all())


def test_quantize_non_finite_groups(lvx):
    x = torch.ones(2, 96, dtype=torch.bfloat16, device=DEV)
    x[0, 40], x[1, 95] = float("nan"), float("-inf")
    q, s = lvx.lvx_fp4_quantize(x)
    s = s.cpu().numpy()
    assert s[0, 1] == 255 and s[1, 2] == 255 and (s != 255).sum() == 4
    # every such group makes NaN of the outputs that read it
    c = torch.zeros(1, 8, device=DEV)
    w, ws = q[:1].repeat(8, 1), torch.tensor(s[:1], device=DEV).repeat(8, 1)
    ws[4:] = 127
    for m in (1, 70):
        c = torch.zeros(m, 8, device=DEV)
        lvx.lvx_linear_fp4(torch.ones(m, 96, dtype=torch.bfloat16, device=DEV), w, ws, c, lvx.EPI_STORE_F32)
        assert bool(torch.isnan(c[:, :4]).all()) and bool(torch.isfinite(c[:, 4:]).all())


def weights(lvx, N, K, tag):
    w = S.randn_bf16((N, K), S.seed_of(tag, "w", N, K), 1 / math.sqrt(K), device=DEV) * torch.exp2(torch.randint(-3, 4, (N, 1), device=DEV).float()).to(torch.bfloat16)
    q, s = lvx.lvx_fp4_quantize(w)
    codes = unpack(q)
    return q, s, (O.e2m1_value(codes).reshape(N, -1, 32) * np.exp2(s.cpu().numpy().astype(np.float64) - 127)[..., None]).reshape(N, K)


def rows8(M, K, tag):
    """E4M3 codes without NaN, some of them subnormal, and a scale per row."""
    c = S.randn_f32((M, K), S.seed_of(tag, "a8", M, K), 60.0, device=DEV).to(torch.float8_e4m3fn).view(torch.uint8).clone()
    c[:, ::7] &= 0x83
    s = torch.exp(S.randn_f32((M,), S.seed_of(tag, "s8", M), 1.0, device=DEV)) / 448
    return c, s, e4m3_decode(c.cpu().numpy()) * S.to_f64(s)[:, None]


def products(lvx, M, N, K, a8, tag):
    q, s, w = weights(lvx, N, K, tag)
    if a8:
        c, sa, a = rows8(M, K, tag)
        call = lambda out, *x, **k: lvx.lvx_linear_fp8_fp4(c, sa, q, s, out, *x, **k)
    else:
        x = S.randn_bf16((M, K + 8), S.seed_of(tag, "a", M, K), 1.0, device=DEV)[:, :K]
        a = S.to_f64(x)
        call = lambda out, *z, **k: lvx.lvx_linear_fp4(x, q, s, out, *z, **k)
    off = (K + 8) * 2.0 ** -24 * (np.abs(a) @ np.abs(w).T)
    return call, a @ w.T, off, mixed(a, w) if a8 and M > 32 else 0.0


def mixed(a, w):
    fours = lambda x: np.abs(x).reshape(len(x), -1, 4).max(-1)
    return 3 * 2.0 ** -12 * (fours(a) @ fours(w).T)


SHAPES = [(1, 8, 32), (1, 264, 5120), (2, 40, 96), (15, 72, 160), (16, 520, 1184), (17, 64, 224), (31, 8, 4096), (33, 136, 128), (48, 1032, 608),
          (64, 256, 64), (65, 24, 352), (100, 392, 1120), (129, 128, 512), (257, 648, 288), (544, 1288, 416)]


# and products that fill the chip: every height of a tile, one step and many, odd numbers of steps and of pairs, a step that is not whole, scales of more than 48 steps
TILES = [(40, 5464, 32), (35, 6000, 416), (70, 4104, 6304), (545, 2568, 96), (550, 5000, 544), (544, 2560, 160), (33, 13824, 768), (97, 5128, 1024)]
# few rows of many channels, which lie in LDS whole: one and several blocks of columns, steps that the waves share unevenly, a step that is not whole
LONG = [(1, 8, 4096), (1, 8200, 5120), (3, 40, 4128), (2, 8232, 6304), (7, 136, 4000), (13, 264, 4096), (4, 72, 13824)]


@pytest.mark.parametrize("a8", [False, True])
@pytest.mark.parametrize("M,N,K", SHAPES + TILES + LONG)
def test_linear(lvx, M, N, K, a8):
    call, ref, off, cut = products(lvx, M, N, K, a8, "lin")
    out = torch.full((M + 1, N + 8), 7.0, dtype=torch.bfloat16, device=DEV)
    call(out[:M, :N])
    assert np.all(np.abs(S.to_f64(out[:M, :N]) - ref) <= 2.0 ** -8 * np.abs(ref) + 2 * (off + cut))
    assert bool((out[M:] == 7).all()) and bool((out[:, N:] == 7).all())
    again = torch.empty_like(out)
    call(again[:M, :N])
    assert torch.equal(again[:M, :N], out[:M, :N])
    o32 = torch.full((M + 1, N + 8), 7.0, device=DEV)
    call(o32[:M, :N], lvx.EPI_STORE_F32)
    assert np.all(np.abs(S.to_f64(o32[:M, :N]) - ref) <= off)
    assert bool((o32[M:] == 7).all()) and bool((o32[:, N:] == 7).all())


@pytest.mark.parametrize("a8", [False, True])
@pytest.mark.parametrize("M,N,K", [(1, 72, 288), (20, 264, 512), (150, 136, 160), (70, 4104, 288), (300, 2568, 160)])
def test_linear_epilogues(lvx, M, N, K, a8):
    call, ref, off, cut = products(lvx, M, N, K, a8, "epi")
    out = torch.empty(M, N, dtype=torch.bfloat16, device=DEV)
    call(out, lvx.EPI_GELU_TANH)
    want = gelu_tanh(ref)
    assert np.all(np.abs(S.to_f64(out) - want) <= 2.0 ** -8 * np.abs(want) + 2 * (off + cut) + 2.0 ** -18 * np.abs(ref))
    r = S.randn_bf16((M, N), S.seed_of("epi_r", M, N), 2.0, device=DEV)
    g = S.randn_f32((N,), S.seed_of("epi_g", N), 1.0, device=DEV)
    for gate in (None, g):
        gg = 1.0 if gate is None else S.to_f64(gate)
        want = S.to_f64(r) + gg * ref
        slack = 2 * (off * np.abs(gg) + 2.0 ** -24 * np.abs(gg * ref))
        c = r.clone()
        call(c, lvx.EPI_RESID_GATE, resid=c, gate=gate)     # in place
        assert np.all(np.abs(S.to_f64(c) - want) <= 2.0 ** -8 * np.abs(want) + slack + 2 * cut * np.abs(gg))
        c = r.float()
        call(c, lvx.EPI_RESID_GATE_F32, resid=c, gate=gate)
        assert np.all(np.abs(S.to_f64(c) - want) <= 2.0 ** -24 * np.abs(want) + slack)


def test_linear_scale_extremes_and_neighbours(lvx):
    """Scale bytes from 2^-100 to 2^100 a row; a NaN in one activation row stays in it."""
    M, N, K = 18, 32, 256
    q, s, w = weights(lvx, N, K, "ext")
    s = torch.randint(27, 228, (N, 1), dtype=torch.uint8, device=DEV).repeat(1, K // 32)
    codes = unpack(q)
    w = (O.e2m1_value(codes).reshape(N, -1, 32) * np.exp2(s.cpu().numpy().astype(np.float64) - 127)[..., None]).reshape(N, K)
    a = S.randn_bf16((M, K), S.seed_of("ext_a"), 1.0, device=DEV).clone()
    a[3, 100] = float("nan")
    c = torch.empty(M, N, device=DEV)
    lvx.lvx_linear_fp4(a, q, s, c, lvx.EPI_STORE_F32)
    keep = [m for m in range(M) if m != 3]
    x = S.to_f64(a)[keep]
    assert np.all(np.abs(S.to_f64(c)[keep] - x @ w.T) <= (K + 8) * 2.0 ** -24 * (np.abs(x) @ np.abs(w).T))
    assert bool(torch.isnan(c[3]).all())


def test_mixed_products_lose_no_more_than_that(lvx):
    """Rows whose channels differ by up to 2^17 within a four, and large terms that cancel: bf16 outputs of many rows within the bound, fp32 outputs within that of fp32 sums."""
    M, N, K = 256, 5120, 128
    c = torch.randint(0, 256, (M, K), device=DEV, generator=torch.Generator(device=DEV).manual_seed(11)).to(torch.uint8)
    c[(c & 127) == 127] = 0
    c[:, 1::16] = c[:, 0::16] ^ 128                    # a pair that cancels where its two weights are equal
    q = torch.randint(0, 256, (N, K // 2), device=DEV, generator=torch.Generator(device=DEV).manual_seed(12)).to(torch.uint8)
    q[:, 0::8] = (q[:, 0::8] & 15) * 17
    s = torch.full((N, K // 32), 127, dtype=torch.uint8, device=DEV)
    one = torch.ones(M, device=DEV)
    a, w = e4m3_decode(c.cpu().numpy()), O.e2m1_value(unpack(q))
    ref, off, cut = a @ w.T, (K + 8) * 2.0 ** -24 * (np.abs(a) @ np.abs(w).T), mixed(a, w)
    out, o32 = torch.empty(M, N, dtype=torch.bfloat16, device=DEV), torch.empty(M, N, device=DEV)
    lvx.lvx_linear_fp8_fp4(c, one, q, s, out)
    lvx.lvx_linear_fp8_fp4(c, one, q, s, o32, lvx.EPI_STORE_F32)
    err = np.abs(S.to_f64(out) - ref) - 2.0 ** -8 * np.abs(ref)
    print("beyond the output's rounding: %.3f of the bound at most" % (err / cut).max(), flush=True)
    assert np.all(err <= cut + off) and np.all(np.abs(S.to_f64(o32) - ref) <= off)


@pytest.mark.parametrize("a8,f32", [(False, False), (True, False), (True, True)])
def test_non_finite_weights_and_rows_of_tiles(lvx, a8, f32):
    """A NaN scale makes NaN of its column, a NaN in a row of its row, whatever lies behind K in a padded row of nothing."""
    M, N, K, pad = 48, 5464, 288, 32
    q, s = lvx.lvx_fp4_quantize(S.randn_bf16((N, K), S.seed_of("nft", "w"), 1.0, device=DEV))
    s = s.clone()
    s[7, 8], s[5000, 0] = 255, 255
    out = torch.empty(M, N, dtype=torch.float32 if f32 else torch.bfloat16, device=DEV)
    if a8:
        a = torch.full((M, K + pad), 0x7f, dtype=torch.uint8, device=DEV)
        a[:, :K] = S.randn_f32((M, K), S.seed_of("nft", "a"), 60.0, device=DEV).to(torch.float8_e4m3fn).view(torch.uint8)
        a[33, 280] = 0x7f
        lvx.lvx_linear_fp8_fp4(a[:, :K], torch.ones(M, device=DEV), q, s, out, lvx.EPI_STORE_F32 if f32 else lvx.EPI_STORE)
    else:
        a = torch.full((M, K + pad), float("nan"), dtype=torch.bfloat16, device=DEV)
        a[:, :K] = S.randn_bf16((M, K), S.seed_of("nft", "a"), 1.0, device=DEV)
        a[33, 280] = float("nan")
        lvx.lvx_linear_fp4(a[:, :K], q, s, out)
    bad = torch.zeros(M, N, dtype=torch.bool, device=DEV)
    bad[:, 7] = bad[:, 5000] = True
    bad[33] = True
    assert torch.equal(torch.isnan(out), bad)


# every tile (rows, columns, groups over K) in each of its three arithmetics (tests/test_fp4_rules.py holds the rule to that), channels up to more than the scales of one panel
FORMS = [(m, n, k) for m, n in ((290, 264), (530, 520), (400, 1288), (200, 4104), (530, 2056), (530, 4104)) for k in (160, 6304)]


@pytest.mark.parametrize("a8", [False, True])
@pytest.mark.parametrize("M,N,K", FORMS)
def test_every_tile(lvx, M, N, K, a8):
    test_linear(lvx, M, N, K, a8)


# rows that lie in LDS whole: blocks of 16 columns to a workgroup for (bf16, 8-bit) rows, 0 for the other kernel
IN_LDS = {(1, 264, 4128): (1, 1), (5, 5128, 5120): (1, 1), (9, 5128, 5120): (2, 1), (16, 2056, 6304): (0, 1), (11, 2056, 6304): (1, 1), (13, 13832, 5120): (0, 2),
          (3, 16456, 4128): (1, 1), (6, 16456, 5152): (4, 4), (16, 5128, 5120): (0, 2), (5, 5128, 13824): (2, 1), (14, 264, 5120): (0, 0)}


@pytest.mark.parametrize("a8", [False, True])
@pytest.mark.parametrize("M,N,K", list(IN_LDS))
def test_rows_in_lds(lvx, M, N, K, a8):
    test_linear(lvx, M, N, K, a8)


def unequal(M, N, K):
    """E4M3 codes that differ by up to 2^17 within a four, with pairs that cancel, and weights that are equal on those pairs."""
    gen = lambda seed: torch.Generator(device=DEV).manual_seed(seed)
    c = torch.randint(0, 256, (M, K), device=DEV, generator=gen(21)).to(torch.uint8)
    c[(c & 127) == 127] = 0
    c[:, 1::16] = c[:, 0::16] ^ 128
    q = torch.randint(0, 256, (N, K // 2), device=DEV, generator=gen(22)).to(torch.uint8)
    q[:, 0::8] = (q[:, 0::8] & 15) * 17
    s = torch.full((N, K // 32), 127, dtype=torch.uint8, device=DEV)
    return c, torch.ones(M, device=DEV), q, s, e4m3_decode(c.cpu().numpy()), O.e2m1_value(unpack(q))


@pytest.mark.parametrize("M,N,K", [(33, 5120, 128), (256, 5120, 128), (530, 520, 160), (96, 4104, 6304)])
def test_many_8bit_rows_are_summed_in_fp32(lvx, M, N, K):
    """Terms far below their neighbours keep their bits, with bf16 outputs as with fp32 ones: those are the same sums, rounded."""
    c, one, q, s, a, w = unequal(M, N, K)
    ref, off = a @ w.T, (K + 8) * 2.0 ** -24 * (np.abs(a) @ np.abs(w).T)
    out, o32 = torch.empty(M, N, dtype=torch.bfloat16, device=DEV), torch.empty(M, N, device=DEV)
    lvx.lvx_linear_fp8_fp4(c, one, q, s, out)
    lvx.lvx_linear_fp8_fp4(c, one, q, s, o32, lvx.EPI_STORE_F32)
    assert np.all(np.abs(S.to_f64(out) - ref) <= 2.0 ** -8 * np.abs(ref) + off) and np.all(np.abs(S.to_f64(o32) - ref) <= off)
    assert torch.equal(out, o32.to(torch.bfloat16))


@pytest.mark.parametrize("M,N,K", [(1, 8200, 5120), (32, 264, 512), (33, 136, 128), (70, 4104, 6304)] + FORMS)
def test_mixed_products_on_request(lvx, M, N, K):
    """With the flag: within the bound of those products in every tile, the same bits from the same call, and no other bits where the rows are few."""
    call, ref, off, cut = products(lvx, M, N, K, True, "mix")
    out = torch.full((M + 1, N + 8), 7.0, dtype=torch.bfloat16, device=DEV)
    call(out[:M, :N], lvx.EPI_STORE | lvx.EPI_MIXED_8X4)
    assert np.all(np.abs(S.to_f64(out[:M, :N]) - ref) <= 2.0 ** -8 * np.abs(ref) + 2 * (off + cut))
    assert bool((out[M:] == 7).all()) and bool((out[:, N:] == 7).all())
    again = torch.empty(M, N, dtype=torch.bfloat16, device=DEV)
    call(again, lvx.EPI_STORE | lvx.EPI_MIXED_8X4)
    assert torch.equal(again, out[:M, :N])
    if M <= 32:
        call(again)
        assert torch.equal(again, out[:M, :N])
    r, g = S.randn_bf16((M, N), S.seed_of("mix_r", M, N), 2.0, device=DEV), S.randn_f32((N,), S.seed_of("mix_g", N), 1.0, device=DEV)
    gg = S.to_f64(g)
    want = S.to_f64(r) + gg * ref
    c = r.clone()
    call(c, lvx.EPI_RESID_GATE | lvx.EPI_MIXED_8X4, resid=c, gate=g)
    assert np.all(np.abs(S.to_f64(c) - want) <= 2.0 ** -8 * np.abs(want) + 2 * (off * np.abs(gg) + 2.0 ** -24 * np.abs(gg * ref)) + 2 * cut * np.abs(gg))
    call(c, lvx.EPI_GELU_TANH | lvx.EPI_MIXED_8X4)
    want = gelu_tanh(ref)
    assert np.all(np.abs(S.to_f64(c) - want) <= 2.0 ** -8 * np.abs(want) + 2 * (off + cut) + 2.0 ** -18 * np.abs(ref))


def test_mixed_products_lose_no_more_than_their_bound(lvx):
    c, one, q, s, a, w = unequal(256, 5120, 128)
    ref, off, cut = a @ w.T, (128 + 8) * 2.0 ** -24 * (np.abs(a) @ np.abs(w).T), mixed(a, w)
    out = torch.empty(256, 5120, dtype=torch.bfloat16, device=DEV)
    lvx.lvx_linear_fp8_fp4(c, one, q, s, out, lvx.EPI_STORE | lvx.EPI_MIXED_8X4)
    err = np.abs(S.to_f64(out) - ref) - 2.0 ** -8 * np.abs(ref)
    print("beyond the output's rounding: %.3f of the bound at most" % (err / cut).max(), flush=True)
    assert np.all(err <= cut + off)


def test_mixed_products_keep_what_is_not_finite(lvx):
    M, N, K = 48, 5464, 288
    q, s = lvx.lvx_fp4_quantize(S.randn_bf16((N, K), S.seed_of("nfm", "w"), 1.0, device=DEV))
    s = s.clone()
    s[7, 8], s[5000, 0] = 255, 255
    a = torch.full((M, K + 32), 0x7f, dtype=torch.uint8, device=DEV)
    a[:, :K] = S.randn_f32((M, K), S.seed_of("nfm", "a"), 60.0, device=DEV).to(torch.float8_e4m3fn).view(torch.uint8)
    a[33, 280] = 0x7f
    out = torch.empty(M, N, dtype=torch.bfloat16, device=DEV)
    lvx.lvx_linear_fp8_fp4(a[:, :K], torch.ones(M, device=DEV), q, s, out, lvx.EPI_STORE | lvx.EPI_MIXED_8X4)
    bad = torch.zeros(M, N, dtype=torch.bool, device=DEV)
    bad[:, 7] = bad[:, 5000] = True
    bad[33] = True
    assert torch.equal(torch.isnan(out), bad)


# products that tiles would take; bytes from row to row, from weight to weight beyond their own, which 32-bit offsets do not reach
FAR_APART = [(50, 4104, 288, 1 << 24, 0), (70, 4104, 160, 1 << 24, 0), (4400, 72, 160, 0, 1 << 24)]


@pytest.mark.parametrize("a8", [False, True])
@pytest.mark.parametrize("M,N,K,lda,ldw", FAR_APART)
def test_rows_far_apart(lvx, M, N, K, lda, ldw, a8):
    q, s, w = weights(lvx, N, K, "far")
    if ldw:
        wide = torch.empty(N, ldw, dtype=torch.uint8, device=DEV)
        wide[:, :K // 2] = q
        q = wide[:, :K // 2]
    if a8:
        x, sa, a = rows8(M, K, "far")
    else:
        x = S.randn_bf16((M, K), S.seed_of("far", "a", M, K), 1.0, device=DEV)
        a = S.to_f64(x)
    if lda:
        wide_a = torch.empty(M, lda // x.element_size(), dtype=x.dtype, device=DEV)
        wide_a[:, :K] = x
        x = wide_a[:, :K]
    ref, off = a @ w.T, (K + 8) * 2.0 ** -24 * (np.abs(a) @ np.abs(w).T)
    out, o32 = torch.empty(M, N, dtype=torch.bfloat16, device=DEV), torch.empty(M, N, device=DEV)
    for c, epi in ((out, lvx.EPI_STORE), (o32, lvx.EPI_STORE_F32)):
        lvx.lvx_linear_fp8_fp4(x, sa, q, s, c, epi) if a8 else lvx.lvx_linear_fp4(x, q, s, c, epi)
    assert np.all(np.abs(S.to_f64(o32) - ref) <= off) and torch.equal(out, o32.to(torch.bfloat16))
    if a8:
        mixed_out = torch.empty_like(out)
        lvx.lvx_linear_fp8_fp4(x, sa, q, s, mixed_out, lvx.EPI_STORE | lvx.EPI_MIXED_8X4)
        assert torch.equal(mixed_out, out)


@pytest.mark.parametrize("M,N,K", [(1, 264, 256), (20, 264, 256), (1, 264, 4096), (16, 2056, 4096), (600, 2056, 256), (300, 4104, 160)])
def test_every_end_of_the_scales(lvx, M, N, K):
    """One weight a column, all codes and signs, times a power of two: exact from byte 0 (subnormal weights) to 252; from 2^128 on weights are infinite; 255 is NaN."""
    col = torch.arange(N, device=DEV) % 16
    q = torch.zeros(N, K // 2, dtype=torch.uint8, device=DEV)
    q[:, 40] = (col << 4).to(torch.uint8)                # channel 81
    level = O.e2m1_value(np.arange(N) % 16)
    for byte in (0, 1, 2, 6, 7, 8, 126, 251, 252, 253, 254, 255):
        s = torch.full((N, K // 32), byte, dtype=torch.uint8, device=DEV)
        up = 2.0 ** (100 if byte < 127 else -100)
        w = level * 2.0 ** (byte - 127)
        want = np.where(np.abs(w) >= 2.0 ** 128, np.copysign(np.inf, w), w * up) if byte < 255 else np.full(N, np.nan)
        a = torch.zeros(M, K, dtype=torch.bfloat16, device=DEV)
        a[:, 81] = up
        a8, row_scales = torch.zeros(M, K, dtype=torch.uint8, device=DEV), torch.full((M,), up, device=DEV)
        a8[:, 81] = 0x38                                 # 1
        c = torch.empty(M, N, device=DEV)
        lvx.lvx_linear_fp4(a, q, s, c, lvx.EPI_STORE_F32)
        assert np.array_equal(S.to_f64(c), np.broadcast_to(want, (M, N)), equal_nan=True), byte
        lvx.lvx_linear_fp8_fp4(a8, row_scales, q, s, c, lvx.EPI_STORE_F32)
        assert np.array_equal(S.to_f64(c), np.broadcast_to(want, (M, N)), equal_nan=True), byte
        for epi in (lvx.EPI_STORE, lvx.EPI_STORE | lvx.EPI_MIXED_8X4):
            out = torch.empty(M, N, dtype=torch.bfloat16, device=DEV)
            lvx.lvx_linear_fp8_fp4(a8, row_scales, q, s, out, epi)
            if not (epi & lvx.EPI_MIXED_8X4 and byte in (253, 254)):
                assert np.array_equal(S.to_f64(out), np.broadcast_to(want, (M, N)), equal_nan=True), (byte, epi)
