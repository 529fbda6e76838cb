"""The norm with the residual's addition against the 64-bit oracle: both residual types, bf16 and 8-bit rows, every way the channels are spread over waves.

Tolerances: sums, squares and products in fp32 put y off by at most (d / 2 + 8) * 2^-24 of itself (d additions of the squares, halved by the root, and a few
roundings); a bf16 output by half a step more (2^-8 of itself); an 8-bit value by 2^-4 of itself or, below the smallest normal code, by 2^-10 of a unit."""
import numpy as np
import pytest
import torch

import lvx_synth as S
from oracle import decoder_oracle as O
from test_gpu_fp8 import e4m3_decode

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

SIZES = [(1, 16), (1, 5120), (3, 8192), (5, 16384), (7, 2048), (4, 2064), (130, 48), (2, 8208), (33, 1280), (1029, 64)]


def inputs(n, d, f32, pad=16):
    x = S.randn_bf16((n, d + pad), S.seed_of("rn_x", n, d), device=DEV)[:, :d]
    r = S.randn_f32((n, d + 2 * pad), S.seed_of("rn_r", n, d), 3.0, device=DEV)[:, :d]
    g = S.randn_f32((d,), S.seed_of("rn_g", d), 1.0, device=DEV)
    return x, r if f32 else r.to(torch.bfloat16), g


def rel32(d):
    return (d / 2 + 8) * 2.0 ** -24


def check_y(y, ref, d):
    got = S.to_f64(y)
    assert np.all(np.abs(got - ref) <= (2.0 ** -8 + 2 * rel32(d)) * np.abs(ref))


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("n,d", SIZES)
def test_norm(lvx, n, d, f32):
    x, r, g = inputs(n, d, f32)
    total = torch.full((n + 1, d + 8), 7.0, dtype=r.dtype, device=DEV)
    y = torch.full((n + 1, d + 24), 7.0, dtype=torch.bfloat16, device=DEV)
    lvx.lvx_rmsnorm_residual(x, r, g, 1e-6, y[:n, :d], sum_out=total[:n, :d])
    h, ref = O.rmsnorm_residual(S.to_f64(x), S.to_f64(r), S.to_f64(g), 1e-6)
    check_y(y[:n, :d], ref, d)
    got = S.to_f64(total[:n, :d])
    assert np.array_equal(got, h.astype(np.float32)) if f32 else np.array_equal(got, O.bf16(h))
    assert bool((total[n:] == 7).all()) and bool((total[:, d:] == 7).all()) and bool((y[n:] == 7).all()) and bool((y[:, d:] == 7).all())
    # 8-bit rows of the same numbers
    q = torch.full((n + 1, d + 32), 77, dtype=torch.uint8, device=DEV)
    sc = torch.full((n + 1,), 7.0, device=DEV)
    lvx.lvx_rmsnorm_residual_fp8(x, r, g, 1e-6, q[:n, :d], sc[:n], sum_out=total[:n, :d])
    most = np.abs(ref).max(1)
    assert np.all(np.abs(S.to_f64(sc[:n]) - most / 448) <= (2 * rel32(d) + 2.0 ** -22) * most / 448)
    s = S.to_f64(sc[:n])[:, None]
    val = e4m3_decode(q[:n, :d].cpu().numpy()) * s
    assert np.all(np.abs(val - ref) <= (2.0 ** -4 + 4 * rel32(d) + 2.0 ** -20) * np.abs(ref) + 2.0 ** -10 * s)
    assert bool((q[n:] == 77).all()) and bool((q[:, d:] == 77).all()) and float(sc[n]) == 7.0


@pytest.mark.parametrize("n,d", [(3, 1024), (2, 5120), (2, 16384)])
def test_norm_optional_arguments(lvx, n, d):
    x, r, g = inputs(n, d, False)
    y = torch.empty(n, d, dtype=torch.bfloat16, device=DEV)
    lvx.lvx_rmsnorm_residual(x, None, None, 1e-5, y)
    check_y(y, O.rmsnorm_residual(S.to_f64(x), None, None, 1e-5)[1], d)
    lvx.lvx_rmsnorm_residual(None, r, g, 1e-5, y)
    check_y(y, O.rmsnorm_residual(None, S.to_f64(r), S.to_f64(g), 1e-5)[1], d)
    r32 = r.float()
    lvx.lvx_rmsnorm_residual(None, r32, g, 1e-5, y)
    check_y(y, O.rmsnorm_residual(None, S.to_f64(r), S.to_f64(g), 1e-5)[1], d)
    # in place: the sum over the residual, the norm over x
    want_sum, want_y = torch.empty(n, d, dtype=torch.bfloat16, device=DEV), torch.empty(n, d, dtype=torch.bfloat16, device=DEV)
    lvx.lvx_rmsnorm_residual(x, r, g, 1e-5, want_y, sum_out=want_sum)
    x2, r2 = x.clone(), r.clone()
    lvx.lvx_rmsnorm_residual(x2, r2, g, 1e-5, x2, sum_out=r2)
    assert torch.equal(r2, want_sum) and torch.equal(x2, want_y)


def test_norm_zero_and_non_finite_rows(lvx):
    n, d = 5, 256
    x, r, g = inputs(n, d, True)
    x, r = x.clone(), r.clone()
    x[1], r[1] = 0, 0
    x[2, 9] = float("nan")
    r[3, 200] = float("inf")
    q, sc = torch.empty(n, d, dtype=torch.uint8, device=DEV), torch.empty(n, device=DEV)
    lvx.lvx_rmsnorm_residual_fp8(x, r, g, 1e-6, q, sc)
    assert float(sc[1]) == 1.0 and not bool((q[1] & 127).any())
    assert torch.isnan(sc[2]) and torch.isnan(sc[3]) and bool(torch.isfinite(sc[[0, 1, 4]]).all())
    assert bool(((q[2] & 127) == 127).all()) and bool(((q[3] & 127) == 127).all())
    clean = torch.empty_like(q), torch.empty_like(sc)
    lvx.lvx_rmsnorm_residual_fp8(x[4:], r[4:], g, 1e-6, clean[0][4:], clean[1][4:])
    assert torch.equal(clean[0][4], q[4]) and torch.equal(clean[1][4], sc[4])     # a row's result is its own
    y = torch.empty(n, d, dtype=torch.bfloat16, device=DEV)
    lvx.lvx_rmsnorm_residual(x, r, g, 1e-6, y)
    assert bool(torch.isnan(y[2]).all()) and bool(torch.isnan(y[3, 200])) and not bool(y[1].any())


@pytest.mark.parametrize("d", [64, 2064, 16384])
def test_tiny_rows_to_8_bits(lvx, d):
    """Rows whose scale max|y| / 448 would be no normal number: it stays at 2^-126, and multiples of it up to 448 are exact (eps 1: y is h)."""
    r = torch.zeros(3, d, device=DEV)
    r[0, 3], r[0, 9], r[1, d - 1] = 2.0 ** -126, -3 * 2.0 ** -126, 416 * 2.0 ** -126
    q, sc = torch.full((3, d), 77, dtype=torch.uint8, device=DEV), torch.empty(3, device=DEV)
    lvx.lvx_rmsnorm_residual_fp8(None, r, None, 1.0, q, sc)
    assert np.array_equal(e4m3_decode(q.cpu().numpy()) * S.to_f64(sc)[:, None], S.to_f64(r))
    assert S.to_f64(sc).tolist() == [2.0 ** -126, 2.0 ** -126, 1.0]
