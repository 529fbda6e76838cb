// Linears with 4-bit weights: C[m][n] = epilogue(sum_k A[m][k] W[n][k]) with W = E2M1 code * 2^e, one E8M0 exponent per 32 input channels.
//
// Weights and scales are read as they lie ([N][K/2] bytes, [N][K/32] bytes): a matrix instruction sums 128 channels of 16 weight rows, and lane
// (row r = lane % 16, group g = lane / 16) takes the 16 bytes of channels 32 g .. 32 g + 31 of row r: one scale group, one scale byte, one 16-byte load.
#include "lvx_fp4.h"

namespace {

struct fp4_args_t {
    const char *A;  // bf16, or E4M3 codes
    const float *row_scales;
    const uint8_t *W, *S;
    void *C;
    const void *R;
    const float *gate;
    int64_t lda, ldw, lds, ldc, ldr;  // lda in bytes
    int M, N, K, epi;
};

// 16 E4M3 codes, exact in bf16
__device__ __forceinline__ bf16x8_t fp8x8_bf16(uint32_t lo, uint32_t hi) {
    bf16x8_t r;
    const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
    const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
    r[0] = a[0], r[1] = a[1], r[2] = b[0], r[3] = b[1], r[4] = c[0], r[5] = c[1], r[6] = d[0], r[7] = d[1];
    return r;
}

// four consecutive columns n .. n + 3 of row m
__device__ __forceinline__ void fp4_store(const fp4_args_t &p, int m, int n, f32x4_t c) {
    float v[4] = {c[0], c[1], c[2], c[3]};
    if (p.row_scales != nullptr) {
        const float s = p.row_scales[m];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] *= s;
    }
    if (p.epi == LVX_EPI_GELU_TANH) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = gelu_tanh_f32(v[i]);
    } else if (p.epi == LVX_EPI_RESID_GATE || p.epi == LVX_EPI_RESID_GATE_F32) {
        if (p.gate != nullptr) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] *= p.gate[n + i];
        }
        if (p.epi == LVX_EPI_RESID_GATE) {
            const uint2 r = *reinterpret_cast<const uint2 *>((const bf16_t *)p.R + m * p.ldr + n);
            v[0] += bf16_lo(r.x), v[1] += bf16_hi(r.x), v[2] += bf16_lo(r.y), v[3] += bf16_hi(r.y);
        } else {
            const float4 r = *reinterpret_cast<const float4 *>((const float *)p.R + m * p.ldr + n);
            v[0] += r.x, v[1] += r.y, v[2] += r.z, v[3] += r.w;
        }
    }
    if (p.epi == LVX_EPI_RESID_GATE_F32 || p.epi == LVX_EPI_STORE_F32)
        *reinterpret_cast<float4 *>((float *)p.C + m * p.ldc + n) = make_float4(v[0], v[1], v[2], v[3]);
    else
        *reinterpret_cast<uint2 *>((bf16_t *)p.C + m * p.ldc + n) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
}

// A workgroup of KW waves owns 16 NB columns and 16 MB rows of C; its waves take every KW-th step of 128 channels.
template <int MB, int NB, int KW, bool A8>
__global__ void __launch_bounds__(64 * KW) lvx_fp4_linear_kernel(fp4_args_t p) {
    __shared__ f32x4_t part[KW][NB * MB][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int r = lane & 15, g = lane >> 4;
    const int n0 = blockIdx.x * 16 * NB, m0 = blockIdx.y * 16 * MB;
    const uint8_t *w_row[NB], *s_row[NB];
    const char *a_row[MB];
    // rows and columns past the end repeat the last one: they are read, multiplied and not stored
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const int n = n0 + 16 * b + r < p.N ? n0 + 16 * b + r : p.N - 1;
        w_row[b] = p.W + n * p.ldw + 16 * g;
        s_row[b] = p.S + n * p.lds + g;
    }
#pragma unroll
    for (int b = 0; b < MB; ++b) {
        const int m = m0 + 16 * b + r < p.M ? m0 + 16 * b + r : p.M - 1;
        a_row[b] = p.A + m * p.lda + (A8 ? 32 : 64) * g;
    }
    f32x4_t acc[NB][MB];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int c = 0; c < MB; ++c) acc[b][c] = {0, 0, 0, 0};

    const int steps = (p.K + 127) / 128;
    for (int t = wave; t < steps; t += KW) {
        const bool in = 128 * t + 32 * g < p.K;  // the last step may hold one to three groups of 32 channels
        uint4 w[NB];
        float s[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            w[b] = in ? *reinterpret_cast<const uint4 *>(w_row[b] + (size_t)64 * t) : make_uint4(0, 0, 0, 0);
            s[b] = in ? lvx_e8m0_f32(s_row[b][(size_t)4 * t]) : 1.0f;
        }
        bf16x8_t a[MB][4];
#pragma unroll
        for (int c = 0; c < MB; ++c) {
            if (A8) {
                uint4 v[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
                if (in) {
                    v[0] = reinterpret_cast<const uint4 *>(a_row[c] + (size_t)128 * t)[0];
                    v[1] = reinterpret_cast<const uint4 *>(a_row[c] + (size_t)128 * t)[1];
                }
                a[c][0] = fp8x8_bf16(v[0].x, v[0].y), a[c][1] = fp8x8_bf16(v[0].z, v[0].w);
                a[c][2] = fp8x8_bf16(v[1].x, v[1].y), a[c][3] = fp8x8_bf16(v[1].z, v[1].w);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint4 v = make_uint4(0, 0, 0, 0);
                    if (in) v = reinterpret_cast<const uint4 *>(a_row[c] + (size_t)256 * t)[j];
                    a[c][j] = *reinterpret_cast<bf16x8_t *>(&v);
                }
            }
        }
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const uint32_t words[4] = {w[b].x, w[b].y, w[b].z, w[b].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bf16x8_t wj = lvx_fp4x8_bf16(words[j], s[b]);
#pragma unroll
                for (int c = 0; c < MB; ++c) acc[b][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wj, a[c][j], acc[b][c], 0, 0, 0);
            }
        }
    }

    if (KW > 1) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int c = 0; c < MB; ++c) part[wave][b * MB + c][lane] = acc[b][c];
        __syncthreads();
    }
    // the blocks are shared out over the waves; the partial sums are added in the order of the waves
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int c = 0; c < MB; ++c) {
            if (KW > 1 && (b * MB + c) % KW != wave) continue;
            f32x4_t v = acc[b][c];
            if (KW > 1) {
                v = part[0][b * MB + c][lane];
#pragma unroll
                for (int k = 1; k < KW; ++k) v += part[k][b * MB + c][lane];
            }
            const int m = m0 + 16 * c + r, n = n0 + 16 * b + 4 * g;
            if (m < p.M && n < p.N) fp4_store(p, m, n, v);
        }
}

// 32 channels of a row per thread
__global__ void __launch_bounds__(256) lvx_fp4_quant_kernel(const bf16_t *x, int64_t ld, int rows, int groups, uint8_t *q, int64_t ldq, uint8_t *s,
                                                            int64_t lds) {
    const size_t total = (size_t)rows * groups;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (size_t)gridDim.x * 256) {
        const size_t r = i / groups, c = i % groups;
        uint4 v[4];
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[j] = reinterpret_cast<const uint4 *>(x + r * ld + 32 * c)[j];
            m = lvx_amax_bf16x2(lvx_amax_bf16x2(lvx_amax_bf16x2(lvx_amax_bf16x2(m, v[j].x), v[j].y), v[j].z), v[j].w);
        }
        const uint32_t byte = lvx_fp4_group_byte(m);
        const float scale = lvx_e8m0_f32(byte);
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = byte == 255 ? 0 : lvx_bf16x8_fp4(v[j].x, v[j].y, v[j].z, v[j].w, scale);
        *reinterpret_cast<uint4 *>(q + r * ldq + 16 * c) = make_uint4(w[0], w[1], w[2], w[3]);
        s[r * lds + c] = (uint8_t)byte;
    }
}

template <int MB, int NB, int KW>
void launch(const fp4_args_t &p, hipStream_t stream) {
    const dim3 grid((p.N + 16 * NB - 1) / (16 * NB), (p.M + 16 * MB - 1) / (16 * MB));
    if (p.row_scales != nullptr)
        hipLaunchKernelGGL((lvx_fp4_linear_kernel<MB, NB, KW, true>), grid, dim3(64 * KW), 0, stream, p);
    else
        hipLaunchKernelGGL((lvx_fp4_linear_kernel<MB, NB, KW, false>), grid, dim3(64 * KW), 0, stream, p);
}

lvx_status_t linear(const void *a, int64_t lda, const float *row_scales, bool a8, const void *w, int64_t ldw, const void *s, int64_t lds, void *c,
                    int64_t ldc, int32_t M, int32_t N, int32_t K, lvx_epilogue_t epi, const void *resid, int64_t ldr, const float *gate,
                    hipStream_t stream) {
    LVX_REQUIRE(a != nullptr && w != nullptr && s != nullptr && c != nullptr && (!a8 || row_scales != nullptr), LVX_ERR_INVALID_ARG,
                "A, W, C or a scale pointer is NULL");
    LVX_REQUIRE(lvx_aligned16(a) && lvx_aligned16(w) && lvx_aligned16(c) && lvx_aligned16(resid) && (((uintptr_t)row_scales | (uintptr_t)gate) & 3u) == 0,
                LVX_ERR_INVALID_ARG, "pointers must be 16-byte aligned (scales and gate as their type)");
    LVX_REQUIRE(M >= 0 && N > 0 && K > 0, LVX_ERR_SHAPE, "M %d, N %d, K %d", M, N, K);
    LVX_REQUIRE(K % LVX_FP4_GROUP == 0, LVX_ERR_SHAPE, "K %d must be a multiple of %d", K, LVX_FP4_GROUP);
    LVX_REQUIRE(N % 8 == 0, LVX_ERR_SHAPE, "N %d must be a multiple of 8", N);
    LVX_REQUIRE(lda >= K && lda % (a8 ? 16 : 8) == 0 && ldw >= K / 2 && ldw % 16 == 0 && lds >= K / LVX_FP4_GROUP && ldc >= N && ldc % 8 == 0,
                LVX_ERR_SHAPE, "bad leading dimension");
    LVX_REQUIRE(M <= 65535 * 16, LVX_ERR_SHAPE, "M %d is more than %d rows", M, 65535 * 16);
    LVX_REQUIRE(epi == LVX_EPI_STORE || epi == LVX_EPI_GELU_TANH || epi == LVX_EPI_RESID_GATE || epi == LVX_EPI_RESID_GATE_F32 || epi == LVX_EPI_STORE_F32,
                LVX_ERR_INVALID_ARG, "unknown epilogue %d", (int)epi);
    if (epi == LVX_EPI_RESID_GATE || epi == LVX_EPI_RESID_GATE_F32) {
        LVX_REQUIRE(resid != nullptr, LVX_ERR_INVALID_ARG, "residual epilogue needs a residual pointer");
        LVX_REQUIRE(ldr >= N && ldr % 8 == 0, LVX_ERR_SHAPE, "bad residual leading dimension");
    }
    if (M == 0) return LVX_OK;
    fp4_args_t p = {};
    p.A = (const char *)a, p.lda = a8 ? lda : 2 * lda;
    p.row_scales = row_scales;
    p.W = (const uint8_t *)w, p.ldw = ldw;
    p.S = (const uint8_t *)s, p.lds = lds;
    p.C = c, p.ldc = ldc;
    p.R = resid, p.ldr = ldr;
    p.gate = gate;
    p.M = M, p.N = N, p.K = K, p.epi = (int)epi;
    if (M <= 16)
        launch<1, 1, 8>(p, stream);
    else if (M <= 32)
        launch<2, 1, 8>(p, stream);
    else
        launch<4, 4, 1>(p, stream);
    LVX_CHECK_HIP(hipGetLastError());
    return LVX_OK;
}

}  // namespace

extern "C" lvx_status_t lvx_fp4_quantize(const void *dev_x, int64_t ld, int32_t rows, int32_t cols, void *dev_q, int64_t ldq, void *dev_scales,
                                         int64_t lds, lvx_stream_t stream) {
    LVX_REQUIRE(dev_x != nullptr && dev_q != nullptr && dev_scales != nullptr, LVX_ERR_INVALID_ARG, "x, q or scales is NULL");
    LVX_REQUIRE(lvx_aligned16(dev_x) && lvx_aligned16(dev_q), LVX_ERR_INVALID_ARG, "x and q must be 16-byte aligned");
    LVX_REQUIRE(rows >= 0 && cols > 0 && cols % LVX_FP4_GROUP == 0, LVX_ERR_SHAPE, "rows %d, cols %d (cols must be a positive multiple of %d)", rows, cols,
                LVX_FP4_GROUP);
    LVX_REQUIRE(ld >= cols && ld % 8 == 0 && ldq >= cols / 2 && ldq % 16 == 0 && lds >= cols / LVX_FP4_GROUP, LVX_ERR_SHAPE,
                "row strides: ld a multiple of 8 and >= cols, ldq a multiple of 16 and >= cols / 2, lds >= cols / %d", LVX_FP4_GROUP);
    if (rows == 0) return LVX_OK;
    const size_t groups = (size_t)rows * (cols / LVX_FP4_GROUP);
    const unsigned grid = (unsigned)(groups < 256 * 4096 ? (groups + 255) / 256 : 4096);
    hipLaunchKernelGGL(lvx_fp4_quant_kernel, dim3(grid), dim3(256), 0, (hipStream_t)stream, (const bf16_t *)dev_x, ld, rows, cols / LVX_FP4_GROUP,
                       (uint8_t *)dev_q, ldq, (uint8_t *)dev_scales, lds);
    LVX_CHECK_HIP(hipGetLastError());
    return LVX_OK;
}

extern "C" lvx_status_t lvx_linear_fp4(const void *dev_a, int64_t lda, const void *dev_wq, int64_t ldw, const void *dev_w_scales, int64_t lds, void *dev_c,
                                       int64_t ldc, int32_t M, int32_t N, int32_t K, lvx_epilogue_t epi, const void *dev_resid, int64_t ldr,
                                       const float *dev_gate, lvx_stream_t stream) {
    return linear(dev_a, lda, nullptr, false, dev_wq, ldw, dev_w_scales, lds, dev_c, ldc, M, N, K, epi, dev_resid, ldr, dev_gate, (hipStream_t)stream);
}

extern "C" lvx_status_t lvx_linear_fp8_fp4(const void *dev_aq, int64_t lda, const float *dev_row_scales, const void *dev_wq, int64_t ldw,
                                           const void *dev_w_scales, int64_t lds, void *dev_c, int64_t ldc, int32_t M, int32_t N, int32_t K,
                                           lvx_epilogue_t epi, const void *dev_resid, int64_t ldr, const float *dev_gate, lvx_stream_t stream) {
    return linear(dev_aq, lda, dev_row_scales, true, dev_wq, ldw, dev_w_scales, lds, dev_c, ldc, M, N, K, epi, dev_resid, ldr, dev_gate,
                  (hipStream_t)stream);
}
