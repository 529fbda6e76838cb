// The residual's addition and the root-mean-square norm of the sum, in one pass over the token:
//
//   h = x + r,   y_c = h_c / sqrt(mean_c(h^2) + eps) * g_c,   8-bit rows: code = E4M3(y * (448 / max|y|)), scale = max|y| / 448.
//
// Bound by HBM: x, r in, h, y out, each once.  A token's channels stay in the registers of one, four or sixteen waves (template T), because the
// norm and, for 8 bits, the row's largest magnitude need the whole row before the first output.  The norm sees h before it is rounded to the
// residual's type; sums and scales are fp32.  4680 tokens x 5120 with an fp32 residual to 8-bit rows: 55 us, 4.8 TB/s; one token 3.4 us, the launch and three trips to memory.
#include "lvx_internal.h"

namespace {

constexpr float E4M3_MAX = 448.0f;
constexpr int MAX_TOKENS = 1 << 22;  // a launch holds fewer than 2^32 threads, and a long row takes 1024

struct norm_args_t {
    const bf16_t *x;     // may be NULL
    const void *r;       // bf16 or fp32, may be NULL
    const float *gain;   // may be NULL
    void *sum;           // type of r, may be NULL
    void *y;             // bf16, or E4M3 codes
    float *row_scales;   // with codes
    int64_t ldx, ldr, ld_sum, ldy;
    float eps, inv_d;
    int n_tokens, chunks;  // chunks of eight channels
};

template <int T>
__device__ __forceinline__ float row_sum(float v, float *lds) {
#pragma unroll
    for (int s = 32; s >= 1; s >>= 1) v += __shfl_xor(v, s);
    if (T == 64) return v;
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < T / 64; ++w) v += lds[w];
    return v;
}

template <int T>
__device__ __forceinline__ uint32_t row_max(uint32_t v, uint32_t *lds) {
#pragma unroll
    for (int s = 32; s >= 1; s >>= 1) {
        const uint32_t o = (uint32_t)__shfl_xor((int)v, s);
        v = v > o ? v : o;
    }
    if (T == 64) return v;
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < T / 64; ++w) v = v > lds[w] ? v : lds[w];
    return v;
}

// T threads per token, up to NI chunks of eight channels each; F32: the residual and the sum are fp32; FP8: 8-bit rows.
template <int T, int NI, bool F32, bool FP8>
__global__ void __launch_bounds__(T < 256 ? 256 : T) lvx_rmsnorm_residual_kernel(norm_args_t p) {
    constexpr int ROWS = T < 256 ? 256 / T : 1;
    __shared__ float lds_sum[16];
    __shared__ uint32_t lds_max[16];
    const int t = threadIdx.x % T;
    const int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / T;
    if (row >= p.n_tokens) return;  // whole waves, and no barrier where ROWS > 1

    float h[NI][8];
    float ss = 0;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        const int c = t + T * i;
#pragma unroll
        for (int e = 0; e < 8; ++e) h[i][e] = 0;
        if (c >= p.chunks) continue;
        if (p.x != nullptr) {
            const uint4 v = reinterpret_cast<const uint4 *>(p.x + row * p.ldx)[c];
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) h[i][2 * e] = bf16_lo(w[e]), h[i][2 * e + 1] = bf16_hi(w[e]);
        }
        if (p.r != nullptr) {
            if (F32) {
                const float4 *src = reinterpret_cast<const float4 *>((const float *)p.r + row * p.ldr) + 2 * c;
                const float4 a = src[0], b = src[1];
                h[i][0] += a.x, h[i][1] += a.y, h[i][2] += a.z, h[i][3] += a.w, h[i][4] += b.x, h[i][5] += b.y, h[i][6] += b.z, h[i][7] += b.w;
            } else {
                const uint4 v = reinterpret_cast<const uint4 *>((const bf16_t *)p.r + row * p.ldr)[c];
                const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) h[i][2 * e] += bf16_lo(w[e]), h[i][2 * e + 1] += bf16_hi(w[e]);
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) ss += h[i][e] * h[i][e];
        if (p.sum != nullptr) {
            if (F32) {
                float4 *dst = reinterpret_cast<float4 *>((float *)p.sum + row * p.ld_sum) + 2 * c;
                dst[0] = make_float4(h[i][0], h[i][1], h[i][2], h[i][3]);
                dst[1] = make_float4(h[i][4], h[i][5], h[i][6], h[i][7]);
            } else {
                reinterpret_cast<uint4 *>((bf16_t *)p.sum + row * p.ld_sum)[c] =
                    make_uint4(pack_bf16x2(h[i][0], h[i][1]), pack_bf16x2(h[i][2], h[i][3]), pack_bf16x2(h[i][4], h[i][5]), pack_bf16x2(h[i][6], h[i][7]));
            }
        }
    }
    const float rstd = 1.0f / sqrtf(row_sum<T>(ss, lds_sum) * p.inv_d + p.eps);

    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        const int c = t + T * i;
        if (c >= p.chunks) continue;
        float g[8] = {1, 1, 1, 1, 1, 1, 1, 1};
        if (p.gain != nullptr) {
            const float4 *src = reinterpret_cast<const float4 *>(p.gain) + 2 * c;
            const float4 a = src[0], b = src[1];
            g[0] = a.x, g[1] = a.y, g[2] = a.z, g[3] = a.w, g[4] = b.x, g[5] = b.y, g[6] = b.z, g[7] = b.w;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            h[i][e] = h[i][e] * rstd * g[e];
            const uint32_t m = __float_as_uint(h[i][e]) & 0x7fffffffu;  // a NaN is above every number and stays the maximum
            most = most > m ? most : m;
        }
        if (!FP8)
            reinterpret_cast<uint4 *>((bf16_t *)p.y + row * p.ldy)[c] =
                make_uint4(pack_bf16x2(h[i][0], h[i][1]), pack_bf16x2(h[i][2], h[i][3]), pack_bf16x2(h[i][4], h[i][5]), pack_bf16x2(h[i][6], h[i][7]));
    }
    if (!FP8) return;

    const float amax = __uint_as_float(row_max<T>(most, lds_max));
    // a scale below the normal numbers would lose bits, and its inverse be infinite
    const bool tiny = amax < E4M3_MAX * 0x1p-126f;
    const float inv = amax == 0.f ? 0.f : tiny ? 0x1p126f : E4M3_MAX / amax;
    if (t == 0) p.row_scales[row] = amax == 0.f ? 1.0f : tiny ? 0x1p-126f : amax / E4M3_MAX;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        const int c = t + T * i;
        if (c >= p.chunks) continue;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            // |y * inv| <= 448 (1 + 2^-23); the comparisons leave a NaN as it is, and its code is the format's NaN
            v[e] = h[i][e] * inv;
            v[e] = v[e] > E4M3_MAX ? E4M3_MAX : v[e];
            v[e] = v[e] < -E4M3_MAX ? -E4M3_MAX : v[e];
        }
        int lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
        lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], lo, true);
        int hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[4], v[5], 0, false);
        hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[6], v[7], hi, true);
        reinterpret_cast<uint2 *>((uint8_t *)p.y + row * p.ldy)[c] = make_uint2((uint32_t)lo, (uint32_t)hi);
    }
}

template <bool F32, bool FP8>
void launch(const norm_args_t &p, hipStream_t stream) {
    // a wave a token spares the barriers where tokens fill the chip; few tokens are spread over more waves (777 x 1280 to 8 bits: 5.7 us on one wave each, 4.4 on four)
    if (p.chunks <= 64 * 4 && p.n_tokens >= 2048)
        hipLaunchKernelGGL((lvx_rmsnorm_residual_kernel<64, 4, F32, FP8>), dim3((p.n_tokens + 3) / 4), dim3(256), 0, stream, p);
    else if (p.chunks <= 256 * 4)
        hipLaunchKernelGGL((lvx_rmsnorm_residual_kernel<256, 4, F32, FP8>), dim3(p.n_tokens), dim3(256), 0, stream, p);
    else
        hipLaunchKernelGGL((lvx_rmsnorm_residual_kernel<1024, 2, F32, FP8>), dim3(p.n_tokens), dim3(1024), 0, stream, p);
}

lvx_status_t entry(const void *x, int64_t ldx, const void *r, int64_t ldr, int32_t f32, const float *gain, float eps, int32_t n, int32_t d,
                   void *sum, int64_t ld_sum, void *y, int64_t ldy, bool fp8, float *row_scales, hipStream_t stream) {
    LVX_REQUIRE(x != nullptr || r != nullptr, LVX_ERR_INVALID_ARG, "x and the residual are both NULL");
    LVX_REQUIRE(r != nullptr || sum == nullptr, LVX_ERR_INVALID_ARG, "a sum is asked for without a residual");
    LVX_REQUIRE(y != nullptr && (!fp8 || row_scales != nullptr), LVX_ERR_INVALID_ARG, "an output pointer is NULL");
    LVX_REQUIRE(lvx_aligned16(x) && lvx_aligned16(r) && lvx_aligned16(gain) && lvx_aligned16(sum) && lvx_aligned16(y) && (((uintptr_t)row_scales) & 3u) == 0,
                LVX_ERR_INVALID_ARG, "pointers must be 16-byte aligned (the row scales 4-byte)");
    LVX_REQUIRE(f32 == 0 || f32 == 1, LVX_ERR_INVALID_ARG, "resid_is_f32 must be 0 or 1");
    LVX_REQUIRE(eps >= 0.f, LVX_ERR_INVALID_ARG, "eps must not be negative");
    const int step = fp8 ? 16 : 8;
    LVX_REQUIRE(d > 0 && d % step == 0 && d <= 16384, LVX_ERR_SHAPE, "d %d must be a positive multiple of %d, at most 16384", d, step);
    LVX_REQUIRE(n >= 0 && n < MAX_TOKENS, LVX_ERR_SHAPE, "n_tokens %d is negative or not below %d", n, MAX_TOKENS);
    LVX_REQUIRE((x == nullptr || (ldx >= d && ldx % 8 == 0)) && (r == nullptr || (ldr >= d && ldr % 8 == 0)) &&
                    (sum == nullptr || (ld_sum >= d && ld_sum % 8 == 0)) && ldy >= d && ldy % step == 0,
                LVX_ERR_SHAPE, "row strides must be >= d and multiples of 8 (16 for the 8-bit rows)");
    if (n == 0) return LVX_OK;
    norm_args_t p = {};
    p.x = (const bf16_t *)x, p.r = r, p.gain = gain, p.sum = sum, p.y = y, p.row_scales = row_scales;
    p.ldx = ldx, p.ldr = ldr, p.ld_sum = ld_sum, p.ldy = ldy;
    p.eps = eps, p.inv_d = 1.0f / (float)d;
    p.n_tokens = n, p.chunks = d / 8;
    if (f32)
        fp8 ? launch<true, true>(p, stream) : launch<true, false>(p, stream);
    else
        fp8 ? launch<false, true>(p, stream) : launch<false, false>(p, stream);
    LVX_CHECK_HIP(hipGetLastError());
    return LVX_OK;
}

}  // namespace

extern "C" lvx_status_t lvx_rmsnorm_residual(const void *dev_x, int64_t ldx, const void *dev_resid, int64_t ldr, int32_t resid_is_f32,
                                             const float *dev_gain, float eps, int32_t n_tokens, int32_t d, void *dev_sum, int64_t ld_sum,
                                             void *dev_y, int64_t ldy, lvx_stream_t stream) {
    return entry(dev_x, ldx, dev_resid, ldr, resid_is_f32, dev_gain, eps, n_tokens, d, dev_sum, ld_sum, dev_y, ldy, false, nullptr, (hipStream_t)stream);
}

extern "C" lvx_status_t lvx_rmsnorm_residual_fp8(const void *dev_x, int64_t ldx, const void *dev_resid, int64_t ldr, int32_t resid_is_f32,
                                                 const float *dev_gain, float eps, int32_t n_tokens, int32_t d, void *dev_sum, int64_t ld_sum,
                                                 void *dev_q, int64_t ldq, float *dev_row_scales, lvx_stream_t stream) {
    return entry(dev_x, ldx, dev_resid, ldr, resid_is_f32, dev_gain, eps, n_tokens, d, dev_sum, ld_sum, dev_q, ldq, true, dev_row_scales,
                 (hipStream_t)stream);
}
