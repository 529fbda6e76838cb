// Linears with 4-bit weights: C[m][n] = epilogue(sum_k A[m][k] W[n][k]) with W = E2M1 code * 2^e, one E8M0 exponent per 32 input channels.
//
// Weights and scales are read as they lie ([N][K/2] bytes, [N][K/32] bytes): a matrix instruction sums 128 channels of 16 weight rows, and lane
// (row r = lane % 16, group g = lane / 16) takes the 16 bytes of channels 32 g .. 32 g + 31 of row r: one scale group, one scale byte, one 16-byte load.
//
// Weights stay exact: below 2^128 (scale bytes up to 252, whatever the code) a code times its scale is a bf16 number, a subnormal one for bytes below 2, which the conversion
// and the matrix cores keep, and its products with a bf16 or E4M3 value are exact in fp32.
#include "lvx_fp4.h"
#include "lvx_fp4_rules.h"

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

// Eight E4M3 codes, exact in bf16
__device__ __forceinline__ bf16x8_t fp8x8_bf16(uint32_t lo, uint32_t hi) {
    bf16x8_t r;
    const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
    const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
    r[0] = a[0], r[1] = a[1], r[2] = b[0], r[3] = b[1], r[4] = c[0], r[5] = c[1], r[6] = d[0], r[7] = d[1];
    return r;
}

// Blocks of 16 columns and MB blocks of 16 rows: a lane has columns n .. n + 3 of row m0 + 16 c + lane % 16.  Everything that is read is requested before the first
// store: the compiler moves no load past a store that may alias it, and each would be waited for in turn.
template <int MB>
__device__ __forceinline__ void fp4_store(const fp4_args_t &p, int m0, int n, const f32x4_t (&acc)[MB], const float (&row_scale)[MB]) {
    if (n >= p.N) return;
    float4 gate = make_float4(1.f, 1.f, 1.f, 1.f);
    float4 r32[MB];
    uint2 r16[MB];
    if (p.epi == LVX_EPI_RESID_GATE || p.epi == LVX_EPI_RESID_GATE_F32) {
        if (p.gate != nullptr) gate = make_float4(p.gate[n], p.gate[n + 1], p.gate[n + 2], p.gate[n + 3]);
#pragma unroll
        for (int c = 0; c < MB; ++c) {
            const int64_t m = m0 + 16 * c;
            if (m >= p.M) continue;
            if (p.epi == LVX_EPI_RESID_GATE)
                r16[c] = *reinterpret_cast<const uint2 *>((const bf16_t *)p.R + m * p.ldr + n);
            else
                r32[c] = *reinterpret_cast<const float4 *>((const float *)p.R + m * p.ldr + n);
        }
    }
#pragma unroll
    for (int c = 0; c < MB; ++c) {
        const int64_t m = m0 + 16 * c;
        if (m >= p.M) continue;
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = acc[c][i] * row_scale[c];
        if (p.epi == LVX_EPI_GELU_TANH) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = gelu_tanh_f32(v[i]);
        } else if (p.epi == LVX_EPI_RESID_GATE) {
            v[0] = v[0] * gate.x + bf16_lo(r16[c].x), v[1] = v[1] * gate.y + bf16_hi(r16[c].x);
            v[2] = v[2] * gate.z + bf16_lo(r16[c].y), v[3] = v[3] * gate.w + bf16_hi(r16[c].y);
        } else if (p.epi == LVX_EPI_RESID_GATE_F32) {
            v[0] = v[0] * gate.x + r32[c].x, v[1] = v[1] * gate.y + r32[c].y, v[2] = v[2] * gate.z + r32[c].z, v[3] = v[3] * gate.w + r32[c].w;
        }
        if (p.epi == LVX_EPI_RESID_GATE_F32 || p.epi == LVX_EPI_STORE_F32)
            *reinterpret_cast<float4 *>((float *)p.C + m * p.ldc + n) = make_float4(v[0], v[1], v[2], v[3]);
        else
            *reinterpret_cast<uint2 *>((bf16_t *)p.C + m * p.ldc + n) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
    }
}

// this lane's rows' scales (1 for bf16 rows)
template <int MODE, int MB>
__device__ __forceinline__ void fp4_row_scales(const fp4_args_t &p, int m0, float (&s)[MB]) {
#pragma unroll
    for (int c = 0; c < MB; ++c) {
        const int m = m0 + 16 * c;
        s[c] = MODE == 0 ? 1.0f : p.row_scales[m < p.M ? m : p.M - 1];
    }
}

enum { A_BF16 = LVX_FP4_A_BF16, A_WIDEN = LVX_FP4_A_WIDEN, A_NATIVE = LVX_FP4_A_NATIVE };

// Matrix products of a step of 128 channels: w[b] the codes of 16 columns, s[b] their scale as a byte (native) or as fp32 bits (widened codes), a[c] the operands of 16 rows.
template <int MODE, int MB, int NB>
__device__ __forceinline__ void fp4_multiply(f32x4_t (&acc)[NB][MB], const uint4 (&w)[NB], const uint32_t (&s)[NB], const uint4 (&a)[MB][MODE == A_BF16 ? 4 : 2]) {
    if (MODE == A_NATIVE) {
        i32x8_t av[MB];
#pragma unroll
        for (int c = 0; c < MB; ++c)
            av[c] = {(int)a[c][0].x, (int)a[c][0].y, (int)a[c][0].z, (int)a[c][0].w, (int)a[c][1].x, (int)a[c][1].y, (int)a[c][1].z, (int)a[c][1].w};
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const i32x8_t wv = {(int)w[b].x, (int)w[b].y, (int)w[b].z, (int)w[b].w, 0, 0, 0, 0};
#pragma unroll
            for (int c = 0; c < MB; ++c)  // formats: 4 = E2M1, 0 = E4M3; the rows' block scales are 2^0
                acc[b][c] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wv, av[c], acc[b][c], 4, 0, 0, (int)s[b], 0, 127);
        }
    } else {
        bf16x8_t x[MB][4];
#pragma unroll
        for (int c = 0; c < MB; ++c) {
            if (MODE == A_WIDEN) {
                x[c][0] = fp8x8_bf16(a[c][0].x, a[c][0].y), x[c][1] = fp8x8_bf16(a[c][0].z, a[c][0].w);
                x[c][2] = fp8x8_bf16(a[c][1].x, a[c][1].y), x[c][3] = fp8x8_bf16(a[c][1].z, a[c][1].w);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) x[c][j] = *reinterpret_cast<const bf16x8_t *>(&a[c][j % (MODE == A_BF16 ? 4 : 2)]);
            }
        }
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const uint32_t words[4] = {w[b].x, w[b].y, w[b].z, w[b].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bf16x8_t wj = lvx_fp4x8_bf16(words[j], __uint_as_float(s[b]));
#pragma unroll
                for (int c = 0; c < MB; ++c) acc[b][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wj, x[c][j], acc[b][c], 0, 0, 0);
            }
        }
    }
}

__device__ __forceinline__ void swap32(uint32_t &a, uint32_t &b) {  // upper half of a <-> lower half of b
    const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
    a = r[0], b = r[1];
}
__device__ __forceinline__ void swap16(uint32_t &a, uint32_t &b) {  // odd rows of 16 lanes of a <-> even rows of b
    const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
    a = r[0], b = r[1];
}

constexpr int PANEL = 48;  // steps whose scales a tile holds in LDS

// ---- few rows: a wave per 16 NB columns and range of K -----------------------------------------------------------------
// Bound by the weights' way from memory (16 8-bit rows x 13824 x 5120: 13.5 us, 2.8 TB/s).  A workgroup of blockDim.x / 64 waves owns 16 NB columns and 16 MB rows; the waves take units of U steps of 128 channels in turn.
// Rows of A are loaded as runs of 64 bytes per row and instruction and exchanged between the lanes (piece 4 j + g of 16 bytes is loaded, 4 g + j is multiplied), scales
// as U words per column: what counts here is the number of cache lines that the loads touch, not their bytes.
template <int MODE, int MB, int NB, int U>
__global__ void __launch_bounds__(512) lvx_fp4_few_kernel(fp4_args_t p) {
    constexpr int AV = MODE == A_BF16 ? 4 : 2, STEP_A = MODE == A_BF16 ? 256 : 128;
    extern __shared__ f32x4_t part[];  // [waves - 1][NB * MB][64]
    const int lane = threadIdx.x & 63, kw = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const int r = lane & 15, g = lane >> 4;
    const int n0 = blockIdx.x * 16 * NB, m0 = blockIdx.y * 16 * MB;
    const uint8_t *w_row[NB], *s_row[NB];
    const char *a_row[MB];
    // columns past the end repeat the last one: they are read, multiplied and not stored
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const int n = n0 + 16 * b + r < p.N ? n0 + 16 * b + r : p.N - 1;
        w_row[b] = p.W + n * p.ldw + 16 * g;
        s_row[b] = p.S + n * p.lds;
    }
#pragma unroll
    for (int c = 0; c < MB; ++c) {
        const int m = m0 + 16 * c + r < p.M ? m0 + 16 * c + r : p.M - 1;
        a_row[c] = p.A + m * p.lda + 16 * g;
    }
    const bool row_in = MB > 1 || m0 + r < p.M;  // one block of rows: lanes of rows past the end load nothing
    f32x4_t acc[NB][MB];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int c = 0; c < MB; ++c) acc[b][c] = {0, 0, 0, 0};

    // the lanes' exchange: 4 x 4 pieces of a row over registers and lane groups are transposed; of eight pieces, a lane group gets 2 g and 2 g + 1
    auto exchange = [&](uint4 (&v)[AV]) {
        uint32_t *x[AV];
#pragma unroll
        for (int j = 0; j < AV; ++j) x[j] = reinterpret_cast<uint32_t *>(&v[j]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (MODE == A_BF16) {
                swap32(x[0][e], x[2 % AV][e]), swap32(x[1][e], x[3 % AV][e]);
                swap16(x[0][e], x[1][e]), swap16(x[2 % AV][e], x[3 % AV][e]);
            } else {
                swap32(x[0][e], x[1][e]);
                swap16(x[0][e], x[1][e]);
            }
        }
    };
    const int whole = p.K / 128, units = whole / U, steps = (p.K + 127) / 128;
    uint4 w[U][NB], a[U][MB][AV];
    for (int u = kw; u < units; u += waves) {
        uint32_t s[NB][U];
#pragma unroll
        for (int i = 0; i < U; ++i)
#pragma unroll
            for (int b = 0; b < NB; ++b) w[i][b] = *reinterpret_cast<const uint4 *>(w_row[b] + (size_t)64 * (u * U + i));
#pragma unroll
        for (int b = 0; b < NB; ++b) __builtin_memcpy(s[b], s_row[b] + (size_t)4 * U * u, 4 * U);
#pragma unroll
        for (int i = 0; i < U; ++i)
#pragma unroll
            for (int c = 0; c < MB; ++c)
#pragma unroll
                for (int j = 0; j < AV; ++j) {
                    a[i][c][j] = make_uint4(0, 0, 0, 0);
                    if (row_in) a[i][c][j] = *reinterpret_cast<const uint4 *>(a_row[c] + (size_t)STEP_A * (u * U + i) + 64 * j);
                }
#pragma unroll
        for (int i = 0; i < U; ++i) {
            uint32_t sc[NB];
#pragma unroll
            for (int b = 0; b < NB; ++b) sc[b] = ((s[b][i] >> (8 * g)) & 255u) << 23;
#pragma unroll
            for (int c = 0; c < MB; ++c) exchange(a[i][c]);
            fp4_multiply<MODE, MB, NB>(acc, w[i], sc, a[i]);
        }
    }
    // the steps behind the whole units, the last of them with one to three groups of 32 channels: the other lanes multiply zeros
    for (int t = units * U + kw; t < steps; t += waves) {
        const int left = p.K - 128 * t;
        uint32_t sc[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            w[0][b] = make_uint4(0, 0, 0, 0), sc[b] = 127u << 23;
            if (32 * g < left) {
                w[0][b] = *reinterpret_cast<const uint4 *>(w_row[b] + (size_t)64 * t);
                sc[b] = (uint32_t)s_row[b][(size_t)4 * t + g] << 23;
            }
        }
#pragma unroll
        for (int c = 0; c < MB; ++c) {
#pragma unroll
            for (int j = 0; j < AV; ++j) {
                a[0][c][j] = make_uint4(0, 0, 0, 0);
                if (row_in && (4 * j + g) * (MODE == A_BF16 ? 8 : 16) < left)
                    a[0][c][j] = *reinterpret_cast<const uint4 *>(a_row[c] + (size_t)STEP_A * t + 64 * j);
            }
            exchange(a[0][c]);
        }
        fp4_multiply<MODE, MB, NB>(acc, w[0], sc, a[0]);
    }

    float row_scale[MB];
    fp4_row_scales<MODE, MB>(p, m0 + r, row_scale);
    if (kw > 0) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int c = 0; c < MB; ++c) part[((kw - 1) * NB * MB + b * MB + c) * 64 + lane] = acc[b][c];
    }
    __syncthreads();
    if (kw > 0) return;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
#pragma unroll
        for (int c = 0; c < MB; ++c)
            for (int k = 1; k < waves; ++k) acc[b][c] += part[((k - 1) * NB * MB + b * MB + c) * 64 + lane];
        fp4_store<MB>(p, m0 + r, n0 + 16 * b + 4 * g, acc[b], row_scale);
    }
}

// ---- rows that fit the LDS ----------------------------------------------------------------------------------------------
// The same for up to sixteen rows that lie in LDS whole, with the columns' scales beside them: the loop then requests nothing but weights, two steps ahead of a wave's own.
// Bound by the weights' way once it runs, and by the rows' way before it: they come 16 bytes a thread at a time, each load waited for, and the first weights with it.
// One row x 15360 x 5120: 9.4 us, 4.4 TB/s.
template <int MODE, int NB>
__global__ void __launch_bounds__(512) lvx_fp4_resident_kernel(fp4_args_t p) {
    constexpr int AV = MODE == A_BF16 ? 4 : 2, STEP_A = MODE == A_BF16 ? 256 : 128;
    extern __shared__ char lds[];  // rows, scales; then the partial sums
    const int lane = threadIdx.x & 63, kw = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const int r = lane & 15, g = lane >> 4;
    const int n0 = blockIdx.x * 16 * NB;
    const int row_bytes = p.K * (MODE == A_BF16 ? 2 : 1), a_pitch = row_bytes + 16, s_bytes = p.K / LVX_FP4_GROUP, s_pitch = ((s_bytes + 15) & ~15) + 4;
    char *s_lds = lds + p.M * a_pitch;
    const uint8_t *w_row[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const int n = n0 + 16 * b + r < p.N ? n0 + 16 * b + r : p.N - 1;  // columns past the end repeat the last one: they are read, multiplied and not stored
        w_row[b] = p.W + n * p.ldw + 16 * g;
    }
    f32x4_t acc[NB][1];
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[b][0] = {0, 0, 0, 0};
    const int whole = p.K / 128;
    uint4 w[2][NB];
    auto load = [&](int t, uint4 (&d)[NB]) {
        if (t >= whole) return;
#pragma unroll
        for (int b = 0; b < NB; ++b) d[b] = *reinterpret_cast<const uint4 *>(w_row[b] + (size_t)64 * t);
    };
    load(kw, w[0]);
    for (int m = 0; m < p.M; ++m)
        for (int c = threadIdx.x; c < row_bytes / 16; c += blockDim.x)
            *reinterpret_cast<uint4 *>(lds + m * a_pitch + 16 * c) = *reinterpret_cast<const uint4 *>(p.A + m * p.lda + 16 * c);
    // scales: a thread takes 16 bytes of a column, a last piece byte by byte
    for (int i = threadIdx.x; i < 16 * NB * 16; i += blockDim.x) {
        const int row = i >> 4, n = n0 + row < p.N ? n0 + row : p.N - 1;
        const uint8_t *src = p.S + n * p.lds;
        for (int at = 16 * (i & 15); at < s_bytes; at += 256) {
            uint32_t e[4] = {0, 0, 0, 0};
            if (at + 16 <= s_bytes) {
                __builtin_memcpy(e, src + at, 16);
            } else {
#pragma unroll
                for (int x = 0; x < 15; ++x)
                    if (at + x < s_bytes) e[x >> 2] |= (uint32_t)src[at + x] << (8 * (x & 3));
            }
            uint32_t *dst = reinterpret_cast<uint32_t *>(s_lds + row * s_pitch + at);
#pragma unroll
            for (int x = 0; x < 4; ++x) dst[x] = e[x];
        }
    }
    __syncthreads();
    load(kw + waves, w[1]);
    const char *a_row = lds + (r < p.M ? r : p.M - 1) * a_pitch;
    const uint8_t *s_row = reinterpret_cast<const uint8_t *>(s_lds + r * s_pitch) + g;
    auto step = [&](int t, bool in, const uint4 (&wt)[NB]) {
        uint4 a[1][AV];
        uint32_t sc[NB];
#pragma unroll
        for (int j = 0; j < AV; ++j) {
            a[0][j] = make_uint4(0, 0, 0, 0);
            if (in) a[0][j] = *reinterpret_cast<const uint4 *>(a_row + STEP_A * t + (STEP_A / 4) * g + 16 * j);
        }
#pragma unroll
        for (int b = 0; b < NB; ++b) sc[b] = in ? (uint32_t)s_row[16 * b * s_pitch + 4 * t] << 23 : 127u << 23;
        fp4_multiply<MODE, 1, NB>(acc, wt, sc, a);
    };
    for (int t = kw; t < whole; t += 2 * waves) {
        step(t, true, w[0]);
        load(t + 2 * waves, w[0]);
        if (t + waves < whole) {
            step(t + waves, true, w[1]);
            load(t + 3 * waves, w[1]);
        }
    }
    // a last step of one to three groups of 32 channels: the other lanes multiply zeros
    if (p.K % 128 != 0 && kw == whole % waves) {
        const bool in = 128 * whole + 32 * g < p.K;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            w[0][b] = make_uint4(0, 0, 0, 0);
            if (in) w[0][b] = *reinterpret_cast<const uint4 *>(w_row[b] + (size_t)64 * whole);
        }
        step(whole, in, w[0]);
    }

    float row_scale[1];
    fp4_row_scales<MODE, 1>(p, r, row_scale);
    __syncthreads();
    f32x4_t *part = reinterpret_cast<f32x4_t *>(lds);  // [waves][NB][64]
#pragma unroll
    for (int b = 0; b < NB; ++b) part[(kw * NB + b) * 64 + lane] = acc[b][0];
    __syncthreads();
    // a wave finishes every waves-th block of columns, adding in the order of the waves
    for (int b = kw; b < NB; b += waves) {
        f32x4_t v[1] = {part[b * 64 + lane]};
        for (int k = 1; k < waves; ++k) v[0] += part[(k * NB + b) * 64 + lane];
        fp4_store<1>(p, r, n0 + 16 * b + 4 * g, v, row_scale);
    }
}

// ---- many rows: tiles of 32 MBW rows and 256 / KG columns -----------------------------------------------------------------
// Bound by the matrix cores and the LDS.  Eight waves: KG groups over K, every KG-th pair of steps each, of two waves over the rows and one or two over the columns.  Rows
// and weights come by direct loads to LDS, RING steps and a pair or two of steps ahead: a stage of the weights is a pair, because a weight row's 128 channels are half a
// cache line and halves cost as much as lines.  A wave reads the next step's operands into registers while it multiplies this one's.  16-byte chunk c of a row of CH
// chunks lies at c ^ (row % CH): the sixteen rows of an operand fall into different banks where a row has 256 bytes; of 128-byte rows those eight apart share theirs, and
// conflicts are more than half of the LDS's cycles.  544 8-bit rows x 5120 x 13824: 84 to 88 us, 0.9 PFLOP/s, the matrix cores busy for a third of it; with mixed products 51 to 53, 1.5.
template <int MODE, int MBW, int KG, int RING>
__global__ void __launch_bounds__(512) lvx_fp4_tile_kernel(fp4_args_t p) {
    constexpr int NB = 4, AV = MODE == A_BF16 ? 4 : 2, ROW = MODE == A_BF16 ? 256 : 128, CH = ROW / 16, MT = 32 * MBW;
    constexpr int WAVES = 8 / KG, NW = WAVES / 2, COLS = 64 * NW;               // waves of a group: two over the rows, NW over the columns
    constexpr int A_STAGE = MT * ROW, W_STAGE = COLS * 128, A_PER = 1024 / ROW;  // A_PER: rows of an instruction
    constexpr int DA = A_STAGE / (1024 * WAVES), DW = 4;                         // requests of a wave per stage
    extern __shared__ char lds[];  // [KG][RING] stages of rows, [KG][2] of weights, the scales; then the partial sums
    uint32_t *scales = reinterpret_cast<uint32_t *>(lds + KG * RING * A_STAGE + KG * 2 * W_STAGE);  // [COLS][PANEL]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int kg = wave / WAVES, in_group = wave % WAVES, mw = in_group / NW, nw = in_group % NW;
    const int r = lane & 15, g = lane >> 4;
    const int n0 = blockIdx.x * COLS, m0 = blockIdx.y * MT;
    const int steps = (p.K + 127) / 128, rounds = (steps + 2 * KG - 1) / (2 * KG);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
    const uint32_t lds_a = lds0 + kg * RING * A_STAGE, lds_w = lds0 + KG * RING * A_STAGE + kg * 2 * W_STAGE;

    // this wave's share of its group's requests: rows past the end repeat the last one (they are multiplied and not stored)
    uint32_t a_off[DA], a_col[DA], w_off[DW], w_col[DW];
#pragma unroll
    for (int i = 0; i < DA; ++i) {
        const int row = (in_group * DA + i) * A_PER + lane / CH;
        a_off[i] = (uint32_t)((m0 + row < p.M ? row : p.M - 1 - m0) * p.lda);
        a_col[i] = (uint32_t)((lane % CH) ^ (row % CH));
    }
#pragma unroll
    for (int i = 0; i < DW; ++i) {
        const int row = (in_group * DW + i) * 8 + lane / 8;
        w_off[i] = (uint32_t)((n0 + row < p.N ? row : p.N - 1 - n0) * p.ldw);
        w_col[i] = (uint32_t)((lane % 8) ^ (row % 8));
    }
    const char *a_base = p.A + (int64_t)m0 * p.lda;
    const uint8_t *w_base = p.W + (int64_t)n0 * p.ldw;
    // the group's j-th step: pairs kg, kg + KG, ... of two steps each
    auto step = [&](int j) { return 2 * (kg + KG * (j >> 1)) + (j & 1); };
    // of the last stage, chunks behind K are not read: the row's first is, in their place, and not used
    auto stage_a = [&](int j) {
        const int t = step(j);
        const uint32_t chunks = (uint32_t)((p.K - 128 * t) * (ROW / 128) / 16), to = lds_a + (j % RING) * A_STAGE;
#pragma unroll
        for (int i = 0; i < DA; ++i)
            lvx_dma16(a_base, a_off[i] + (a_col[i] < chunks ? (uint32_t)t * ROW + 16 * a_col[i] : 0), to + (in_group * DA + i) * 1024);
    };
    auto stage_w = [&](int j) {  // of the pair that begins with step j
        const int q = kg + KG * (j >> 1);
        const uint32_t chunks = (uint32_t)((p.K - 256 * q) / 32), to = lds_w + ((j >> 1) & 1) * W_STAGE;
#pragma unroll
        for (int i = 0; i < DW; ++i)
            lvx_dma16(w_base, w_off[i] + (w_col[i] < chunks ? (uint32_t)q * 128 + 16 * w_col[i] : 0), to + (in_group * DW + i) * 1024);
    };
    // the scales of the PANEL steps (of all groups) from the groups' step j on: 16 bytes = four steps of a column a piece
    auto load_scales = [&](int j) {
        const int b0 = 4 * KG * j, row_bytes = p.K / LVX_FP4_GROUP;
        constexpr int ALL = COLS * (PANEL / 4), PIECES = (ALL + 511) / 512;
        uint4 v[PIECES];
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int piece = threadIdx.x + 512 * i, row = piece / (PANEL / 4), at = b0 + 16 * (piece % (PANEL / 4));
            const uint8_t *src = p.S + (n0 + row < p.N ? n0 + row : p.N - 1) * p.lds + at;
            uint32_t e[4] = {0, 0, 0, 0};
            if (ALL % 512 != 0 && piece >= ALL) continue;
            if (at + 16 <= row_bytes) {
                __builtin_memcpy(e, src, 16);
            } else if (at < row_bytes) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (at + 4 * k + 4 <= row_bytes) {
                        __builtin_memcpy(&e[k], src + 4 * k, 4);
                    } else {
#pragma unroll
                        for (int x = 0; x < 3; ++x)
                            if (at + 4 * k + x < row_bytes) e[k] |= (uint32_t)src[4 * k + x] << (8 * x);
                    }
                }
            }
            v[i] = make_uint4(e[0], e[1], e[2], e[3]);
        }
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int piece = threadIdx.x + 512 * i;
            if (ALL % 512 != 0 && piece >= ALL) continue;
            *reinterpret_cast<uint4 *>(scales + (piece / (PANEL / 4)) * PANEL + 4 * (piece % (PANEL / 4))) = v[i];
        }
    };
    f32x4_t acc[NB][MBW];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int c = 0; c < MBW; ++c) acc[b][c] = {0, 0, 0, 0};

    struct operands_t {
        uint4 a[MBW][AV], w[NB];
        uint32_t s[NB];
    } x[2];
    auto read = [&](int j, operands_t &d) {
        const int t = step(j);
        if (t >= steps) return;
        const char *a_src = lds + kg * RING * A_STAGE + (j % RING) * A_STAGE + (mw * 16 * MBW + r) * ROW;
        const char *w_src = lds + KG * RING * A_STAGE + (kg * 2 + ((j >> 1) & 1)) * W_STAGE + (nw * 64 + r) * 128;
        const uint8_t *mine = reinterpret_cast<const uint8_t *>(scales + (nw * 64 + r) * PANEL + t % PANEL) + g;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            d.w[b] = *reinterpret_cast<const uint4 *>(w_src + b * 16 * 128 + 16 * ((4 * (j & 1) + g) ^ (r % 8)));
            d.s[b] = (uint32_t)mine[16 * b * PANEL * 4] << (MODE == A_NATIVE ? 0 : 23);
        }
#pragma unroll
        for (int c = 0; c < MBW; ++c)
#pragma unroll
            for (int i = 0; i < AV; ++i) {
                const int chunk = MODE == A_BF16 ? 4 * g + i : MODE == A_WIDEN ? 2 * g + i : g + 4 * i;
                d.a[c][i] = *reinterpret_cast<const uint4 *>(a_src + c * 16 * ROW + 16 * (chunk ^ (r % CH)));
            }
        const int left = p.K - 128 * t;
        if (left < 128) {  // lanes of channels behind K multiply zeros
#pragma unroll
            for (int c = 0; c < MBW; ++c)
#pragma unroll
                for (int i = 0; i < AV; ++i)
                    if ((MODE == A_NATIVE ? 16 * g + 64 * i : 32 * g) >= left) d.a[c][i] = make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int b = 0; b < NB; ++b) d.s[b] = 32 * g < left ? d.s[b] : 127u << (MODE == A_NATIVE ? 0 : 23);
        }
    };
    // Iteration j multiplies step j (in registers), reads step j + 1 (in LDS) and requests the rows of step j + RING into the place of step j, and the weights of the pair that
    // begins with it into the place of the pair before, which every wave has read.  Requests complete in order: with three stages those of this iteration may be left when
    // the ones before have to be there.
    auto iteration = [&](int j, bool odd, const operands_t &now, operands_t &next) {
        __syncthreads();
        const bool more = step(j + RING) < steps, more_w = more && odd == (RING == 3);
        if (more) stage_a(j + RING);
        if (more_w) stage_w(j + RING);
        if (odd && (j + 1) % (PANEL / KG) == 0) {
            load_scales(j + 1);
            __syncthreads();
        }
        read(j + 1, next);
        if (step(j) < steps) fp4_multiply<MODE, MBW, NB>(acc, now.w, now.s, now.a);
        if (RING == 3 && more_w)
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(DA + DW) : "memory");
        else if (RING == 3 && more)
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(DA) : "memory");
        else
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    };
#pragma unroll
    for (int j = 0; j < RING; ++j)
        if (step(j) < steps) stage_a(j);
    if (step(0) < steps) stage_w(0);
    if (RING == 3 && step(2) < steps) stage_w(2);
    load_scales(0);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    read(0, x[0]);
    for (int j = 0; j < 2 * rounds; j += 2) {
        iteration(j, false, x[0], x[1]);
        iteration(j + 1, true, x[1], x[0]);
    }
    __syncthreads();

    float row_scale[MBW];
    fp4_row_scales<MODE, MBW>(p, m0 + mw * 16 * MBW + r, row_scale);
    // each group finishes NB / KG of the columns' blocks with the others' sums, adding in the order of the groups
    f32x4_t *part = reinterpret_cast<f32x4_t *>(lds);
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int c = 0; c < MBW; ++c)
            if (b / (NB / KG) != kg) part[((wave * NB + b) * MBW + c) * 64 + lane] = acc[b][c];
    __syncthreads();
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        if (b / (NB / KG) != kg) continue;
        f32x4_t sum[MBW];
#pragma unroll
        for (int c = 0; c < MBW; ++c) {
#pragma unroll
            for (int k = 0; k < KG; ++k) {
                const f32x4_t its = k == kg ? acc[b][c] : part[(((k * WAVES + in_group) * NB + b) * MBW + c) * 64 + lane];
                sum[c] = k == 0 ? its : sum[c] + its;
            }
        }
        fp4_store<MBW>(p, m0 + mw * 16 * MBW + r, n0 + nw * 64 + 16 * b + 4 * g, sum, row_scale);
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

template <int MODE, int MB, int NB, int U>
void launch_few(const fp4_args_t &p, int most_waves, hipStream_t stream) {
    // as many waves as share the units of U steps evenly
    const int units = (p.K + 128 * U - 1) / (128 * U), rounds = (units + most_waves - 1) / most_waves, waves = (units + rounds - 1) / rounds;
    const dim3 grid((p.N + 16 * NB - 1) / (16 * NB), (p.M + 16 * MB - 1) / (16 * MB));
    hipLaunchKernelGGL((lvx_fp4_few_kernel<MODE, MB, NB, U>), grid, dim3(64 * waves), (waves - 1) * NB * MB * 1024, stream, p);
}

template <int MODE, int NB>
void launch_resident(const fp4_args_t &p, hipStream_t stream) {
    const int steps = (p.K + 127) / 128, rounds = (steps + 7) / 8, waves = (steps + rounds - 1) / rounds;
    const int operands = (int)lvx_fp4_resident_bytes(MODE == A_BF16 ? 2 : 1, p.M, p.K, NB), sums = waves * NB * 1024;
    hipLaunchKernelGGL((lvx_fp4_resident_kernel<MODE, NB>), dim3((p.N + 16 * NB - 1) / (16 * NB)), dim3(64 * waves), operands > sums ? operands : sums, stream, p);
}

template <int MODE, int MBW, int KG, int RING>
void launch_tile(const fp4_args_t &p, hipStream_t stream) {
    constexpr int cols = 256 / KG, stages = KG * RING * 32 * MBW * (MODE == A_BF16 ? 256 : 128) + KG * 2 * cols * 128, sums = 8 * 4 * MBW * 1024;
    constexpr int bytes = stages + cols * PANEL * 4;
    static_assert(bytes <= 160 * 1024 && sums <= bytes && PANEL % (2 * KG) == 0, "LDS");
    const dim3 grid((p.N + cols - 1) / cols, (p.M + 32 * MBW - 1) / (32 * MBW));
    hipLaunchKernelGGL((lvx_fp4_tile_kernel<MODE, MBW, KG, RING>), grid, dim3(512), bytes, stream, p);
}

template <int MODE>
void launch_tile_8(const fp4_args_t &p, int blocks, bool four, hipStream_t stream) {
    if (four)
        blocks == 2 ? launch_tile<MODE, 2, 4, 2>(p, stream) : launch_tile<MODE, 1, 4, 3>(p, stream);
    else
        blocks == 3 ? launch_tile<MODE, 3, 2, 3>(p, stream) : blocks == 2 ? launch_tile<MODE, 2, 2, 3>(p, stream) : launch_tile<MODE, 1, 2, 3>(p, stream);
}

// Few rows, or many that lie too far apart for the tiles.  More columns to a workgroup share the loads of A; that pays where enough workgroups are left (16 8-bit rows x 5120 x 5120: two blocks of
// columns are fastest, 8.4 us; 16 bf16 rows x 13824 x 5120: 14.3 with four, 17.5 with two; 1280 columns: one).
template <int MODE>
void linear_few(const fp4_args_t &p, hipStream_t stream) {
    const int nb = lvx_fp4_resident(MODE == A_BF16 ? 2 : 1, p.M, p.N, p.K);
    if (nb != 0) {
        nb == 4 ? launch_resident<MODE, 4>(p, stream) : nb == 2 ? launch_resident<MODE, 2>(p, stream) : launch_resident<MODE, 1>(p, stream);
        return;
    }
    const int blocks = (p.M + 15) / 16, tiles = (blocks + 3) / 4, mb = (blocks + tiles - 1) / tiles;
    const bool two = p.N >= 4096;
    if (mb == 1)
        p.N >= 12800 ? launch_few<MODE, 1, 4, 2>(p, 8, stream) : two ? launch_few<MODE, 1, 2, 2>(p, 8, stream) : launch_few<MODE, 1, 1, 2>(p, 8, stream);
    else if (mb == 2)
        two ? launch_few<MODE, 2, 2, 2>(p, 5, stream) : launch_few<MODE, 2, 1, 2>(p, 5, stream);
    else if (mb == 3)
        two ? launch_few<MODE, 3, 2, 2>(p, 5, stream) : launch_few<MODE, 3, 1, 2>(p, 5, stream);
    else
        two ? launch_few<MODE, 4, 2, MODE == A_BF16 ? 1 : 2>(p, 4, stream) : launch_few<MODE, 4, 1, MODE == A_BF16 ? 1 : 2>(p, 4, stream);
}

void linear_launch(const fp4_args_t &p, bool a8, bool mixed, hipStream_t stream) {
    // 8-bit rows are widened to bf16, whose products with the weights are exact, and summed in fp32.  A caller may ask for the mixed instruction, E4M3 by E2M1 at twice the rate
    // (544 x 5120 x 13824: 51 us against 84): it lines the products of four neighbouring channels up with the largest of them and cuts what lies 12 binary places below
    // its leading bit (measured; the fours and the steps are added in fp32), on normal rows 4e-6 of a sum.  Up to 32 rows are bound by the weights and are widened all the same.
    const int mode = !a8 ? A_BF16 : mixed && p.M > 32 ? A_NATIVE : A_WIDEN;
    const lvx_fp4_plan_t pl = lvx_fp4_call_plan(mode, p.M, p.N, p.K, p.lda, p.ldw);
    if (pl.blocks == 0) {
        a8 ? linear_few<A_WIDEN>(p, stream) : linear_few<A_BF16>(p, stream);
        return;
    }
    const bool four = pl.groups == 4;
    if (mode == A_BF16)
        four ? launch_tile<A_BF16, 1, 4, 2>(p, stream) : pl.blocks == 2 ? launch_tile<A_BF16, 2, 2, 2>(p, stream) : launch_tile<A_BF16, 1, 2, 3>(p, stream);
    else if (mode == A_NATIVE)
        launch_tile_8<A_NATIVE>(p, pl.blocks, four, stream);
    else
        launch_tile_8<A_WIDEN>(p, pl.blocks, four, stream);
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
    LVX_REQUIRE(K <= 1 << 30, LVX_ERR_SHAPE, "K %d is more than 2^30 channels", K);  // steps and units of steps are counted in 32 bits, rounded up
    LVX_REQUIRE(N % 8 == 0 && N <= 1 << 24, LVX_ERR_SHAPE, "N %d must be a multiple of 8, at most 2^24", N);
    LVX_REQUIRE(lda >= K && lda % (a8 ? 16 : 8) == 0 && ldw >= K / 2 && ldw % 16 == 0 && lds >= K / LVX_FP4_GROUP && ldc >= N && ldc % 8 == 0,
                LVX_ERR_SHAPE, "bad leading dimension");
    LVX_REQUIRE(M <= 1 << 20, LVX_ERR_SHAPE, "M %d is more than 2^20 rows", M);
    const bool mixed = a8 && ((int)epi & LVX_EPI_MIXED_8X4) != 0;
    if (mixed) epi = (lvx_epilogue_t)((int)epi & ~LVX_EPI_MIXED_8X4);
    LVX_REQUIRE(epi == LVX_EPI_STORE || epi == LVX_EPI_GELU_TANH || epi == LVX_EPI_RESID_GATE || epi == LVX_EPI_RESID_GATE_F32 || epi == LVX_EPI_STORE_F32,
                LVX_ERR_INVALID_ARG, "unknown epilogue %d", (int)epi);
    LVX_REQUIRE(!mixed || (epi != LVX_EPI_RESID_GATE_F32 && epi != LVX_EPI_STORE_F32), LVX_ERR_INVALID_ARG, "mixed products are for bf16 outputs, not epilogue %d", (int)epi);
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
    linear_launch(p, a8, mixed, stream);
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
