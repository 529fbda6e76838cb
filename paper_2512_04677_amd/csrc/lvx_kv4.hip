// KV cache in 4 bits for grouped-head attention of many sequences: append, read back, attention.
//
// Storage: [layer][sequence][kv head][tile of 64 keys], a record per tile, laid out as the matrix instructions take it, so that every load of the
// attention is a wave's contiguous 1 KB and nothing is transposed or shuffled there:
//   K       a lane (r = lane % 16, g = lane / 16) holds, per block of 16 keys, D / 4 consecutive channels from g D / 4 on of one key.  Row r of block kb is key
//           32 (kb / 2) + 8 (r / 4) + 4 (kb % 2) + r % 4: with that order the scores a lane gets for two blocks are those of eight consecutive keys,
//           which is what the second product takes as its operand.
//   V       transposed: a lane holds eight consecutive keys (a word) of channel 16 cb + r, per channel block cb and half of the tile.
//   scales  E8M0 per key and 32 channels of K (applied by the conversion to bf16, exactly), bf16 per key of V (applied to the probability in fp32: the
//           second product sums over keys, so a scale of V can neither wait until after it nor, unless a power of two, go into its operand without rounding).
//
// One token each of 32 sequences of up to 24960 keys (8 kv heads, 40 heads, 510 MB): 91 us with the join, 5.6 TB/s, bound by HBM.  1560 tokens of 40 heads against 24960 keys:
// 730 to 780 us on different cards, 1.0 to 1.06 PFLOP/s, bound by the vector unit (conversions, exponentials, packing: about 350 instructions a wave and tile beside 64 matrix products).
#include "lvx_fp4.h"
#include "lvx_kv4_rules.h"

#include <new>

struct lvx_kv4 {
    lvx_kv4_desc_t desc;
    uint8_t *base;
    int64_t record, head_stride, seq_stride, layer_stride;  // bytes
};

namespace {

constexpr int TILE = LVX_KEY_TILE;

// Offsets within a tile's record.
template <int D>
struct tile_t {
    static constexpr int V = 32 * D, KS = 64 * D, VS = 66 * D, BYTES = 66 * D + 128;
    static __device__ __forceinline__ int row_of(int key) { return ((key >> 3) & 3) * 4 + (key & 3); }     // row within its block of 16
    static __device__ __forceinline__ int block_of(int key) { return (key >> 5) * 2 + ((key >> 2) & 1); }  // which of the tile's four blocks
    // the 16 bytes of channels 32 grp .. 32 grp + 31 of a key: one piece for D = 128, two of eight bytes (lanes 16 apart) for D = 64
    static __device__ __forceinline__ int k_piece(int key, int grp, int half) {
        const int r = row_of(key), kb = block_of(key);
        if (D == 128) return kb * 1024 + (grp * 16 + r) * 16 + 8 * half;
        return (kb >> 1) * 1024 + ((2 * grp + half) * 16 + r) * 16 + (kb & 1) * 8;
    }
    static __device__ __forceinline__ int k_scale(int key, int grp) { return KS + (grp * 16 + row_of(key)) * 4 + block_of(key); }
    // the word of channel c for the eight keys from `key` (a multiple of eight) on
    static __device__ __forceinline__ int v_word(int key, int c) {
        const int cb = c >> 4, g = (key >> 3) & 3, t = key >> 5;
        return V + (cb >> 1) * 1024 + (g * 16 + (c & 15)) * 16 + ((cb & 1) * 2 + t) * 4;
    }
    static __device__ __forceinline__ int v_scale(int key) { return VS + 2 * key; }
};

// The call's tokens of sequence s: rows first .. first + n - 1; the last of them is key count - 1.
struct batch_t {
    const int32_t *starts;  // NULL: n_each tokens for every sequence
    const int32_t *counts;
    int32_t n_each, n_tokens;
};
struct span_t {
    int first, n, count;  // count: as given, it may pass the slot
};
__device__ __forceinline__ span_t span_of(const batch_t &b, int s) {
    span_t r;
    if (b.starts != nullptr) {
        // whatever the array holds, no row outside [0, n_tokens) is touched
        const int lo = b.starts[s], hi = b.starts[s + 1];
        r.first = lo < 0 ? 0 : lo;
        const int end = hi < b.n_tokens ? hi : b.n_tokens;
        r.n = end > r.first ? end - r.first : 0;
        r.n = r.n < b.n_each ? r.n : b.n_each;
    } else {
        r.first = s * b.n_each, r.n = b.n_each;
    }
    const int c = b.counts[s];
    r.count = c > -(1 << 30) ? c : -(1 << 30);
    return r;
}
// keys that token i of the span sees, of those that the slot holds
__device__ __forceinline__ int keys_seen(const span_t &sp, int i, bool causal, int max_keys) {
    const int c = causal ? sp.count - (sp.n - 1 - i) : sp.count;
    return c < 0 ? 0 : c < max_keys ? c : max_keys;
}

struct append_args_t {
    uint8_t *base;  // of the layer
    int64_t head_stride, seq_stride;
    const bf16_t *k, *v;
    int64_t ld;
    batch_t batch;
    int32_t kv_heads, max_keys;
};

// maximum over a row of 16 lanes, in all of them
__device__ __forceinline__ uint32_t row_max(uint32_t v) {
#define LVX_ROR(n_)                                                                                     \
    {                                                                                                   \
        const uint32_t o = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x120 + n_, 0xf, 0xf, false);     \
        v = v > o ? v : o;                                                                              \
    }
    LVX_ROR(8) LVX_ROR(4) LVX_ROR(2) LVX_ROR(1)
#undef LVX_ROR
    return v;
}
__device__ __forceinline__ uint32_t swap_max(uint32_t a, uint32_t b, bool halves) {  // lanes of the lower half (even rows): a's maximum over the halves (row pairs), the others: b's
    if (halves) {
        const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
        return r[0] > r[1] ? r[0] : r[1];
    }
    const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
    return r[0] > r[1] ? r[0] : r[1];
}

// A wave quantises 8 NG aligned keys of one head: the keys of a word of V are never shared between waves, so a word that keeps other keys' codes is read and written by one.
// Bound by the loads' way and, for prompts, by the bytes (32 x 24960 keys of 8 heads 945 us, 4.4 TB/s; 4 prompts of up to 1560 tokens 11 us).
template <int D, int NG>
__global__ void __launch_bounds__(256) lvx_kv4_append_kernel(append_args_t p) {
    typedef tile_t<D> T;
    const int lane = threadIdx.x & 63;
    const int s = blockIdx.y, head = blockIdx.z * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (head >= p.kv_heads) return;
    const int c_raw = p.batch.counts[s];
    const span_t sp = span_of(p.batch, s);
    const int64_t pos0 = (int64_t)c_raw - sp.n;  // position of the first token, before clipping
    const int64_t lo = pos0 > 0 ? pos0 : 0, hi = c_raw < p.max_keys ? c_raw : p.max_keys;
    const int64_t first = (lo & ~(8ll * NG - 1)) + 8ll * NG * blockIdx.x;
    if (first >= hi || sp.n <= 0) return;
    uint8_t *rec = p.base + s * p.seq_stride + head * p.head_stride + (first / TILE) * T::BYTES;
    const int kt0 = (int)(first % TILE);

    // keys: a thread per key and group of 32 channels
    if (lane < 8 * NG * (D / 32)) {
        const int i = lane / (D / 32), grp = lane % (D / 32);
        const int64_t key = first + i;
        if (key >= lo && key < hi) {
            const uint4 *src = reinterpret_cast<const uint4 *>(p.k + (sp.first + (key - pos0)) * p.ld + head * D + 32 * grp);
            uint4 x[4];
            uint32_t m = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = src[j];
#pragma unroll
            for (int j = 0; j < 4; ++j) m = lvx_amax_bf16x2(lvx_amax_bf16x2(lvx_amax_bf16x2(lvx_amax_bf16x2(m, x[j].x), x[j].y), x[j].z), x[j].w);
            const uint32_t byte = lvx_fp4_group_byte(m);
            const float scale = lvx_e8m0_f32(byte);
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = byte == 255 ? 0 : lvx_bf16x8_fp4(x[j].x, x[j].y, x[j].z, x[j].w, scale);
            *reinterpret_cast<uint2 *>(rec + T::k_piece(kt0 + i, grp, 0)) = make_uint2(w[0], w[1]);
            *reinterpret_cast<uint2 *>(rec + T::k_piece(kt0 + i, grp, 1)) = make_uint2(w[2], w[3]);
            rec[T::k_scale(kt0 + i, grp)] = (uint8_t)byte;
        }
    }

    // values: a lane has D / 64 channels of all keys
    constexpr int C = D / 64;
    uint32_t x[NG][8];
#pragma unroll
    for (int n = 0; n < NG; ++n)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t key = first + 8 * n + i;
            x[n][i] = 0;
            if (key < lo || key >= hi) continue;
            const bf16_t *src = p.v + (sp.first + (key - pos0)) * p.ld + head * D + C * lane;
            x[n][i] = C == 2 ? *reinterpret_cast<const uint32_t *>(src) : (uint32_t)*reinterpret_cast<const uint16_t *>(src);
        }
#pragma unroll
    for (int n = 0; n < NG; ++n) {
        const int64_t key0 = first + 8 * n;
        const int kt = kt0 + 8 * n;
        if (key0 >= hi || key0 + 8 <= lo) continue;
        // the eight maxima over the wave: over its halves, its pairs of rows, its rows of 16 lanes
        uint32_t m[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) m[i] = lvx_amax_bf16x2(0, x[n][i]);
#pragma unroll
        for (int i = 0; i < 4; ++i) m[i] = swap_max(m[2 * i], m[2 * i + 1], true);  // lower half: key 2 i, upper: 2 i + 1
#pragma unroll
        for (int i = 0; i < 2; ++i) m[i] = row_max(swap_max(m[2 * i], m[2 * i + 1], false));  // even rows: keys 4 i, 4 i + 1, odd rows: 4 i + 2, 4 i + 3
        uint32_t word[C];
#pragma unroll
        for (int c = 0; c < C; ++c) word[c] = 0;
        uint32_t keep = 0;  // nibbles of keys that this call does not write
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (key0 + i < lo || key0 + i >= hi) {
                keep |= 15u << (4 * i);
                continue;
            }
            const uint32_t most = __builtin_amdgcn_readlane(m[i >> 2], 32 * (i & 1) + 16 * ((i >> 1) & 1));
            const uint32_t sb = pack_bf16x2(__uint_as_float(most) / 6.0f, 0.f) & 0xffffu;
            float scale = bf16_bits_to_f32(sb);
            scale = scale < 0x1p-120f ? 0x1p-120f : scale;
            // x / scale has more than the bits that separate it from a border between two codes, so the division's rounding decides nothing
            const uint32_t code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0, bf16_lo(x[n][i]) / scale, bf16_hi(x[n][i]) / scale, 1.0f, 0);
#pragma unroll
            for (int c = 0; c < C; ++c) word[c] |= ((code >> (4 * c)) & 15u) << (4 * i);
            if (lane == 0) *reinterpret_cast<uint16_t *>(rec + T::v_scale(kt + i)) = (uint16_t)(__float_as_uint(scale) >> 16);
        }
#pragma unroll
        for (int c = 0; c < C; ++c) {
            uint32_t *dst = reinterpret_cast<uint32_t *>(rec + T::v_word(kt, C * lane + c));
            if (keep != 0) word[c] |= *dst & keep;
            *dst = word[c];
        }
    }
}

struct gather_args_t {
    const uint8_t *base;
    int64_t head_stride, seq_stride;
    bf16_t *k, *v;  // [sequence][n_keys][ld]
    int64_t ld;
    const int32_t *counts;
    int32_t first_key, n_keys, kv_heads, max_keys;
};

// A thread reads eight channels of eight aligned keys, or writes zeros behind the sequence's last key.
template <int D>
__global__ void __launch_bounds__(256) lvx_kv4_gather_kernel(gather_args_t p) {
    typedef tile_t<D> T;
    const int s = blockIdx.y, per_key = p.kv_heads * (D / 8);
    const int g0 = p.first_key / 8, groups = (p.first_key + p.n_keys + 7) / 8 - g0;
    const int64_t total = (int64_t)groups * per_key;
    const int count = p.counts[s] < p.max_keys ? p.counts[s] : p.max_keys;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int e = (int)(i % per_key), head = e / (D / 8), c0 = 8 * (e % (D / 8)), grp = c0 / 32, in = c0 % 32;
        const int key0 = 8 * (g0 + (int)(i / per_key)), kt = key0 % TILE;
        uint32_t kw[8], vw[8], kb[8];
        uint4 vs = make_uint4(0, 0, 0, 0);
        if (key0 < count) {
            const uint8_t *rec = p.base + s * p.seq_stride + head * p.head_stride + (int64_t)(key0 / TILE) * T::BYTES;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                kw[j] = *reinterpret_cast<const uint32_t *>(rec + T::k_piece(kt + j, grp, in / 16) + (in % 16) / 2);
                kb[j] = rec[T::k_scale(kt + j, grp)];
                vw[j] = *reinterpret_cast<const uint32_t *>(rec + T::v_word(kt, c0 + j));
            }
            vs = *reinterpret_cast<const uint4 *>(rec + T::v_scale(kt));
        }
        const uint32_t vsw[4] = {vs.x, vs.y, vs.z, vs.w};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int key = key0 + j;
            if (key < p.first_key || key >= p.first_key + p.n_keys) continue;
            uint4 ko = make_uint4(0, 0, 0, 0), vo = ko;
            if (key < count) {
                const bf16x8_t kx = lvx_fp4x8_bf16(kw[j], lvx_e8m0_f32(kb[j]));
                ko = *reinterpret_cast<const uint4 *>(&kx);
                uint32_t w = 0;
#pragma unroll
                for (int c = 0; c < 8; ++c) w |= ((vw[c] >> (4 * j)) & 15u) << (4 * c);
                const float f = (j & 1) ? bf16_hi(vsw[j >> 1]) : bf16_lo(vsw[j >> 1]);
                const bf16x8_t vx = lvx_fp4x8_bf16(w, 1.0f);
                vo.x = pack_bf16x2((float)vx[0] * f, (float)vx[1] * f), vo.y = pack_bf16x2((float)vx[2] * f, (float)vx[3] * f);
                vo.z = pack_bf16x2((float)vx[4] * f, (float)vx[5] * f), vo.w = pack_bf16x2((float)vx[6] * f, (float)vx[7] * f);
            }
            const int64_t at = ((int64_t)s * p.n_keys + key - p.first_key) * p.ld + head * D + c0;
            *reinterpret_cast<uint4 *>(p.k + at) = ko;
            *reinterpret_cast<uint4 *>(p.v + at) = vo;
        }
    }
}

struct attn_args_t {
    const uint8_t *base;
    int64_t head_stride, seq_stride;
    const bf16_t *q;
    bf16_t *out;
    int64_t ld_q, ld_out;
    batch_t batch;
    int32_t n_seqs, n_heads, kv_heads, group, max_keys, causal, splits, row_tiles;
    float scale_log2;
    float *part_o;   // [split][token row][head][D], un-normalised
    float2 *part_ml; // [split][token row][head]: reference (log2) and sum
};

// f over the four lanes that share a query (16 apart), in all of them
template <typename F>
__device__ __forceinline__ float across(float v, F f) {
    const uint32_t u = __float_as_uint(v);
    const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const uint32_t w = __float_as_uint(f(__uint_as_float(a[0]), __uint_as_float(a[1])));
    const auto b = __builtin_amdgcn_permlane16_swap(w, w, false, false);
    return f(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Rows of a workgroup: (token, head of the group) pairs of one sequence and kv head, row = token * group + head, 16 RB per wave, WR waves side by side;
// WK waves share the keys, every WK-th tile each.
template <int D, int RB, int WR, int WK>
__global__ void __launch_bounds__(64 * WR * WK, 2) lvx_kv4_attention_kernel(attn_args_t p) {
    typedef tile_t<D> T;
    constexpr int CB = D / 16, KS = D / 32;  // channel blocks, steps of 32 channels
    __shared__ f32x4_t join_o[WK > 1 ? WR * WK * RB * CB * 64 : 1];
    __shared__ float2 join_ml[WK > 1 ? WR * WK * RB * 16 : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wr = wave % WR, wk = wave / WR;
    const int r = lane & 15, g = lane >> 4;
    // the last rows first: a causal prompt's last see the most keys
    const int head = blockIdx.x % p.kv_heads, rt = p.row_tiles - 1 - (blockIdx.x / p.kv_heads) % p.row_tiles, split = blockIdx.x / p.kv_heads / p.row_tiles;
    const int s = blockIdx.y;
    const span_t sp = span_of(p.batch, s);
    const int n_rows = sp.n * p.group;
    if (rt * 16 * RB * WR >= n_rows) return;

    // this lane's rows: token, head and the number of keys they see
    int seen[RB];
    const int row0 = (rt * WR + wr) * 16 * RB;
    bf16x8_t q[RB][KS];
#pragma unroll
    for (int b = 0; b < RB; ++b) {
        const int row = row0 + 16 * b + r;
        seen[b] = 0;
#pragma unroll
        for (int j = 0; j < KS; ++j) q[b][j] = bf16x8_t{};
        if (row < n_rows) {  // rows behind the last one read nothing: every other row may be another workgroup's, which stores its output over it
            const int i = row / p.group;
            seen[b] = keys_seen(sp, i, p.causal, p.max_keys);
            const uint4 *src = reinterpret_cast<const uint4 *>(p.q + (int64_t)(sp.first + i) * p.ld_q + (head * p.group + row % p.group) * D + (D / 4) * g);
#pragma unroll
            for (int j = 0; j < KS; ++j) {
                const uint4 v = src[j];
                q[b][j] = *reinterpret_cast<const bf16x8_t *>(&v);
            }
        }
    }
    // the keys that any of the workgroup's rows sees, and those that all of this wave's rows see
    const int last_row = (rt + 1) * 16 * RB * WR < n_rows ? (rt + 1) * 16 * RB * WR - 1 : n_rows - 1;
    const int most = keys_seen(sp, last_row / p.group, p.causal, p.max_keys);
    const int least = keys_seen(sp, row0 < n_rows ? row0 / p.group : sp.n - 1, p.causal, p.max_keys);
    const int tiles = (most + TILE - 1) / TILE, per = (tiles + p.splits - 1) / p.splits;
    const int t0 = split * per, t1 = t0 + per < tiles ? t0 + per : tiles;

    f32x4_t o[RB][CB];
    float ref[RB], sum[RB];
    bool unset[RB];  // a row of the block has no reference yet and sees keys from here on
#pragma unroll
    for (int b = 0; b < RB; ++b) {
        ref[b] = row0 + 16 * b + r < n_rows ? -INFINITY : INFINITY;  // a row behind the last one: every power is zero, and it has no say in the votes
        sum[b] = 0, unset[b] = true;
#pragma unroll
        for (int c = 0; c < CB; ++c) o[b][c] = {0, 0, 0, 0};
    }

    const uint8_t *rec0 = p.base + s * p.seq_stride + head * p.head_stride;
    uint4 kq[D / 32];
    uint32_t ks = 0;
    auto load_keys = [&](int t) {
        const uint8_t *rec = rec0 + (int64_t)t * T::BYTES;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) kq[i] = *reinterpret_cast<const uint4 *>(rec + i * 1024 + lane * 16);
        ks = *reinterpret_cast<const uint32_t *>(rec + T::KS + ((D == 128 ? g : g >> 1) * 16 + r) * 4);
    };
    if (t0 + wk < t1) load_keys(t0 + wk);
    for (int t = t0 + wk; t < t1; t += WK) {
        const uint8_t *rec = rec0 + (int64_t)t * T::BYTES;
        uint4 vq[CB / 2], vsw[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) vsw[h] = *reinterpret_cast<const uint4 *>(rec + T::VS + 64 * h + 16 * g);
#pragma unroll
        for (int c2 = 0; c2 < CB / 2; ++c2) vq[c2] = *reinterpret_cast<const uint4 *>(rec + T::V + c2 * 1024 + lane * 16);
        // of the two waves of a SIMD the one with matrix products to issue goes first (801 -> 748 us for 1560 tokens of 40 heads against 24960 keys)
        if (WK == 1) __builtin_amdgcn_s_setprio(1);
        // scores, transposed: a lane has four keys of each block for its query
        f32x4_t x[RB][4];
#pragma unroll
        for (int b = 0; b < RB; ++b)
#pragma unroll
            for (int kb = 0; kb < 4; ++kb) x[b][kb] = {0, 0, 0, 0};
        // two blocks of keys in turn: a product waits for the one before it on the same sums
#pragma unroll
        for (int kp = 0; kp < 4; kp += 2) {
#pragma unroll
            for (int j = 0; j < KS; ++j) {
                bf16x8_t kf[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint4 v = kq[D == 128 ? kp + h : kp >> 1];
                    const uint32_t w[4] = {D == 128 || h == 0 ? v.x : v.z, D == 128 || h == 0 ? v.y : v.w, v.z, v.w};
                    kf[h] = lvx_fp4x8_bf16(w[j], lvx_e8m0_f32((ks >> (8 * (kp + h))) & 255u));
                }
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int b = 0; b < RB; ++b) x[b][kp + h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[h], q[b][j], x[b][kp + h], 0, 0, 0);
            }
        }
        // Registers bound how far ahead the next keys are requested: behind the scores where waves share the keys, else when the scores are done with.
        if (WK > 1 && t + WK < t1) load_keys(t + WK);
        if (WK == 1) __builtin_amdgcn_s_setprio(0);
        // softmax; lane's keys: 32 (kb / 2) + 8 g + 4 (kb % 2) + i
        const bool masked = TILE * (t + 1) > least;
        bf16x8_t pf[RB][2];
#pragma unroll
        for (int b = 0; b < RB; ++b) {
            float y[16];
            float base = ref[b] == -INFINITY ? 0.f : ref[b], l = 0;
            auto exponents = [&]() {
                l = 0;
#pragma unroll
                for (int kb = 0; kb < 4; ++kb)
#pragma unroll
                    for (int i = 0; i < 4; ++i) y[4 * kb + i] = x[b][kb][i] * p.scale_log2 - base;
                if (masked) {
                    const int left = seen[b] - TILE * t - 8 * g;
#pragma unroll
                    for (int kb = 0; kb < 4; ++kb)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (left <= 32 * (kb >> 1) + 4 * (kb & 1) + i) y[4 * kb + i] = -INFINITY;
                }
            };
            auto powers = [&]() {
#pragma unroll
                for (int i = 0; i < 16; ++i) y[i] = __builtin_amdgcn_exp2f(y[i]);
                float part[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) part[i] = (y[i] + y[i + 4]) + (y[i + 8] + y[i + 12]);
                l = (part[0] + part[1]) + (part[2] + part[3]);
            };
            // The reference that is subtracted only has to keep the powers inside fp32.  With the running maximum the largest probability is 1 and its rounding exact, which
            // peaked rows notice (errors of 1.7e-3 against 2.1e-3 with a reference that lags by up to 2^20): where the cache's bytes bound the kernel, that is what it is.
            // Where the vector unit does (one wave per tile of keys), it is the first tile's maximum, and a tile whose powers reach 2^4 of it moves it.  A power rounds to bf16 by
            // the same share of itself wherever the reference lies; only one of exactly 1 does not round (outputs 2.25e-3 off against 2.12e-3 with the running maximum, which
            // takes 763 us for 731).
            // A row whose scores so far are all -infinity takes its reference from the next tile, above zero or below.
            constexpr bool RUNNING = WK > 1;
            bool move = unset[b];
            float m = -INFINITY;
            auto maximum = [&]() {
#pragma unroll
                for (int i = 0; i < 16; ++i) m = fmaxf(m, y[i]);
                m = across(m, [](float a, float b) { return fmaxf(a, b); });
            };
            exponents();
            if (RUNNING) {
                maximum();
                move = move || __any(m > 0.f);
            } else if (!move) {
                powers();
                move = __any(!(l < 0x1p4f));
                if (move) exponents();
            }
            if (move) {
                if (!RUNNING) maximum();
                const float next = fmaxf(ref[b], m + base);
                base = next == -INFINITY ? 0.f : next;
                const float shrink = __builtin_amdgcn_exp2f(ref[b] - base);
                ref[b] = next;
                unset[b] = __any(next == -INFINITY && seen[b] > TILE * (t + 1));
                exponents();
                sum[b] *= shrink;
#pragma unroll
                for (int c = 0; c < CB; ++c)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[b][c][i] *= shrink;
            }
            if (RUNNING || move) powers();
            sum[b] += l;
            // the probability times the value's scale, rounded to bf16 once
            const uint32_t w[8] = {vsw[0].x, vsw[0].y, vsw[0].z, vsw[0].w, vsw[1].x, vsw[1].y, vsw[1].z, vsw[1].w};
            float z[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) z[i] = y[i] * ((i & 1) ? bf16_hi(w[i >> 1]) : bf16_lo(w[i >> 1]));
            if (masked) {  // a hidden key's scale may be anything; a NaN that is seen stays, however small its probability
                int left = seen[b] - TILE * t - 8 * g;
                asm volatile("" : "+v"(left));  // compared afresh: the conditions above, kept until here, cost the kernel for prompts 50 of 785 us
#pragma unroll
                for (int kb = 0; kb < 4; ++kb)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (left <= 32 * (kb >> 1) + 4 * (kb & 1) + i) z[4 * kb + i] = 0.f;
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint4 v = make_uint4(pack_bf16x2(z[8 * h], z[8 * h + 1]), pack_bf16x2(z[8 * h + 2], z[8 * h + 3]), pack_bf16x2(z[8 * h + 4], z[8 * h + 5]),
                                           pack_bf16x2(z[8 * h + 6], z[8 * h + 7]));
                pf[b][h] = *reinterpret_cast<const bf16x8_t *>(&v);
            }
        }
        if (WK == 1 && t + WK < t1) load_keys(t + WK);
        if (WK == 1) __builtin_amdgcn_s_setprio(1);
        // outputs, transposed: a lane has four channels of each block for its query
#pragma unroll
        for (int c2 = 0; c2 < CB / 2; ++c2) {
            const uint32_t w[4] = {vq[c2].x, vq[c2].y, vq[c2].z, vq[c2].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int e = (i & 1) * 2 + (i >> 1);  // the two blocks of channels in turn
                const bf16x8_t vf = lvx_fp4x8_bf16(w[e], 1.0f);
#pragma unroll
                for (int b = 0; b < RB; ++b)
                    o[b][2 * c2 + (e >> 1)] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[b][e & 1], o[b][2 * c2 + (e >> 1)], 0, 0, 0);
            }
        }
    }
#pragma unroll
    for (int b = 0; b < RB; ++b) {
        sum[b] = across(sum[b], [](float a, float b) { return a + b; });
    }

    // The waves that shared the keys leave their results to each other: every wave joins, in the order of the waves, and stores its share of the channel blocks.
    if (WK > 1) {
#pragma unroll
        for (int b = 0; b < RB; ++b) {
            if (g == 0) join_ml[((wr * WK + wk) * RB + b) * 16 + r] = make_float2(ref[b], sum[b]);
#pragma unroll
            for (int c = 0; c < CB; ++c) join_o[(((wr * WK + wk) * RB + b) * CB + c) * 64 + lane] = o[b][c];
        }
        __syncthreads();
    }
#pragma unroll
    for (int b = 0; b < RB; ++b) {
        const int row = row0 + 16 * b + r;
        const bool there = row < n_rows;
        const int64_t token = sp.first + row / p.group;
        const int head_of = head * p.group + row % p.group;
        float factor[WK];
        if (WK > 1) {
            ref[b] = -INFINITY, sum[b] = 0;
            float2 ml[WK];
#pragma unroll
            for (int k = 0; k < WK; ++k) {
                ml[k] = join_ml[((wr * WK + k) * RB + b) * 16 + r];
                ref[b] = fmaxf(ref[b], ml[k].x);
            }
#pragma unroll
            for (int k = 0; k < WK; ++k) {
                factor[k] = __builtin_amdgcn_exp2f(ml[k].x - (ref[b] == -INFINITY ? 0.f : ref[b]));
                sum[b] += ml[k].y * factor[k];
            }
        }
        const int64_t at = ((int64_t)split * p.batch.n_tokens + token) * p.n_heads + head_of;
        const float inv = seen[b] > 0 ? 1.0f / sum[b] : 0.f;  // a row that sees no key is zero
        if (p.splits > 1 && there && g == 0 && wk == 0) p.part_ml[at] = make_float2(ref[b], sum[b]);
#pragma unroll
        for (int c = 0; c < CB; ++c) {
            if (WK > 1 && (b * CB + c) % WK != wk) continue;
            f32x4_t v = o[b][c];
            if (WK > 1) {
                v = {0, 0, 0, 0};
#pragma unroll
                for (int k = 0; k < WK; ++k) {
                    const f32x4_t its = join_o[(((wr * WK + k) * RB + b) * CB + c) * 64 + lane];
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] += its[i] * factor[k];
                }
            }
            if (!there) continue;
            if (p.splits > 1)
                *reinterpret_cast<f32x4_t *>(p.part_o + at * D + 16 * c + 4 * g) = v;
            else
                *reinterpret_cast<uint2 *>(p.out + token * p.ld_out + head_of * D + 16 * c + 4 * g) =
                    make_uint2(pack_bf16x2(v[0] * inv, v[1] * inv), pack_bf16x2(v[2] * inv, v[3] * inv));
        }
    }
}

// Joins the ranges of keys: a wave per token row and head, D / 64 channels a lane.
template <int D>
__global__ void __launch_bounds__(256) lvx_kv4_combine_kernel(attn_args_t p) {
    constexpr int C = D / 64;
    const int lane = threadIdx.x & 63;
    const int s = blockIdx.y;
    const span_t sp = span_of(p.batch, s);
    const int row = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= sp.n * p.n_heads) return;
    const int i = row / p.n_heads, head = row % p.n_heads;
    const int64_t at0 = (int64_t)(sp.first + i) * p.n_heads + head, step = (int64_t)p.batch.n_tokens * p.n_heads;
    // lane k has range k's reference and sum
    const float2 ml = lane < p.splits ? p.part_ml[at0 + lane * step] : make_float2(-INFINITY, 0.f);
    float ref = ml.x;
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) ref = fmaxf(ref, __shfl_xor(ref, d));
    const float factor = __builtin_amdgcn_exp2f(ml.x - (ref == -INFINITY ? 0.f : ref));
    float sum = ml.y * factor;
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) sum += __shfl_xor(sum, d);
    float o[C] = {};
    const float *src = p.part_o + at0 * D + C * lane;
    for (int k0 = 0; k0 < p.splits; k0 += 8) {
        float x[8][C];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float *from = src + (k0 + k < p.splits ? k0 + k : 0) * step * D;
#pragma unroll
            for (int c = 0; c < C; ++c) x[k][c] = from[c];
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float f = k0 + k < p.splits ? __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(factor), k0 + k)) : 0.f;
#pragma unroll
            for (int c = 0; c < C; ++c) o[c] += k0 + k < p.splits ? x[k][c] * f : 0.f;
        }
    }
    const float inv = keys_seen(sp, i, p.causal, p.max_keys) > 0 ? 1.0f / sum : 0.f;
    bf16_t *dst = p.out + (sp.first + i) * p.ld_out + head * D + C * lane;
    if (C == 2)
        *reinterpret_cast<uint32_t *>(dst) = pack_bf16x2(o[0] * inv, o[C - 1] * inv);
    else
        *reinterpret_cast<uint16_t *>(dst) = (uint16_t)pack_bf16x2(o[0] * inv, 0.f);
}

lvx_status_t check_desc(const lvx_kv4_desc_t *d) {
    LVX_REQUIRE(d != nullptr, LVX_ERR_INVALID_ARG, "cache descriptor is NULL");
    LVX_REQUIRE(d->n_layers > 0 && d->n_seqs > 0 && d->n_kv_heads > 0 && d->max_keys > 0, LVX_ERR_SHAPE,
                "layers %d, sequences %d, kv heads %d and keys %d must be positive", d->n_layers, d->n_seqs, d->n_kv_heads, d->max_keys);
    LVX_REQUIRE(d->head_dim == 64 || d->head_dim == 128, LVX_ERR_UNSUPPORTED, "head_dim %d is not 64 or 128", d->head_dim);
    LVX_REQUIRE(d->n_seqs <= 65535 && d->n_kv_heads <= 1024 && d->max_keys <= (1 << 26), LVX_ERR_SHAPE,
                "at most 65535 sequences, 1024 kv heads and 2^26 keys");
    return LVX_OK;
}

// bytes of the whole cache, 0 if they do not fit 62 bits
uint64_t cache_bytes(const lvx_kv4_desc_t *d) {
    const uint64_t tiles = ((uint64_t)d->max_keys + TILE - 1) / TILE, record = 66ull * d->head_dim + 128;
    const unsigned __int128 n = (unsigned __int128)(tiles * record) * (uint64_t)d->n_kv_heads * (uint64_t)d->n_seqs * (uint64_t)d->n_layers;
    return n >> 62 ? 0 : (uint64_t)n;
}

lvx_status_t check_call(const lvx_kv4_t *c, int32_t layer, const int32_t *starts, int32_t n_tokens, int32_t max_tokens, const int32_t *counts) {
    LVX_REQUIRE(c != nullptr, LVX_ERR_INVALID_ARG, "cache handle is NULL");
    LVX_REQUIRE(layer >= 0 && layer < c->desc.n_layers, LVX_ERR_INVALID_ARG, "layer %d outside [0,%d)", layer, c->desc.n_layers);
    LVX_REQUIRE(counts != nullptr && (((uintptr_t)counts | (uintptr_t)starts) & 3u) == 0, LVX_ERR_INVALID_ARG,
                "key counts are NULL, or counts or starts are not 4-byte aligned");
    LVX_REQUIRE(n_tokens >= 0 && max_tokens >= 0, LVX_ERR_SHAPE, "tokens %d, tokens of a sequence %d", n_tokens, max_tokens);
    LVX_REQUIRE((int64_t)max_tokens * c->desc.n_seqs >= n_tokens, LVX_ERR_SHAPE, "%d tokens are more than %d sequences of at most %d", n_tokens,
                c->desc.n_seqs, max_tokens);
    LVX_REQUIRE(starts != nullptr || (int64_t)max_tokens * c->desc.n_seqs == n_tokens, LVX_ERR_SHAPE,
                "without starts every sequence has max_tokens tokens: %d x %d are not %d", c->desc.n_seqs, max_tokens, n_tokens);
    return LVX_OK;
}

}  // namespace

extern "C" size_t lvx_kv4_bytes(const lvx_kv4_desc_t *desc) {
    if (check_desc(desc) != LVX_OK) return 0;
    const uint64_t n = cache_bytes(desc);
    if (n == 0) lvx_fail(LVX_ERR_SHAPE, "the cache is larger than 2^62 bytes");
    return (size_t)n;
}

extern "C" lvx_status_t lvx_kv4_init(const lvx_kv4_desc_t *desc, void *dev_storage, size_t bytes, lvx_kv4_t **out) {
    LVX_REQUIRE(out != nullptr, LVX_ERR_INVALID_ARG, "out is NULL");
    LVX_TRY(check_desc(desc));
    const uint64_t need = cache_bytes(desc);
    LVX_REQUIRE(need != 0, LVX_ERR_SHAPE, "the cache is larger than 2^62 bytes");
    LVX_REQUIRE(dev_storage != nullptr && (((uintptr_t)dev_storage) & 255u) == 0, LVX_ERR_INVALID_ARG, "storage is NULL or not 256-byte aligned");
    LVX_REQUIRE(bytes >= need, LVX_ERR_SHAPE, "storage of %zu bytes, %llu needed", bytes, (unsigned long long)need);
    lvx_kv4_t *c = new (std::nothrow) lvx_kv4_t;
    LVX_REQUIRE(c != nullptr, LVX_ERR_INVALID_ARG, "out of host memory");
    c->desc = *desc;
    c->base = (uint8_t *)dev_storage;
    c->record = 66ll * desc->head_dim + 128;
    c->head_stride = ((int64_t)desc->max_keys + TILE - 1) / TILE * c->record;
    c->seq_stride = c->head_stride * desc->n_kv_heads;
    c->layer_stride = c->seq_stride * desc->n_seqs;
    *out = c;
    return LVX_OK;
}

extern "C" lvx_status_t lvx_kv4_destroy(lvx_kv4_t *cache) {
    LVX_REQUIRE(cache != nullptr, LVX_ERR_INVALID_ARG, "cache handle is NULL");
    delete cache;
    return LVX_OK;
}

extern "C" lvx_status_t lvx_kv4_append(lvx_kv4_t *cache, int32_t layer, const void *dev_k, const void *dev_v, int64_t ld, const int32_t *dev_starts,
                                       int32_t n_tokens, int32_t max_tokens, const int32_t *dev_key_counts, lvx_stream_t stream) {
    LVX_TRY(check_call(cache, layer, dev_starts, n_tokens, max_tokens, dev_key_counts));
    LVX_REQUIRE(dev_k != nullptr && dev_v != nullptr && lvx_aligned16(dev_k) && lvx_aligned16(dev_v), LVX_ERR_INVALID_ARG,
                "k or v is NULL or not 16-byte aligned");
    const lvx_kv4_desc_t &d = cache->desc;
    LVX_REQUIRE(ld >= (int64_t)d.n_kv_heads * d.head_dim && ld % 8 == 0, LVX_ERR_SHAPE, "row stride %lld must be a multiple of 8, at least %lld", (long long)ld,
                (long long)d.n_kv_heads * d.head_dim);
    if (n_tokens == 0) return LVX_OK;
    append_args_t p = {};
    p.base = cache->base + layer * cache->layer_stride;
    p.head_stride = cache->head_stride, p.seq_stride = cache->seq_stride;
    p.k = (const bf16_t *)dev_k, p.v = (const bf16_t *)dev_v, p.ld = ld;
    p.batch = {dev_starts, dev_key_counts, max_tokens, n_tokens};
    p.kv_heads = d.n_kv_heads, p.max_keys = d.max_keys;
    // max_tokens keys from any position on touch at most this many aligned groups; a wave takes two of eight keys where sequences bring that many
    const int64_t span = max_tokens < d.max_keys ? max_tokens : d.max_keys;
    const int per = max_tokens > 8 ? 16 : 8;
    const dim3 grid((unsigned)((span + 2 * per - 2) / per), d.n_seqs, (d.n_kv_heads + 3) / 4);
    auto *kernel = d.head_dim == 128 ? (per == 16 ? lvx_kv4_append_kernel<128, 2> : lvx_kv4_append_kernel<128, 1>)
                                     : (per == 16 ? lvx_kv4_append_kernel<64, 2> : lvx_kv4_append_kernel<64, 1>);
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, (hipStream_t)stream, p);
    LVX_CHECK_HIP(hipGetLastError());
    return LVX_OK;
}

extern "C" lvx_status_t lvx_kv4_gather(const lvx_kv4_t *cache, int32_t layer, int32_t first_key, int32_t n_keys, const int32_t *dev_key_counts,
                                       void *dev_k_out, void *dev_v_out, int64_t ld, lvx_stream_t stream) {
    LVX_TRY(check_call(cache, layer, nullptr, 0, 0, dev_key_counts));
    LVX_REQUIRE(dev_k_out != nullptr && dev_v_out != nullptr && lvx_aligned16(dev_k_out) && lvx_aligned16(dev_v_out), LVX_ERR_INVALID_ARG,
                "k or v is NULL or not 16-byte aligned");
    const lvx_kv4_desc_t &d = cache->desc;
    LVX_REQUIRE(first_key >= 0 && n_keys >= 0 && (int64_t)first_key + n_keys <= d.max_keys, LVX_ERR_SHAPE, "keys [%d, %lld) outside [0, %d)", first_key,
                (long long)first_key + n_keys, d.max_keys);
    LVX_REQUIRE(ld >= (int64_t)d.n_kv_heads * d.head_dim && ld % 8 == 0, LVX_ERR_SHAPE, "row stride %lld must be a multiple of 8, at least %lld", (long long)ld,
                (long long)d.n_kv_heads * d.head_dim);
    if (n_keys == 0) return LVX_OK;
    gather_args_t p = {};
    p.base = cache->base + layer * cache->layer_stride;
    p.head_stride = cache->head_stride, p.seq_stride = cache->seq_stride;
    p.k = (bf16_t *)dev_k_out, p.v = (bf16_t *)dev_v_out, p.ld = ld;
    p.counts = dev_key_counts;
    p.first_key = first_key, p.n_keys = n_keys, p.kv_heads = d.n_kv_heads, p.max_keys = d.max_keys;
    const int64_t items = ((int64_t)n_keys + 14) / 8 * d.n_kv_heads * (d.head_dim / 8);
    const dim3 grid((unsigned)(items < 256 * 4096 ? (items + 255) / 256 : 4096), d.n_seqs);
    if (d.head_dim == 128)
        hipLaunchKernelGGL(lvx_kv4_gather_kernel<128>, grid, dim3(256), 0, (hipStream_t)stream, p);
    else
        hipLaunchKernelGGL(lvx_kv4_gather_kernel<64>, grid, dim3(256), 0, (hipStream_t)stream, p);
    LVX_CHECK_HIP(hipGetLastError());
    return LVX_OK;
}

namespace {

template <int D>
void attn_launch(const lvx_kv4_plan_t &pl, const attn_args_t &p, dim3 grid, hipStream_t stream) {
    if (pl.rows == 16)
        hipLaunchKernelGGL((lvx_kv4_attention_kernel<D, 1, 1, 8>), grid, dim3(512), 0, stream, p);
    else if (pl.rows == 32)
        hipLaunchKernelGGL((lvx_kv4_attention_kernel<D, 2, 1, 8>), grid, dim3(512), 0, stream, p);
    else if (pl.rows == 64)
        hipLaunchKernelGGL((lvx_kv4_attention_kernel<D, 2, 2, 2>), grid, dim3(256), 0, stream, p);
    else
        hipLaunchKernelGGL((lvx_kv4_attention_kernel<D, 2, 4, 1>), grid, dim3(256), 0, stream, p);
}

// for the partial outputs of any call of up to max_tokens tokens a sequence
uint64_t attn_scratch(const lvx_kv4_desc_t &d, int n_heads, int max_tokens) {
    return lvx_kv4_partial_rows(d.n_seqs, d.max_keys, n_heads, max_tokens) * (4ull * d.head_dim + 8);
}

}  // namespace

extern "C" size_t lvx_kv4_attention_workspace_bytes(const lvx_kv4_t *cache, int32_t n_heads, int32_t max_tokens) {
    if (cache == nullptr || n_heads <= 0 || n_heads % cache->desc.n_kv_heads != 0 || max_tokens < 0) {
        lvx_fail(LVX_ERR_INVALID_ARG, "cache handle is NULL, heads %d are no positive multiple of the kv heads, or tokens %d are negative", n_heads, max_tokens);
        return 0;
    }
    const uint64_t n = attn_scratch(cache->desc, n_heads, max_tokens);
    return (size_t)(n > 256 ? n : 256);
}

extern "C" lvx_status_t lvx_kv4_attention(const lvx_kv4_t *cache, int32_t layer, const void *dev_q, int64_t ld_q, int32_t n_heads, const int32_t *dev_starts,
                                          int32_t n_tokens, int32_t max_tokens, const int32_t *dev_key_counts, int32_t causal, float scale, void *dev_out,
                                          int64_t ld_out, void *dev_workspace, size_t workspace_bytes, lvx_stream_t stream) {
    LVX_TRY(check_call(cache, layer, dev_starts, n_tokens, max_tokens, dev_key_counts));
    const lvx_kv4_desc_t &d = cache->desc;
    LVX_REQUIRE(dev_q != nullptr && dev_out != nullptr && dev_workspace != nullptr && lvx_aligned16(dev_q) && lvx_aligned16(dev_out) && lvx_aligned16(dev_workspace),
                LVX_ERR_INVALID_ARG, "q, out or workspace is NULL or not 16-byte aligned");
    LVX_REQUIRE(n_heads > 0 && n_heads % d.n_kv_heads == 0 && n_heads <= 65536, LVX_ERR_SHAPE, "heads %d are no multiple of the %d kv heads, or more than 65536",
                n_heads, d.n_kv_heads);
    LVX_REQUIRE(causal == 0 || causal == 1, LVX_ERR_INVALID_ARG, "causal must be 0 or 1");
    LVX_REQUIRE(ld_q >= (int64_t)n_heads * d.head_dim && ld_q % 8 == 0 && ld_out >= (int64_t)n_heads * d.head_dim && ld_out % 8 == 0, LVX_ERR_SHAPE,
                "row strides must be multiples of 8 and at least heads * head_dim");
    LVX_REQUIRE((int64_t)max_tokens * n_heads <= INT32_MAX / 2, LVX_ERR_SHAPE, "%d tokens of %d heads are too many rows", max_tokens, n_heads);
    if (n_tokens == 0) return LVX_OK;
    const lvx_kv4_plan_t pl = lvx_kv4_plan(d.n_seqs, d.n_kv_heads, d.max_keys, n_heads, max_tokens);
    LVX_REQUIRE(workspace_bytes >= attn_scratch(d, n_heads, max_tokens), LVX_ERR_SHAPE, "workspace of %zu bytes, %llu needed", workspace_bytes,
                (unsigned long long)attn_scratch(d, n_heads, max_tokens));
    const int64_t grid_x = (int64_t)pl.splits * pl.row_tiles * d.n_kv_heads;
    LVX_REQUIRE(grid_x <= INT32_MAX / 512, LVX_ERR_SHAPE, "%d tokens of %d heads are too many rows", max_tokens, n_heads);
    attn_args_t p = {};
    p.base = cache->base + layer * cache->layer_stride;
    p.head_stride = cache->head_stride, p.seq_stride = cache->seq_stride;
    p.q = (const bf16_t *)dev_q, p.out = (bf16_t *)dev_out, p.ld_q = ld_q, p.ld_out = ld_out;
    p.batch = {dev_starts, dev_key_counts, max_tokens, n_tokens};
    p.n_seqs = d.n_seqs, p.n_heads = n_heads, p.kv_heads = d.n_kv_heads, p.group = n_heads / d.n_kv_heads;
    p.max_keys = d.max_keys, p.causal = causal, p.splits = pl.splits, p.row_tiles = pl.row_tiles;
    p.scale_log2 = scale * LVX_LOG2E;
    p.part_o = (float *)dev_workspace;
    p.part_ml = (float2 *)(p.part_o + (size_t)pl.splits * n_tokens * n_heads * d.head_dim);
    const dim3 grid((unsigned)grid_x, d.n_seqs);
    d.head_dim == 128 ? attn_launch<128>(pl, p, grid, (hipStream_t)stream) : attn_launch<64>(pl, p, grid, (hipStream_t)stream);
    LVX_CHECK_HIP(hipGetLastError());
    if (pl.splits > 1) {
        const dim3 cgrid((unsigned)(((int64_t)max_tokens * n_heads + 3) / 4), d.n_seqs);
        if (d.head_dim == 128)
            hipLaunchKernelGGL(lvx_kv4_combine_kernel<128>, cgrid, dim3(256), 0, (hipStream_t)stream, p);
        else
            hipLaunchKernelGGL(lvx_kv4_combine_kernel<64>, cgrid, dim3(256), 0, (hipStream_t)stream, p);
        LVX_CHECK_HIP(hipGetLastError());
    }
    return LVX_OK;
}
