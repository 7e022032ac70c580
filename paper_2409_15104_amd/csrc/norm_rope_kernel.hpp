// Norms of queries and keys per head, the rotation of positions, and the way of new keys and values into a paged cache (gfx950).
//
//   x' = x w / sqrt(mean(x^2) + eps)                      over the 128 dims of a head row, if there is a weight
//   (a, b) -> (a cos - b sin, b cos + a sin)              of the pairs (i, i + R / 2) or (2 i, 2 i + 1) of the first R dims
//
// all in fp32, rounded to bf16 once at the end.  Memory-bound: a head row is 256 bytes in and 256 out for 128 x 7 flop, so it is
// read once, by 16 lanes with 16 bytes each, and everything is done in registers: the sum of squares by four row rotations
// (DPP), the pairs of the usual R = 128 by one more.  A wavefront keeps to one token and takes four head rows at a time:
// the token's angles are fetched once for all of them, and its place in the cache looked up once.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "paged_common.hpp"

namespace pec {

struct NormRopeParams {
    const __bf16 *q, *k, *v;                 // [tokens][heads][128], strides in elements between tokens
    __bf16 *q_out, *k_out;                   // packed; k_out null: the keys go to the cache
    int64_t q_stride, k_stride, v_stride;
    const float *q_weight, *k_weight;        // [128] or null
    const float* table;                      // [n_positions][rotary]: cosines, then sines
    const int32_t* positions;                // or null: pos0 + token (without a cache)
    int64_t pos0;
    int32_t n_positions, rotary, interleaved;
    float eps;
    int32_t tokens, n_q_heads, n_kv_heads;   // n_q_heads 0: no queries
    int32_t parts;                           // wavefronts per token
    PagedKv cache;                           // append only
    PagedBatch batch;
};

constexpr int kNormRopeThreads = 256;
constexpr int kNormRopeAhead = 4;            // groups of four head rows requested together

__device__ __forceinline__ float row_rotated(float x, int ctrl) {     // 16 lanes rotated among themselves; ctrl is a constant
    switch (ctrl) {
        case 1: return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x121, 0xf, 0xf, true));
        case 2: return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x122, 0xf, 0xf, true));
        case 4: return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x124, 0xf, 0xf, true));
        default: return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x128, 0xf, 0xf, true));
    }
}

// PAIRS: which values a rotation combines: kPairsNone, kPairsFar (i, i + 64), kPairsHalf (i, i + R / 2) of any R, kPairsNext
// (2 i, 2 i + 1).
enum { kPairsNone = 0, kPairsFar = 1, kPairsHalf = 2, kPairsNext = 3 };

template <bool NORM, int PAIRS, bool APPEND>
__global__ __launch_bounds__(kNormRopeThreads) void norm_rope_kernel(const NormRopeParams p) {
    const int lane = threadIdx.x & 63, c = lane & 15, sub = lane >> 4;
    const int64_t w = (int64_t)blockIdx.x * (kNormRopeThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int token = (int)(w / p.parts), part = (int)(w % p.parts);
    if (token >= p.tokens) return;
    const int rows = p.n_q_heads + (APPEND ? 2 : 1) * p.n_kv_heads;
    const int quads = (rows + 3) / 4, per_part = (quads + p.parts - 1) / p.parts;
    const int quad_end = min(quads, (part + 1) * per_part);

    // where head row r of the token comes from (null: there is no such row)
    auto source = [&](int r) -> const __bf16* {
        if (r < p.n_q_heads) return p.q + token * p.q_stride + r * kHeadDim;
        r -= p.n_q_heads;
        if (r < p.n_kv_heads) return p.k + token * p.k_stride + r * kHeadDim;
        r -= p.n_kv_heads;
        if (APPEND && r < p.n_kv_heads) return p.v + token * p.v_stride + r * kHeadDim;
        return nullptr;
    };
    auto fetch = [&](int quad) {
        const __bf16* src = quad < quad_end ? source(4 * quad + sub) : nullptr;
        u32x4 x = {0u, 0u, 0u, 0u};
        if (src) x = *reinterpret_cast<const u32x4*>(src + 8 * c);
        return x;
    };
    u32x4 ahead[kNormRopeAhead];
#pragma unroll
    for (int i = 0; i < kNormRopeAhead; ++i) ahead[i] = fetch(part * per_part + i);

    // ---- the token's position, and its place in the cache
    int64_t at;
    unsigned char *k_slot = nullptr, *v_slot = nullptr;      // null: no place for it
    if constexpr (APPEND) {
        const int b = __builtin_amdgcn_readfirstlane(paged_owner(p.batch, token));
        if (b < 0) return;                                   // a row behind the last sequence
        const PagedSeq s = paged_seq(p.batch, b);
        at = (int64_t)s.len_k - s.len_q + (token - s.q0);
        if (at >= 0 && at < p.batch.max_keys) {
            const uint32_t number = (uint32_t)p.batch.table[(int64_t)b * p.batch.table_len + (at >> p.cache.log_page)];
            if (number <= p.cache.last_page) {
                const int64_t off = number * p.cache.page_b + (at & ((1 << p.cache.log_page) - 1)) * (int64_t)p.cache.row_b;
                k_slot = p.cache.k + off;
                v_slot = p.cache.v + off;
            }
        }
    } else {
        at = p.positions ? (int64_t)p.positions[token] : p.pos0 + token;
    }

    // ---- angles: y[i] = x[i] cs[i] + partner(x)[i] sn[i], the signs in sn
    float cs[8], sn[8];
    int partner = lane;
    if constexpr (PAIRS != kPairsNone) {
        const int half = p.rotary >> 1;
        const float* row = p.table + max((int64_t)0, min(at, (int64_t)p.n_positions - 1)) * p.rotary;
        if (8 * c < p.rotary) {
            if constexpr (PAIRS == kPairsNext) {
                const f32x4 co = *reinterpret_cast<const f32x4*>(row + 4 * c), si = *reinterpret_cast<const f32x4*>(row + half + 4 * c);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    cs[i] = co[i >> 1];
                    sn[i] = i & 1 ? si[i >> 1] : -si[i >> 1];
                }
            } else {
                const bool upper = 8 * c >= half;
                const float* col = row + 8 * c - (upper ? half : 0);
                partner = upper ? lane - half / 8 : lane + half / 8;
#pragma unroll
                for (int i = 0; i < 8; i += 4) {
                    const f32x4 co = *reinterpret_cast<const f32x4*>(col + i), si = *reinterpret_cast<const f32x4*>(col + half + i);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        cs[i + e] = co[e];
                        sn[i + e] = upper ? si[e] : -si[e];
                    }
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                cs[i] = 1.f;
                sn[i] = 0.f;
            }
        }
    }
    float qw[8], kw[8];
    if constexpr (NORM) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            qw[i] = p.q_weight ? p.q_weight[8 * c + i] : 1.f;
            kw[i] = p.k_weight ? p.k_weight[8 * c + i] : 1.f;
        }
    }

    // ---- head rows, four at a time
    for (int quad0 = part * per_part; quad0 < quad_end; quad0 += kNormRopeAhead) {
        u32x4 now[kNormRopeAhead];
#pragma unroll
        for (int i = 0; i < kNormRopeAhead; ++i) {
            now[i] = ahead[i];
            ahead[i] = fetch(quad0 + kNormRopeAhead + i);
        }
#pragma unroll
        for (int i = 0; i < kNormRopeAhead; ++i) {
            const int r = 4 * (quad0 + i) + sub;
            const bool is_q = r < p.n_q_heads, is_k = !is_q && r < p.n_q_heads + p.n_kv_heads;
            u32x4 y = now[i];
            if constexpr (NORM || PAIRS != kPairsNone) {
                float x[8];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[2 * e] = __builtin_bit_cast(float, now[i][e] << 16);
                    x[2 * e + 1] = __builtin_bit_cast(float, now[i][e] & 0xffff0000u);
                }
                if constexpr (NORM) {
                    float ss = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], ss);
                    ss += row_rotated(ss, 8);
                    ss += row_rotated(ss, 4);
                    ss += row_rotated(ss, 2);
                    ss += row_rotated(ss, 1);
                    const bool has = is_q ? p.q_weight != nullptr : p.k_weight != nullptr;
                    const float inv = has ? 1.f / sqrtf(fmaf(ss, 1.f / kHeadDim, p.eps)) : 1.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = x[e] * inv * (is_q ? qw[e] : kw[e]);
                }
                float z[8];
                if constexpr (PAIRS == kPairsNone) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) z[e] = x[e];
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float other = PAIRS == kPairsNext ? x[e ^ 1] : PAIRS == kPairsFar ? row_rotated(x[e], 8) : __shfl(x[e], partner);
                        z[e] = PAIRS == kPairsHalf && 8 * c >= p.rotary ? x[e] : fmaf(other, sn[e], x[e] * cs[e]);
                    }
                    if constexpr (PAIRS == kPairsNext) {
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (8 * c >= p.rotary) z[e] = x[e];      // (not x * 1 + y * 0: y may be infinite)
                    }
                }
                if (is_q || is_k) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        y[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{z[2 * e], z[2 * e + 1]}, bf16x2));
                }
            }
            if (quad0 + i >= quad_end || r >= rows) continue;
            if (is_q) {
                *reinterpret_cast<u32x4*>(p.q_out + ((int64_t)token * p.n_q_heads + r) * kHeadDim + 8 * c) = y;
            } else if (!APPEND) {
                *reinterpret_cast<u32x4*>(p.k_out + ((int64_t)token * p.n_kv_heads + r - p.n_q_heads) * kHeadDim + 8 * c) = y;
            } else {
                unsigned char* const slot = is_k ? k_slot : v_slot;
                const int h = r - p.n_q_heads - (is_k ? 0 : p.n_kv_heads);
                if (slot) *reinterpret_cast<u32x4*>(slot + (int64_t)h * p.cache.head_b + 16 * c) = y;
            }
        }
    }
}

}  // namespace pec
