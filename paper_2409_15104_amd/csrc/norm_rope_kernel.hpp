// Norms of queries and keys per head, the rotation of positions, and the way of new keys and values into a paged cache (gfx950).
//
//   x' = x w / sqrt(mean(x^2) + eps)                      over the 128 dims of a head row, if there is a weight
//   (a, b) -> (a cos - b sin, b cos + a sin)              of the pairs (i, i + R / 2) or (2 i, 2 i + 1) of the first R dims
//
// all in fp32, rounded to bf16 once at the end.  Memory-bound: a head row is 256 bytes in and 256 out, so it is read once, by 16
// lanes with 16 bytes each, and everything is done in registers: the sum of squares by four row rotations (DPP), the pairs of
// the usual R = 128 by one more.  A wavefront keeps to one token and takes four head rows at a time: the token's angles are
// fetched once for all of them, and its place in the cache looked up once.
//
// The vector ALU comes close behind memory (a wavefront instruction for every 1 KiB holds up its SIMD for 4 cycles, and 6 TB/s
// are 1 KiB per compute unit every 100), so the norm's factor, which all of a row shares, is applied last, and the weights go into
// the token's angles: y = (x (w cos) + partner(x) (partner(w) sin)) / |x|, 24 operations per 8 values, and 1 / sqrt is one
// instruction (v_rsq_f32, 1 ulp).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "paged_common.hpp"
#include "paged_mx_common.hpp"

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
    PagedKv cache;                           // append only; of a cache in 4 bits the codes
    PagedBatch batch;
    unsigned char *k_scale, *v_scale;        // append to a cache in 4 bits only, as in PagedMx
    int64_t scale_page_b;
    uint32_t scale_head_b;
};

constexpr int kNormRopeThreads = 256;
constexpr int kNormRopeRow = 1 << 23;        // workgroups in a row of the grid: a dimension of a launch counts its threads in 32 bits
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
// TO: where the keys go, and the values with them: packed rows (no values), a paged cache, a paged cache in 4 bits.
enum { kToRows = 0, kToPages = 1, kToMxPages = 2 };

template <bool NORM, int PAIRS, int TO>
__global__ __launch_bounds__(kNormRopeThreads) void norm_rope_kernel(const NormRopeParams p) {
    constexpr bool APPEND = TO != kToRows, MX = TO == kToMxPages;
    const int lane = threadIdx.x & 63, c = lane & 15, sub = lane >> 4;
    const int64_t w = ((int64_t)blockIdx.y * kNormRopeRow + blockIdx.x) * (kNormRopeThreads / 64) +
                      __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int token = (int)(w / p.parts), part = (int)(w % p.parts);
    if (token >= p.tokens) return;
    // groups of four head rows: queries, keys, values
    const int q_quads = (p.n_q_heads + 3) / 4, k_quads = (p.n_kv_heads + 3) / 4, quads = q_quads + (APPEND ? 2 : 1) * k_quads;
    const int per_part = (quads + p.parts - 1) / p.parts, begin = part * per_part, end = min(quads, begin + per_part);
    // Groups requested ahead.  With a cache one: the lookups are a chain of three trips, which more wavefronts (fewer registers)
    // hide better; 5,300 tokens of 32 / 8 heads 37.2 us with two, 31.7 with one, without a cache 16,384 of 64 / 8 122 and 124.
    constexpr int kNormRopeAhead = APPEND ? 1 : 2;
    enum { Q, K, V };
    auto kind_of = [&](int i) { return i < q_quads ? Q : i < q_quads + k_quads ? K : V; };
    auto fetch = [&](int i) {
        u32x4 x = {0u, 0u, 0u, 0u};
        if (i >= end) return x;
        const int kind = kind_of(i), head = 4 * (i - (kind == Q ? 0 : kind == K ? q_quads : q_quads + k_quads)) + sub;
        const __bf16* const row = kind == Q ? p.q + token * p.q_stride : kind == K ? p.k + token * p.k_stride : p.v + token * p.v_stride;
        if (head < (kind == Q ? p.n_q_heads : p.n_kv_heads))
            x = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(row + head * kHeadDim + 8 * c));
        return x;
    };
    u32x4 ahead[kNormRopeAhead];
#pragma unroll
    for (int i = 0; i < kNormRopeAhead; ++i) ahead[i] = fetch(begin + i);

    // ---- the token's position, and its place in the cache
    int64_t at;
    unsigned char *k_slot = nullptr, *v_slot = nullptr;      // null: no place for it
    [[maybe_unused]] int64_t scale_off = 0;
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
                if constexpr (MX) scale_off = number * p.scale_page_b + (at & ((1 << p.cache.log_page) - 1)) + ((c >> 2) << p.cache.log_page);
            }
        }
    } else {
        at = p.positions ? (int64_t)p.positions[token] : p.pos0 + token;
    }

    // ---- angles: y[i] = x[i] cs[i] + partner(x)[i] sn[i], the signs in sn
    float cs[8], sn[8];
    int partner = lane, partner_dim = 8 * c;         // of the lane's first value (kPairsNext: the pairs sit inside a lane)
    const bool turns = PAIRS != kPairsNone && 8 * c < p.rotary;
    if constexpr (PAIRS != kPairsNone) {
        const int half = p.rotary >> 1;
        const float* row = p.table + max((int64_t)0, min(at, (int64_t)p.n_positions - 1)) * p.rotary;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            cs[i] = 1.f;
            sn[i] = 0.f;
        }
        if (turns) {
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
                partner_dim += upper ? -half : half;
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
        }
    }

    // ---- head rows, four at a time; the weights of their kind go into the angles
    constexpr float kSmallMean = 0x1p-100f;
    const bool small_eps = __builtin_bit_cast(uint32_t, p.eps) < __builtin_bit_cast(uint32_t, kSmallMean);      // (it is not negative)
    float a[8], b[8];
    bool normed = false;
    int kind_now = -1;
    for (int i0 = begin; i0 < end; i0 += kNormRopeAhead) {
#pragma unroll
        for (int j = 0; j < kNormRopeAhead; ++j) {
            const int i = i0 + j;
            if (i >= end) break;
            const u32x4 raw = ahead[j];
            ahead[j] = fetch(i + kNormRopeAhead);
            const int kind = kind_of(i), head = 4 * (i - (kind == Q ? 0 : kind == K ? q_quads : q_quads + k_quads)) + sub;
            u32x4 y = raw;
            if ((NORM || PAIRS != kPairsNone) && kind != V) {
                if (kind != kind_now) {
                    kind_now = kind;
                    const float* const weight = kind == Q ? p.q_weight : p.k_weight;
                    normed = NORM && weight != nullptr;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        a[e] = PAIRS == kPairsNone ? 1.f : cs[e];
                        b[e] = PAIRS == kPairsNone ? 0.f : sn[e];
                    }
                    if (NORM && normed) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            a[e] *= weight[8 * c + e];
                            if (PAIRS != kPairsNone) b[e] *= weight[PAIRS == kPairsNext ? 8 * c + (e ^ 1) : partner_dim + e];
                        }
                    }
                }
                float x[8];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[2 * e] = __builtin_bit_cast(float, raw[e] << 16);
                    x[2 * e + 1] = __builtin_bit_cast(float, raw[e] & 0xffff0000u);
                }
                float inv = 1.f;
                if (NORM && normed) {
                    auto mean = [&](float eps) {      // of the squares, and eps
                        float ss = 0.f;
#pragma unroll
                        for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], ss);
                        ss += row_rotated(ss, 8);
                        ss += row_rotated(ss, 4);
                        ss += row_rotated(ss, 2);
                        ss += row_rotated(ss, 1);
                        return fmaf(ss, 1.f / kHeadDim, eps);
                    };
                    float m = mean(p.eps);
                    if (small_eps) {      // rows whose squares may be too small for fp32, and their mean for v_rsq_f32, a factor larger
                        const float up = m < kSmallMean ? 1.f / kSmallMean : 1.f;
#pragma unroll
                        for (int e = 0; e < 8; ++e) x[e] *= up;
                        m = mean(p.eps * up * up);
                    }
                    inv = __builtin_amdgcn_rsqf(m);
                }
                float z[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    z[e] = x[e] * a[e];
                    if constexpr (PAIRS != kPairsNone) {
                        const float other = PAIRS == kPairsNext ? x[e ^ 1] : PAIRS == kPairsFar ? row_rotated(x[e], 8) : __shfl(x[e], partner);
                        // (a value that is not turned takes nothing of its partner, which may be infinite)
                        if (PAIRS == kPairsFar || turns) z[e] = fmaf(other, b[e], z[e]);
                    }
                    if (NORM) z[e] *= inv;
                }
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    y[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{z[2 * e], z[2 * e + 1]}, bf16x2));
            }
            if (head >= (kind == Q ? p.n_q_heads : p.n_kv_heads)) continue;
            if (kind == Q) {
                *reinterpret_cast<u32x4*>(p.q_out + ((int64_t)token * p.n_q_heads + head) * kHeadDim + 8 * c) = y;
            } else if (!APPEND) {
                *reinterpret_cast<u32x4*>(p.k_out + ((int64_t)token * p.n_kv_heads + head) * kHeadDim + 8 * c) = y;
            } else if constexpr (MX) {
                // Keys are rounded to bf16 before: what is held is what a cache of bf16 would be rounded to, whether a call norms
                // and rotates or pec_qk_norm_rope has done so.  A group's largest magnitude is two steps among four lanes; a lane
                // stores its four bytes of codes, one of four the scale byte.  6,060 tokens of 8 KV heads 11.5 us, 2.7 TB/s.
                unsigned char* const slot = kind == K ? k_slot : v_slot;
                const uint32_t byte = mx_scale_byte(mx_top_of_group(y));
                if (slot) {
                    *reinterpret_cast<uint32_t*>(slot + (int64_t)head * p.cache.head_b + 4 * c) = mx_codes(y, byte);
                    if ((c & 3) == 0) (kind == K ? p.k_scale : p.v_scale)[scale_off + (int64_t)head * p.scale_head_b] = (unsigned char)byte;
                }
            } else {
                unsigned char* const slot = kind == K ? k_slot : v_slot;
                if (slot) *reinterpret_cast<u32x4*>(slot + (int64_t)head * p.cache.head_b + 16 * c) = y;
            }
        }
    }
}

}  // namespace pec
