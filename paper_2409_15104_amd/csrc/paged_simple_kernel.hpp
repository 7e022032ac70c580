// Attention over a paged cache written out plainly (gfx950): one wavefront per query row of a head, exact running maximum, fp32
// weights, nothing but the keys that the row sees is touched.  The cross-check of the fast kernels (PEC_FLAG_SIMPLE_KERNEL).
//
// In blocks of 64 keys: a lane per key for the scores (its key row read 16 bytes at a time, the query row from LDS), then two
// dims per lane for O += p V, the weights handed round.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "paged_common.hpp"

namespace pec {

struct PagedAttnParams {
    const __bf16* q;             // [total_q][n_q_heads][128], q_stride elements between tokens
    void* out;                   // [total_q][n_q_heads][128] bf16 or fp32
    float* lse;                  // [n_q_heads][total_q]
    int64_t q_stride;
    int32_t n_q_heads, n_kv_heads, group;
    int32_t causal, out_f32;
    float scale, scale_log2;     // scale_log2 = scale * log2(e)
    PagedKv cache;
    PagedBatch batch;
};

// O (two dims per lane) and LSE of one query row over keys [key0, key_end) of its sequence.  `q_row`: 128 floats in LDS.
struct PlainRow {
    float o0, o1, lse;
};
__device__ __forceinline__ PlainRow plain_row(const PagedKv& cache, const int32_t* table_row, int kvh, const float* q_row,
                                              float scale, int key0, int key_end) {
    const int lane = threadIdx.x & 63;
    const int64_t head_off = (int64_t)kvh * cache.head_b;
    auto row_of = [&](int key) {
        return page_in_cache(cache, table_row[key >> cache.log_page]) * cache.page_b +
               (key & ((1 << cache.log_page) - 1)) * (int64_t)cache.row_b + head_off;
    };
    float m = -INFINITY, den = 0.f, o0 = 0.f, o1 = 0.f;
    for (int k0 = key0; k0 < key_end; k0 += 64) {
        const int n = min(64, key_end - k0);
        float s = -INFINITY;
        if (lane < n) {
            const u32x4* row = reinterpret_cast<const u32x4*>(cache.k + row_of(k0 + lane));
            float dot = 0.f;
            for (int c = 0; c < 16; ++c) {
                const u32x4 x = row[c];
                for (int e = 0; e < 4; ++e) {
                    dot = fmaf(__builtin_bit_cast(float, x[e] << 16), q_row[8 * c + 2 * e], dot);
                    dot = fmaf(__builtin_bit_cast(float, x[e] & 0xffff0000u), q_row[8 * c + 2 * e + 1], dot);
                }
            }
            s = dot * scale;
        }
        float top = s;       // NaN is passed over here and comes back in with the weights
        for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
        const float m_new = fmaxf(m, top);
        const float ref = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = expf(m - ref);
        const float p = lane < n ? expf(s - ref) : 0.f;
        float sum = p;
        for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off);
        den = den * alpha + sum;
        o0 *= alpha;
        o1 *= alpha;
        for (int j = 0; j < n; ++j) {
            const float w = __shfl(p, j);
            const uint32_t x = reinterpret_cast<const uint32_t*>(cache.v + row_of(k0 + j))[lane];
            o0 = fmaf(w, __builtin_bit_cast(float, x << 16), o0);
            o1 = fmaf(w, __builtin_bit_cast(float, x & 0xffff0000u), o1);
        }
        m = m_new;
    }
    if (key_end <= key0) return PlainRow{0.f, 0.f, -INFINITY};
    const float inv = den == 0.f ? 0.f : 1.f / den;
    return PlainRow{o0 * inv, o1 * inv, den == 0.f ? -INFINITY : m + logf(den)};
}

__global__ __launch_bounds__(64) void paged_simple_kernel(const PagedAttnParams p) {
    __shared__ float q_row[kHeadDim];
    const int lane = threadIdx.x;
    for (int64_t i = blockIdx.x; i < (int64_t)p.batch.total_q * p.n_q_heads; i += gridDim.x) {
        const int token = (int)(i / p.n_q_heads), head = (int)(i % p.n_q_heads);
        const int b = paged_owner(p.batch, token);
        if (b < 0) continue;     // a row behind the last sequence stays as it is
        const PagedSeq s = paged_seq(p.batch, b);
        __syncthreads();
        const __bf16* q = p.q + token * p.q_stride + head * kHeadDim;
        q_row[2 * lane] = (float)q[2 * lane];
        q_row[2 * lane + 1] = (float)q[2 * lane + 1];
        __syncthreads();
        int end = s.len_k;
        if (p.causal) end = max(0, min(end, s.len_k - s.len_q + (token - s.q0) + 1));
        const PlainRow r = plain_row(p.cache, p.batch.table + (int64_t)b * p.batch.table_len, head / p.group, q_row, p.scale, 0, end);
        const int64_t at = ((int64_t)token * p.n_q_heads + head) * kHeadDim + 2 * lane;
        if (p.out_f32) {
            *reinterpret_cast<f32x2*>(static_cast<float*>(p.out) + at) = f32x2{r.o0, r.o1};
        } else {
            *reinterpret_cast<bf16x2*>(static_cast<__bf16*>(p.out) + at) = __builtin_convertvector(f32x2{r.o0, r.o1}, bf16x2);
        }
        if (lane == 0) p.lse[(int64_t)head * p.batch.total_q + token] = r.lse;
    }
}

}  // namespace pec
