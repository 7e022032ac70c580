// Attention over a paged cache written out plainly (gfx950): one wavefront per query row of a head, exact running maximum, fp32
// weights, nothing but the keys that the row sees is touched (plain_row()).  The cross-check of the fast kernels
// (PEC_FLAG_SIMPLE_KERNEL).
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

__global__ __launch_bounds__(64) void paged_simple_kernel(const PagedAttnParams p) {
    const int lane = threadIdx.x;
    for (int64_t i = blockIdx.x; i < (int64_t)p.batch.total_q * p.n_q_heads; i += gridDim.x) {
        const int token = (int)(i / p.n_q_heads), head = (int)(i % p.n_q_heads);
        const int b = paged_owner(p.batch, token);
        if (b < 0) continue;     // a row behind the last sequence stays as it is
        const PagedSeq s = paged_seq(p.batch, b);
        const __bf16* q = p.q + token * p.q_stride + head * kHeadDim + 2 * lane;
        int end = s.len_k;
        if (p.causal) end = max(0, min(end, s.len_k - s.len_q + (token - s.q0) + 1));
        const PlainRow r = plain_row(p.cache, p.batch.table + (int64_t)b * p.batch.table_len, head / p.group, (float)q[0], (float)q[1],
                                     p.scale, 0, end);
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
