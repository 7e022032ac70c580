// Attention over a paged cache in 4 bits written out plainly (gfx950): one wavefront per query row of a head, exact running maximum,
// fp32 weights, nothing but the keys that the row sees is touched.  The cross-check of the fast kernels (PEC_FLAG_SIMPLE_KERNEL).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "paged_mx_common.hpp"
#include "paged_simple_kernel.hpp"

namespace pec {

__global__ __launch_bounds__(64) void paged_mx_simple_kernel(const PagedAttnParams p, const PagedMx cache) {
    const int lane = threadIdx.x;
    auto of_lane = [](float x, int l) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), l)); };
    for (int64_t i = blockIdx.x; i < (int64_t)p.batch.total_q * p.n_q_heads; i += gridDim.x) {
        const int token = (int)(i / p.n_q_heads), head = (int)(i % p.n_q_heads), kvh = head / p.group;
        const int b = paged_owner(p.batch, token);
        if (b < 0) continue;     // a row behind the last sequence stays as it is
        const PagedSeq s = paged_seq(p.batch, b);
        const int32_t* const table_row = p.batch.table + (int64_t)b * p.batch.table_len;
        const __bf16* q = p.q + token * p.q_stride + head * kHeadDim + 2 * lane;
        const float q0 = (float)q[0], q1 = (float)q[1];
        int end = s.len_k;
        if (p.causal) end = max(0, min(end, s.len_k - s.len_q + (token - s.q0) + 1));
        struct Place {
            int64_t codes, scales;
        };
        auto place = [&](int key) {
            const int64_t page = min((uint32_t)table_row[key >> cache.log_page], cache.last_page);
            const int slot = key & ((1 << cache.log_page) - 1);
            return Place{page * cache.page_b + (int64_t)slot * cache.row_b + (int64_t)kvh * cache.head_b,
                         page * cache.scale_page_b + (int64_t)kvh * cache.scale_head_b + slot};
        };
        float m = -INFINITY, den = 0.f, o0 = 0.f, o1 = 0.f;
        for (int k0 = 0; k0 < end; k0 += 64) {
            const int n = min(64, end - k0);
            const Place at = place(k0 + min(lane, n - 1));
            float dot = 0.f;
            for (int c = 0; c < 16; ++c) {
                const uint32_t codes = *reinterpret_cast<const uint32_t*>(cache.k + at.codes + 4 * c);
                const u32x4 x = mx_values(codes, mx_scale_of(cache.ks[at.scales + ((c >> 2) << cache.log_page)]));
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    dot = fmaf(__builtin_bit_cast(float, x[e] << 16), of_lane(q0, 4 * c + e), dot);
                    dot = fmaf(__builtin_bit_cast(float, x[e] & 0xffff0000u), of_lane(q1, 4 * c + e), dot);
                }
            }
            const float score = lane < n ? dot * p.scale : -INFINITY;
            float top = score;       // NaN is passed over here and comes back in with the weights
            for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
            const float m_new = fmaxf(m, top), ref = m_new == -INFINITY ? 0.f : m_new;
            const float alpha = expf(m - ref);
            const float w = lane < n ? expf(score - ref) : 0.f;
            float sum = w;
            for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off);
            den = den * alpha + sum;
            o0 *= alpha;
            o1 *= alpha;
            for (int j = 0; j < n; ++j) {
                const Place key = place(k0 + j);
                const uint32_t pair = cache.v[key.codes + lane];
                const float scale = mx_scale_of(cache.vs[key.scales + ((lane >> 4) << cache.log_page)]);
                const uint32_t x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(pair, scale, 0));
                const float wj = of_lane(w, j);
                o0 = fmaf(wj, __builtin_bit_cast(float, x << 16), o0);
                o1 = fmaf(wj, __builtin_bit_cast(float, x & 0xffff0000u), o1);
            }
            m = m_new;
        }
        const float inv = den == 0.f || end <= 0 ? 0.f : 1.f / den;
        const int64_t at = ((int64_t)token * p.n_q_heads + head) * kHeadDim + 2 * lane;
        const f32x2 o = {o0 * inv, o1 * inv};
        if (p.out_f32) *reinterpret_cast<f32x2*>(static_cast<float*>(p.out) + at) = o;
        else *reinterpret_cast<bf16x2*>(static_cast<__bf16*>(p.out) + at) = __builtin_convertvector(o, bf16x2);
        if (lane == 0) p.lse[(int64_t)head * p.batch.total_q + token] = den == 0.f ? -INFINITY : m + logf(den);
    }
}

}  // namespace pec
