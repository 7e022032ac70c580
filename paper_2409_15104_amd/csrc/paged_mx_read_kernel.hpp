// Tokens of a paged cache in 4 bits read back into packed bf16 rows (gfx950).
//
// Memory-bound: 68 bytes in and 256 out for a head row.  A wavefront takes four tokens, sixteen lanes each: four bytes of codes and
// the group's scale byte in, 16 bytes out per lane, so that every store is whole rows, marked as not read again soon.  4 x 22,800 tokens
// of 8 heads (495 MB, four fifths of it written) 109 us, 4.5 TB/s, where a copy of as much runs at 4.9 ... 5.4 (eight tokens to a
// wavefront 121 us, a quarter of the heads 118); 1,931 tokens 6.7 us.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "paged_mx_common.hpp"

namespace pec {

struct PagedMxReadParams {
    PagedMx cache;
    PagedBatch batch;
    __bf16 *k_out, *v_out;       // [tokens][n_kv_heads][128]
    int32_t n_kv_heads, parts;   // wavefronts that share four tokens' heads
};

constexpr int kMxReadRow = 1 << 23;          // workgroups in a row of the grid: a dimension of a launch counts its threads in 32 bits

__global__ __launch_bounds__(256) void paged_mx_read_kernel(const PagedMxReadParams p) {
    const int lane = threadIdx.x & 63, c = lane & 15, sub = lane >> 4;
    const int64_t w = ((int64_t)blockIdx.y * kMxReadRow + blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t first = w / p.parts * 4;
    const int part = (int)(w % p.parts);
    if (first >= p.batch.total_q) return;
    // ---- the four tokens' places; `there`: a token of a sequence, `held`: which has a page
    bool there = false, held = false;
    int64_t codes = 0, scales = 0;
    int owner = -1, end = 0;                 // of the sequence in hand
    for (int i = 0; i < 4; ++i) {
        const int token = (int)first + i;
        if (token >= p.batch.total_q) break;
        if (i == 0 || token >= end || owner < 0) owner = __builtin_amdgcn_readfirstlane(paged_owner(p.batch, token));
        if (owner < 0) continue;             // behind the last sequence
        const PagedSeq s = paged_seq(p.batch, owner);
        end = s.q0 + s.len_q;
        if (sub != i) continue;
        there = true;
        const int64_t at = (int64_t)s.len_k - s.len_q + (token - s.q0);
        if (at < 0 || at >= p.batch.max_keys) continue;
        const uint32_t number = (uint32_t)p.batch.table[(int64_t)owner * p.batch.table_len + (at >> p.cache.log_page)];
        if (number > p.cache.last_page) continue;
        held = true;
        const int slot = (int)at & ((1 << p.cache.log_page) - 1);
        codes = number * p.cache.page_b + (int64_t)slot * p.cache.row_b + 4 * c;
        scales = number * p.cache.scale_page_b + ((c >> 2) << p.cache.log_page) + slot;
    }
    if (!there) return;
    const int per = (2 * p.n_kv_heads + p.parts - 1) / p.parts, begin = part * per, stop = min(2 * p.n_kv_heads, begin + per);
    const int64_t row = (first + sub) * p.n_kv_heads;
#pragma unroll 4
    for (int i = begin; i < stop; ++i) {
        const bool is_v = i >= p.n_kv_heads;
        const int head = is_v ? i - p.n_kv_heads : i;
        u32x4 x = {0u, 0u, 0u, 0u};
        if (held) {
            const uint32_t raw = *reinterpret_cast<const uint32_t*>((is_v ? p.cache.v : p.cache.k) + codes + (int64_t)head * p.cache.head_b);
            const uint32_t byte = ((is_v ? p.cache.vs : p.cache.ks) + scales + (int64_t)head * p.cache.scale_head_b)[0];
            x = mx_values(raw, mx_scale_of(byte));
        }
        __builtin_nontemporal_store(x, reinterpret_cast<u32x4*>((is_v ? p.v_out : p.k_out) + (row + head) * kHeadDim + 8 * c));
    }
}

}  // namespace pec
