// Sequences with many new tokens over a paged cache in 4 bits (gfx950): their keys and values are turned into bf16 once, in the call's
// workspace, and the pipelined kernel reads them there.
//
// A chunk's rows read every key many times (512 tokens of 4 heads to a KV head: eight workgroups of 256 rows), the conversion would be
// done as often, and the tile loop of fwd_il_kernel has neither a register nor an issue slot to spare for it.  Done once it is
// 136 bytes in and 512 out per key and KV head, memory-bound: 28,900 keys of 8 heads (156 MB) 34 us, 4.6 TB/s; the pages are dealt out
// in 4 us.  512 new tokens on them, 32 / 8 heads, take 260 us in all, straight from the codes 400.
//
// The area is a paged cache of its own, pages of 64 keys by heads; a sequence has consecutive pages, so its row of the block table is
// a stretch of one table that counts 0, 1, 2 ..., beginning at the sequence's first page.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "paged_mx_common.hpp"
#include "paged_step_kernel.hpp"

namespace pec {

constexpr int kMxAreaPage = 64;
constexpr int kMxAreaHeadBytes = kMxAreaPage * kRowBytes;      // of a page

struct MxAreaParams {
    PagedMx cache;
    PagedBatch batch;            // (area null: all sequences)
    int32_t capacity;            // pages
    int32_t n_kv_heads;
    int32_t* area;               // [batch] first page, -1: none
    int32_t* owner;              // [capacity] sequence of a page
    int32_t* table;              // [capacity + 1]
    int32_t* used;               // pages
    unsigned char *k, *v;        // [capacity][n_kv_heads][64][128] bf16
};

// Pages for the sequences, in their order, as long as there is room.
__global__ __launch_bounds__(1024) void paged_mx_area_kernel(const MxAreaParams p) {
    __shared__ int32_t sums[16], firsts[1024], counts[1024];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    int ahead = 0, used = 0;
    for (int b0 = 0; b0 < p.batch.batch; b0 += 1024) {
        const int b = b0 + tid;
        int pages = 0;
        bool many = false;
        if (b < p.batch.batch) {
            const PagedSeq s = paged_seq<true>(p.batch, b);
            many = s.len_q > 0;
            pages = many ? (s.len_k + kMxAreaPage - 1) / kMxAreaPage : 0;
        }
        const int upto = wave_prefix(pages);      // (sums stop at 2^31 - 1, which is no page of any area)
        if (lane == 63) sums[wave] = upto;
        __syncthreads();
        int before = ahead, all = ahead;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if (i == wave) before = all;
            all = add_up(all, sums[i]);
        }
        const int end = add_up(before, upto), first = end - pages;
        const bool fits = many && end <= p.capacity && before != kTooMany;
        if (b < p.batch.batch) p.area[b] = fits ? first : -1;
        firsts[tid] = first;
        counts[tid] = fits ? pages : 0;
        ahead = all;
        __syncthreads();
        for (int i = wave; i < min(1024, p.batch.batch - b0); i += 16) {
            const int n = counts[i], at = firsts[i];
            for (int x = lane; x < n; x += 64) {
                p.owner[at + x] = b0 + i;
                p.table[at + x] = at + x;
            }
            if (n > 0) used = max(used, at + n);
        }
        __syncthreads();
    }
    if (lane == 0) sums[wave] = used;
    __syncthreads();
    if (tid == 0) {
        for (int i = 0; i < 16; ++i) used = max(used, sums[i]);
        *p.used = used;
    }
}

// Codes into the area: a workgroup per page and KV head, four keys to a wavefront at a time, a lane takes eight dims.
__global__ __launch_bounds__(256) void paged_mx_fill_kernel(const MxAreaParams p) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, sub = lane >> 4;
    const int64_t units = (int64_t)min(*p.used, p.capacity) * p.n_kv_heads;
    for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
        const int page = (int)(unit / p.n_kv_heads), head = (int)(unit - (int64_t)page * p.n_kv_heads);
        const int b = p.owner[page];
        const int key0 = (page - p.area[b]) * kMxAreaPage + 16 * wave + sub, len_k = paged_seq(p.batch, b).len_k;
        const int32_t* const row = p.batch.table + (int64_t)b * p.batch.table_len;
        uint32_t codes[2][4], bytes[2][4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int key = min(key0 + 4 * r, len_k - 1), slot = key & ((1 << p.cache.log_page) - 1);
            const int64_t number = min((uint32_t)row[key >> p.cache.log_page], p.cache.last_page);
            const int64_t at = number * p.cache.page_b + (int64_t)slot * p.cache.row_b + (int64_t)head * p.cache.head_b + 4 * c;
            const int64_t scale_at = number * p.cache.scale_page_b + (int64_t)head * p.cache.scale_head_b + ((c >> 2) << p.cache.log_page) + slot;
            codes[0][r] = *reinterpret_cast<const uint32_t*>(p.cache.k + at);
            codes[1][r] = *reinterpret_cast<const uint32_t*>(p.cache.v + at);
            bytes[0][r] = p.cache.ks[scale_at];
            bytes[1][r] = p.cache.vs[scale_at];
        }
        const int64_t to = unit * kMxAreaHeadBytes + (16 * wave + sub) * kRowBytes + 16 * c;
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (key0 + 4 * r < len_k) {
                *reinterpret_cast<u32x4*>(p.k + to + 4 * r * kRowBytes) = mx_values(codes[0][r], mx_scale_of(bytes[0][r]));
                *reinterpret_cast<u32x4*>(p.v + to + 4 * r * kRowBytes) = mx_values(codes[1][r], mx_scale_of(bytes[1][r]));
            }
    }
}

}  // namespace pec
