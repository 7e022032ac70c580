// A key/value cache in pages and the batch whose sequences live in it (gfx950): what the paged kernels share.
//
// Token t of a sequence sits in slot t % page_size of the page that its row of the block table names at t / page_size.  The
// lengths and the table are device data that the host never sees, so every kernel bounds what it reads from them itself:
// offsets are clamped as in a colocated batch, lengths to what the table's rows hold, page numbers to the cache.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.hpp"

namespace pec {

typedef const __attribute__((address_space(4))) int32_t* ConstInts;   // read-only in a launch: scalar loads

// Division of numbers below 2^31 by one the host knows: a product and a shift (m = floor(2^(31 + l) / d) + 1, l = ceil(log2 d)) in
// the place of some thirty instructions.  The kernels of small calls are little but address arithmetic.
struct FastDiv {
    uint32_t m;
    int32_t shift, d;
    __host__ __device__ __forceinline__ int div(int x) const { return (int)((uint64_t)m * (uint32_t)x >> shift); }
};
inline FastDiv fast_div(int d) {
    int l = 0;
    while (((int64_t)1 << l) < d) ++l;
    return FastDiv{(uint32_t)(((uint64_t)1 << (31 + l)) / (uint64_t)d + 1), 31 + l, d};
}

struct PagedKv {
    unsigned char* k;            // element (page, slot, head, dim) at page_b * page + row_b * slot + head_b * head + 2 * dim bytes
    unsigned char* v;
    int64_t page_b;
    uint32_t row_b, head_b;      // less than 2^31 bytes inside a page
    uint32_t last_page;          // pages - 1
    int32_t log_page;            // log2 of the page size
};

struct PagedBatch {
    const int32_t* cu_q;         // [batch + 1]
    const int32_t* len_k;        // [batch], the new tokens among them
    const int32_t* table;        // [batch][table_len]
    int32_t batch, table_len, total_q;
    int32_t max_keys;            // table_len pages, at most 2^30 keys
};

struct PagedSeq {
    int32_t q0, len_q, len_k;
};
__device__ __forceinline__ PagedSeq paged_seq(const PagedBatch& b, int i) {
    PagedSeq s;
    s.q0 = min(max(b.cu_q[i], 0), b.total_q);
    s.len_q = min(max(b.cu_q[i + 1], s.q0), b.total_q) - s.q0;
    s.len_k = min(max(b.len_k[i], 0), b.max_keys);
    return s;
}

// Number of the page, inside the cache whatever the table says.
__device__ __forceinline__ uint32_t page_in_cache(const PagedKv& c, int32_t number) { return min((uint32_t)number, c.last_page); }

// O (two dims per lane) and LSE of one query row over keys [key0, key_end) of its sequence, written out plainly: fp32 weights, the
// exact running maximum, no key looked at that the row does not see.  In blocks of 64 keys: a lane per key for the scores, then
// two dims per lane for O += p V, the weights handed round.  q0, q1: the row's values 2 * lane and 2 * lane + 1.
struct PlainRow {
    float o0, o1, lse;
};
__device__ __forceinline__ PlainRow plain_row(const PagedKv& cache, const int32_t* table_row, int kvh, float q0, float q1,
                                              float scale, int key0, int key_end) {
    const int lane = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0));
    const int64_t head_off = (int64_t)kvh * cache.head_b;
    auto row_of = [&](int key) {
        return page_in_cache(cache, table_row[key >> cache.log_page]) * cache.page_b +
               (key & ((1 << cache.log_page) - 1)) * (int64_t)cache.row_b + head_off;
    };
    auto of_lane = [](float x, int l) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), l)); };
    float m = -INFINITY, den = 0.f, o0 = 0.f, o1 = 0.f;
    for (int k0 = key0; k0 < key_end; k0 += 64) {
        const int n = min(64, key_end - k0);
        const u32x4* const row = reinterpret_cast<const u32x4*>(cache.k + row_of(k0 + min(lane, n - 1)));
        float dot = 0.f;
        for (int c = 0; c < 16; ++c) {
            const u32x4 x = row[c];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                dot = fmaf(__builtin_bit_cast(float, x[e] << 16), of_lane(q0, 4 * c + e), dot);
                dot = fmaf(__builtin_bit_cast(float, x[e] & 0xffff0000u), of_lane(q1, 4 * c + e), dot);
            }
        }
        const float s = lane < n ? dot * scale : -INFINITY;
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
            const float w = of_lane(p, j);
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

// The sequence that owns packed row `token`, or -1.  Called by whole wavefronts with a uniform token: 64 offsets are looked at
// at a time, so 4,096 sequences take two trips to memory and not the twelve of a binary search.
__device__ __forceinline__ int paged_owner(const PagedBatch& b, int token) {
    const int lane = threadIdx.x & 63;
    int lo = 0, n = b.batch;       // the owner is the last sequence of lo ... lo + n - 1 that starts at or before the token
    while (n > 64) {
        const int step = (n + 63) / 64, at = lo + lane * step;
        const uint64_t before = __ballot(lane * step < n && b.cu_q[min(at, b.batch)] <= token);
        if (before == 0) return -1;
        const int l = 63 - __builtin_clzll(before);
        n = min(step, n - l * step);
        lo += l * step;
    }
    const int at = min(lo + lane, b.batch - 1);
    const int first = b.cu_q[at], end = b.cu_q[at + 1];
    const uint64_t mine = __ballot(lane < n && first <= token && token < end);     // (of empty sequences none)
    return mine == 0 ? -1 : lo + __builtin_ctzll(mine);
}

// The 32 query rows of a wavefront over keys [first, first + n_keys) of their sequence, row l32 over those up to its own last_vis (both
// counted from `first`), where keys behind first_vis -- not seen by all rows -- may have infinite or NaN values: these are zeros in
// the products and are added by hand to the rows that see them.  From memory straight to registers, without LDS and without a pause
// for the rest of its workgroup: a lane takes a key's row for the scores, and a dim of sixteen keys for O += V P.  5 us for 32 keys,
// latency, where plain_row() takes 20 for 64 keys of one row: 512 new tokens behind 30,000, a NaN in the last one's value, 71 -> 1.4 ms
// (0.26 without it).  o: dims 32 dt + 8 b + 4 hl + i of row l32 at [dt][4 b + i], divided by the sum of the weights.
__device__ __forceinline__ void rows_again(const PagedKv& cache, const int32_t* table_row, int kvh, const __bf16* qrow, bool valid, float sl2,
                                           int first, int n_keys, int first_vis, int last_vis, f32x16 (&o)[4]) {
    const int lane = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0)), l32 = lane & 31, hl = lane >> 5;
    bf16x8 qf[8];
#pragma unroll
    for (int t = 0; t < 8; ++t) {
        u32x4 raw = {0u, 0u, 0u, 0u};
        if (valid) raw = *reinterpret_cast<const u32x4*>(qrow + 16 * t + 8 * hl);
        qf[t] = __builtin_bit_cast(bf16x8, raw);
    }
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[dt][r] = 0.f;
    float m_run = -INFINITY, l_run = 0.f;
    for (int key0 = 0; key0 < n_keys; key0 += 32) {
        const int at = first + min(key0 + l32, n_keys - 1);
        const int64_t off = page_in_cache(cache, table_row[at >> cache.log_page]) * cache.page_b +
                            (at & ((1 << cache.log_page) - 1)) * (int64_t)cache.row_b + (int64_t)kvh * cache.head_b;
        f32x16 s;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            const bf16x8 kf = *reinterpret_cast<const bf16x8*>(cache.k + off + 32 * t + 16 * hl);
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[t], s, 0, 0, 0);
        }
        const int lim = min(last_vis, n_keys - 1) - key0 - 4 * hl;
        float mx = -INFINITY;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            if (8 * (r >> 2) + (r & 3) > lim) s[r] = -INFINITY;
            mx = fmaxf(mx, s[r]);
        }
        mx = fmaxf(mx, __shfl_xor(mx, 32)) * sl2;
        const float m_new = mx > m_run ? mx : m_run, m_use = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = __builtin_amdgcn_exp2f(m_run - m_use);
        m_run = m_new;
        l_run *= alpha;
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[dt][r] *= alpha;
        bool odd = false;
#pragma unroll
        for (int t2 = 0; t2 < 2; ++t2) {
            u32x4 packed;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const f32x2 x = {__builtin_amdgcn_exp2f(fmaf(s[8 * t2 + 2 * e], sl2, -m_use)),
                                 __builtin_amdgcn_exp2f(fmaf(s[8 * t2 + 2 * e + 1], sl2, -m_use))};
                l_run += x[0] + x[1];
                packed[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));      // (as in the other products)
            }
            const unsigned char* row[8];      // of the keys whose weights this lane holds
            bool past[8], some[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int j = 16 * t2 + 8 * (i >> 2) + 4 * hl + (i & 3);
                const uint32_t lo = __shfl((int)(uint32_t)off, j), hi = __shfl((int)(off >> 32), j);
                row[i] = cache.v + (int64_t)((uint64_t)hi << 32 | lo) + 2 * l32;
                past[i] = key0 + j >= n_keys;
                some[i] = key0 + j > first_vis;
            }
#pragma unroll
            for (int dt = 0; dt < 4; ++dt) {
                uint16_t x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = *reinterpret_cast<const uint16_t*>(row[i] + 64 * dt);
                u32x4 vf;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const bool out = (x[i] & 0x7f80u) == 0x7f80u && some[i];
                    odd |= out && !past[i];
                    const uint32_t y = past[i] || out ? 0u : x[i];
                    if (i & 1) vf[i >> 1] |= y << 16;
                    else vf[i >> 1] = y;
                }
                o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf), __builtin_bit_cast(bf16x8, packed), o[dt], 0, 0, 0);
            }
        }
        if (__any(odd)) {
            for (int j = max(0, first_vis + 1 - key0); j < min(32, n_keys - key0); ++j) {
                const uint32_t lo = __shfl((int)(uint32_t)off, j), hi = __shfl((int)(off >> 32), j);
                const unsigned char* const vrow = cache.v + (int64_t)((uint64_t)hi << 32 | lo) + 8 * hl;
#pragma unroll
                for (int dt = 0; dt < 4; ++dt)
#pragma unroll
                    for (int b = 0; b < 4; ++b) {
                        const bf16x4 x = *reinterpret_cast<const bf16x4*>(vrow + 64 * dt + 16 * b);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float y = (float)x[i];
                            if (!__builtin_isfinite(y) && key0 + j <= last_vis) o[dt][4 * b + i] += y;
                        }
                    }
            }
        }
    }
    const float l_tot = l_run + __shfl_xor(l_run, 32), inv = l_tot == 0.f ? 0.f : 1.f / l_tot;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[dt][r] = n_keys > 0 ? o[dt][r] * inv : 0.f;
}

}  // namespace pec
