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

}  // namespace pec
