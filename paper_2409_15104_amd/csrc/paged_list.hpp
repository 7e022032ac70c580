// Work list of fwd_il_kernel<kFwdPaged>, built on the device from lengths that only the device knows, and the merge of the
// items' partial results.
//
// An item is a query tile (bm positions of a sequence, for the 256 / bm heads that share a workgroup) and a range of its keys.
// Few items would leave compute units idle, and so would a few more than a whole number per compute unit, so the keys are cut
// into ranges where the estimate below says so; ranges of a sequence start at the same keys for all of its tiles, and the list
// has them side by side, so that the workgroups of an XCD walk the same keys at the same time and find them in its L2.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "aux_kernels.hpp"
#include "paged_common.hpp"

namespace pec {

struct PagedSplit {      // a query tile whose keys are cut into ranges
    int32_t seq, qtile, slot0, n_ranges;
};
struct PagedListParams {
    PagedBatch batch;
    int32_t bm, log_bm, group, units, causal;        // positions per item; units of an item, over all KV heads
    int32_t few_rows;                        // sequences with at most so many rows per KV head are another launch's
    int32_t capacity, slot_capacity, cu;
    WorkItem* work;
    int32_t* counters;                       // [0] items, [2] split tiles, [8 .. 15] draw counters
    PagedSplit* splits;
};

constexpr int kPagedListSeqs = 1024, kPagedListBuckets = 1024;

// Keys that tile t of the sequence walks, and the first of its tiles that walks more than x.
struct PagedTiles {
    int n, len_q, len_k, log_bm, causal;
    __device__ __forceinline__ PagedTiles(const PagedSeq& s, const PagedListParams& p)
        : len_q(s.len_q), len_k(s.len_k), log_bm(p.log_bm), causal(p.causal) {
        n = len_q * p.group > p.few_rows ? (int)((uint32_t)(len_q + p.bm - 1) >> log_bm) : 0;      // (rows are below 2^31)
    }
    __device__ __forceinline__ int keys(int t) const { return causal ? max(0, len_k - len_q + min(len_q, (t + 1) << log_bm)) : len_k; }
    __device__ __forceinline__ int first_beyond(int x) const {
        if (len_k <= x) return n;
        const int y = x - (len_k - len_q);
        return causal && y > 0 ? min(n - 1, y >> log_bm) : 0;
    }
    // Items of all tiles with ranges of `range` keys, and how many tiles are not cut: this lane's share of the sum, the ranges
    // from number `first` on, every `step`-th.
    __device__ __forceinline__ int items(int range, int first, int step) const {
        int sum = first == 0 ? n : 0;
        for (int64_t x = (int64_t)range * (first == 0 ? step : first); x < len_k; x += (int64_t)range * step) sum += n - first_beyond((int)x);
        return sum;
    }
};

// Keys per range, as the smallest of sixteen estimates, one per wavefront; 0x40000000: no tile is cut.  In tile steps of 64
// keys: an item takes 8 besides its own (its first loads, its results), its partial results 4 more, and their merge with its
// launch 8 per call; items that are all alike run in whole rounds, others even out but for half an item at the end.
// SOME: of sequences in the area of a call on a cache in 4 bits, whose pages there take the place of their row of the block table.
template <bool SOME>
__global__ __launch_bounds__(1024) void paged_list_kernel(const PagedListParams p) {
    struct Seq {
        PagedSeq s;
        int n_items;
    };
    __shared__ Seq seqs[kPagedListSeqs];
    __shared__ int32_t bucket[kPagedListBuckets];
    __shared__ int32_t red[16], n_slots, n_split;
    __shared__ float cost[16];
    __shared__ int32_t cand[16];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const PagedBatch& bt = p.batch;
    if (tid == 0) n_slots = n_split = 0;
    if (tid >= 8 && tid < 16) p.counters[tid] = 0;

    // ---- the longest walk, then the estimates.  Up to 1,024 sequences are read once and stay in LDS.
    const bool held = bt.batch <= kPagedListSeqs;
    auto seq_at = [&](int b) { return held ? seqs[b].s : paged_seq<SOME>(bt, b); };
    // Lanes that share a sequence: of up to 64, as many as a wavefront has for each; above, one.
    int log_per = 0;
    while (bt.batch << log_per << 1 <= 64) ++log_per;
    const int per = 1 << log_per, sub = lane & (per - 1), mine = lane >> log_per;
    int longest = 0;
    for (int b = tid; b < bt.batch; b += 1024) {
        const PagedSeq s = paged_seq<SOME>(bt, b);
        if (held) seqs[b].s = s;
        const PagedTiles t(s, p);
        if (t.n > 0) longest = max(longest, t.keys(t.n - 1));
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) longest = max(longest, __shfl_xor(longest, off));
    if (lane == 0) red[wave] = longest;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 16; ++w) longest = max(longest, red[w]);
    const int whole = (longest + kBN - 1) / kBN;           // tile steps of the longest item
    {
        // candidates: the longest walk in 1, 2, 3, ... 8, 10, 12, 16, 20, 24, 32, 48, 64 ranges of at least 16 steps
        const int parts = wave < 8 ? wave + 1 : wave == 8 ? 10 : wave == 9 ? 12 : wave == 10 ? 16 : wave == 11 ? 20
                        : wave == 12 ? 24 : wave == 13 ? 32 : wave == 14 ? 48 : 64;
        const int steps = max(16, (whole + parts - 1) / parts), range = wave == 0 || p.slot_capacity == 0 ? 0x40000000 : steps * kBN;
        float items = 0.f, uncut = 0.f, tiles = 0.f, keys = 0.f;      // (whole numbers, exact up to 2^24 of them)
        for (int b = mine; b < bt.batch; b += 64 >> log_per) {
            const PagedTiles t(seq_at(b), p);
            if (t.n == 0) continue;
            items += (float)t.items(range, sub, per);
            if (sub != 0) continue;
            uncut += (float)t.first_beyond(range);
            tiles += (float)t.n;
            keys += ((float)t.keys(0) + (float)t.keys(t.n - 1)) * (float)t.n * 0.5f;
        }
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) {
            items += __shfl_xor(items, off);
            uncut += __shfl_xor(uncut, off);
            tiles += __shfl_xor(tiles, off);
            keys += __shfl_xor(keys, off);
        }
        // (offsets that fall make sequences overlap, and then there may be more tiles than the list has room for: no item at all)
        if (tiles > 1.001f * (p.capacity - p.slot_capacity)) {
            if (tid == 0) p.counters[0] = p.counters[2] = 0;
            return;
        }
        if (lane == 0) {
            const float cut = items - uncut;      // items with partial results
            const float units = (float)p.units, work = (keys / kBN + 0.5f * tiles + 8.f * items + 4.f * cut) * units / p.cu;
            const float one = (float)min(whole, range / kBN) + 8.f + (cut > 0.f ? 4.f : 0.f);
            const float rounds = ceilf(items * units / p.cu);
            float c = fmaxf(one, fminf(rounds * one, work + 0.5f * one)) + (cut > 0.f ? 8.f : 0.f);
            if (cut > p.slot_capacity) c = INFINITY;
            cost[wave] = c;
            cand[wave] = range;
        }
    }
    __syncthreads();
    int range;
    {
        float least = cost[lane & 15];
        int best = lane & 15;
#pragma unroll
        for (int off = 8; off > 0; off >>= 1) {
            const float other = __shfl_xor(least, off);
            const int its = __shfl_xor(best, off);
            if (other < least || (other == least && its < best)) {
                least = other;
                best = its;
            }
        }
        range = cand[__builtin_amdgcn_readfirstlane(best)];
    }

    // ---- items of sequence `b`, from place `pos0` of the list on: range by range, the last tile first
    auto place = [&](int b, const PagedSeq& sq, int pos0) {
        const PagedTiles t(sq, p);
        const int table_row = SOME ? bt.area[b] : b;
        for (int tile = lane; tile < t.n; tile += 64) {
            const int keys = t.keys(tile), n_ranges = max(1, (int)(((int64_t)keys + range - 1) / range));
            int slot0 = -1;
            if (n_ranges > 1) {
                slot0 = atomicAdd(&n_slots, n_ranges);
                if (slot0 + n_ranges > p.slot_capacity) slot0 = -1;      // (never, unless the offsets change under the launch)
                else p.splits[atomicAdd(&n_split, 1)] = PagedSplit{b, tile, slot0, n_ranges};
            }
            int pos = pos0 + t.n - 1 - tile;
            for (int r = 0; r < n_ranges; ++r) {
                if (r > 0) pos += t.n - (r == 1 ? 0 : t.first_beyond((r - 1) * range));
                const int key0 = r * range;
                if ((uint32_t)pos < (uint32_t)p.capacity)
                    p.work[pos] = WorkItem{sq.q0, sq.len_q, table_row, sq.len_k, tile, slot0 < 0 ? -1 : slot0 + r,
                                           {n_ranges > 1 ? key0 : 0, n_ranges > 1 ? min(keys, key0 + range) : keys}};
            }
        }
    };

    // ---- sequences by their longest walk.  Up to 64: a wavefront adds up for itself what is ahead of its ones, without a barrier.
    if (bt.batch <= 64) {
        int walk = -1, n_items = 0;
        if (mine < bt.batch) {
            const PagedTiles t(seqs[mine].s, p);
            if (t.n > 0) {
                walk = t.keys(t.n - 1);
                n_items = t.items(range, sub, per);
            }
        }
        for (int off = per >> 1; off > 0; off >>= 1) n_items += __shfl_xor(n_items, off);
        auto sum = [&](int x) {
            for (int off = 32; off >= per; off >>= 1) x += __shfl_xor(x, off);
            return x;
        };
        if (wave == 15) {       // (the least to do otherwise)
            const int total = sum(n_items);
            if (lane == 0) p.counters[0] = min(total, p.capacity);
        }
        for (int b = wave; b < bt.batch; b += 16) {
            if (__builtin_amdgcn_readlane(n_items, b << log_per) == 0) continue;
            const int its = __builtin_amdgcn_readlane(walk, b << log_per);
            place(b, seqs[b].s, sum(walk > its || (walk == its && mine < b) ? n_items : 0));
        }
        __syncthreads();
        if (tid == 0) p.counters[2] = n_split;
        return;
    }

    // ---- of more, by buckets of alike ones
    for (int t = tid; t < kPagedListBuckets; t += 1024) bucket[t] = 0;
    __syncthreads();
    auto load_seq = [&](int c0) {
        const int b = c0 + tid;
        if (b >= bt.batch) return;
        Seq q;
        q.s = held ? seqs[tid].s : paged_seq<SOME>(bt, b);
        const PagedTiles t(q.s, p);
        q.n_items = t.n > 0 ? t.items(range, 0, 1) : 0;
        seqs[tid] = q;
    };
    auto bucket_of = [&](const Seq& q) {
        const PagedTiles t(q.s, p);
        return t.n > 0 ? (int)min((int64_t)kPagedListBuckets - 1, (int64_t)t.keys(t.n - 1) * kPagedListBuckets / (longest + 1)) : 0;
    };
    for (int c0 = 0; c0 < bt.batch; c0 += kPagedListSeqs) {
        if (c0 > 0) __syncthreads();
        load_seq(c0);
        if (c0 + tid < bt.batch && seqs[tid].n_items > 0) atomicAdd(&bucket[bucket_of(seqs[tid])], seqs[tid].n_items);
    }
    __syncthreads();
    const int total = block_suffix_sum_1024(bucket, kPagedListBuckets, red);
    if (tid == 0) p.counters[0] = min(total, p.capacity);
    for (int c0 = 0; c0 < bt.batch; c0 += kPagedListSeqs) {
        if (bt.batch > kPagedListSeqs) {
            __syncthreads();
            load_seq(c0);
        }
        __shared__ int32_t pos0[kPagedListSeqs];
        if (c0 + tid < bt.batch && seqs[tid].n_items > 0) pos0[tid] = atomicAdd(&bucket[bucket_of(seqs[tid])], seqs[tid].n_items);
        __syncthreads();
        const int n = min(bt.batch - c0, kPagedListSeqs);
        for (int i = wave; i < n; i += 16) {
            if (seqs[i].n_items > 0) place(c0 + i, seqs[i].s, pos0[i]);
        }
    }
    __syncthreads();
    if (tid == 0) p.counters[2] = n_split;
}

// Merges the ranges of split tiles, a row per half wavefront, eight rows per workgroup at a time, four ranges requested at once.  A
// row is latency (28 ranges: seven trips), so rows are spread as wide as they go: 3 x 118 new tokens behind 30,000, 2 / 2 heads, 88 us
// per call with 32 rows per workgroup, 66 with eight.
__global__ __launch_bounds__(256) void paged_ranges_merge_kernel(const PagedListParams p, const float* part_out, const float* part_lse,
                                                                 int log_heads, int n_q_heads, int out_f32, void* out, float* lse) {
    constexpr int AHEAD = 4;
    const int n_split = p.counters[2], per_kvh = p.group >> log_heads, c = threadIdx.x & 31;
    for (int i = blockIdx.x; i < n_split * p.units * 32; i += gridDim.x) {      // (slots are few: this is far below 2^31)
        const int split = i / (p.units * 32), unit = (i >> 5) % p.units, row = (i & 31) * 8 + (threadIdx.x >> 5), strip = row >> 5;
        const int kvh = unit / per_kvh, u = unit - kvh * per_kvh;
        const int head = kvh * p.group + (u << log_heads) + (strip >> (3 - log_heads));
        const PagedSplit sp = p.splits[split];
        const PagedSeq s = paged_seq(p.batch, sp.seq);
        const int pos = sp.qtile * p.bm + ((strip << 5) & (p.bm - 1)) + (row & 31);
        if (pos >= s.len_q) continue;
        const int64_t first = ((int64_t)sp.slot0 * p.units + unit) * 256 + row, step = (int64_t)p.units * 256;
        float mx = -INFINITY, den = 0.f;
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
        for (int n0 = 0; n0 < sp.n_ranges; n0 += AHEAD) {
            float l[AHEAD];
            f32x4 o[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                l[k] = -INFINITY;
                o[k] = f32x4{0.f, 0.f, 0.f, 0.f};
                if (n0 + k < sp.n_ranges) {
                    const int64_t at = first + (n0 + k) * step;
                    l[k] = part_lse[at];
                    o[k] = *reinterpret_cast<const f32x4*>(part_out + at * kHeadDim + 4 * c);
                }
            }
            float top = mx;
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) top = fmaxf(top, l[k]);      // (NaN: as if it were not there)
            const float ref = top == -INFINITY ? 0.f : top, alpha = expf(mx - ref);
            den *= alpha;
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] *= alpha;
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const float w = expf(l[k] - ref);
                den += w;
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[e] = fmaf(w, o[k][e], acc[e]);
            }
            mx = top;
        }
        const float inv = den == 0.f ? 0.f : 1.f / den;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] *= inv;
        const int64_t token = s.q0 + pos, idx = (token * n_q_heads + head) * kHeadDim + 4 * c;
        if (out_f32) *reinterpret_cast<f32x4*>(static_cast<float*>(out) + idx) = acc;
        else *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(out) + idx) = __builtin_convertvector(acc, bf16x4);
        if (c == 0) lse[(int64_t)head * p.batch.total_q + token] = den == 0.f ? -INFINITY : mx + logf(den);
    }
}

}  // namespace pec
