// Attention over a paged cache for sequences with few new tokens: decode steps, drafted tokens, short chunks (gfx950).
//
// Such a call reads each key and value once for a handful of query rows and is bound by memory, so the aim is an equal share of
// the bytes for every wavefront and requests on their way all the time.  A unit is up to 32 NT query rows that share a KV head:
// the (token, head of the group) pairs of a sequence, in this order, so that a group of 8 heads and 5 drafted tokens is one
// unit of 40 rows and its keys are read once.  All units' 32-key tiles, sequence by sequence, form one line for each KV head
// that is cut into equal spans, a wavefront of the chip for each; neighbouring wavefronts take the same span of neighbouring
// heads, so that whole token rows of the cache are read together.  The lengths are only known on the device, so every workgroup
// adds them up when it starts (a lane per sequence).  A wavefront walks its span on its own, without a workgroup barrier: tiles
// go from memory straight to LDS, K(j + S) requested as soon as the scores of tile j have read their stage, V(j + S) as soon as
// O += P V has, S stages each.  Where a span ends inside a unit the piece leaves its fp32 result in one of the wavefront's two slots
// (a span ends inside at most two units), and paged_merge_kernel merges the pieces of a unit by log-sum-exp.
//
// Pages: one load instruction moves four keys, and pages hold eight at least, so an instruction stays inside a page and takes
// its address from scalar registers.  The page numbers of the next tile are scalar loads a tile ahead: they count against
// lgkmcnt, which the LDS reads bring to zero anyway, and not against vmcnt, by which the tiles are waited for.
//
// NT = 1: eight wavefronts per workgroup, one stage.  NT = 2 (up to 64 rows): four wavefronts with 512 registers each, two stages
// (eight with one stage, and 256 registers, spill: 318 us in the place of 187 for the 24 sequences below).
//
// What bounds it, spans with their merge: memory, 4 sequences of 107,500 tokens, 64 / 8 heads (1.76 GB) 275 us, 6.4 TB/s, as a
// streaming read; 64 of 27 ... 7,400, 32 / 8 (450 MB) 83 us, of which the merge takes 6; 24 x 5 drafted tokens behind 10,350,
// 64 / 8, rows of two fragments (1.02 GB) 187 us, 5.7 TB/s while the spans run.  Units: latency, 4 of 540, 32 / 8 (9 MB), 10.2 us:
// three trips to memory, then up to three tiles of each wavefront one behind the other, and the join (11.7 as spans with a merge).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "paged_common.hpp"
#include "paged_simple_kernel.hpp"

namespace pec {

constexpr int kPagedWaves1 = 8, kPagedWaves2 = 4;     // wavefronts per workgroup of up to 32 and up to 64 rows a unit
constexpr int kStepTile = 32;
constexpr int kStepTileBytes = kStepTile * kRowBytes;
constexpr int kUnitsRow = 1 << 22;                     // workgroups in a row of the units' grid, whose dimensions count threads in 32 bits
constexpr int kPagedChunks = 1024;                     // sequences are added up 64 at a time: up to 65,536 of them

// Sums that stop at kTooMany: the host refuses calls of so many steps, but offsets that fall can make sequences overlap, and
// sums of overlapping ones anything.
constexpr int kTooMany = 0x7fffffff;
__device__ __forceinline__ int add_up(int x, int y) { return (int)min((uint32_t)x + (uint32_t)y, (uint32_t)kTooMany); }

// How a call's sequences are cut: R = 2^log_r rows a unit; a sequence has less than 2^31 rows.
struct StepCut {
    FastDiv group;
    int log_r, causal, most_rows;
    // keys that row tile `rt` of `s` walks, its steps (tiles of 32 keys, at least one), row tiles of s, steps of all of them
    __device__ __forceinline__ int keys(const PagedSeq& s, int rt) const {
        if (!causal) return s.len_k;
        const int last_row = min(s.len_q * group.d, (rt + 1) << log_r) - 1;
        return max(0, min(s.len_k, s.len_k - s.len_q + group.div(last_row) + 1));
    }
    __device__ __forceinline__ int tiles(const PagedSeq& s, int rt) const { return max(1, (keys(s, rt) + kStepTile - 1) / kStepTile); }
    __device__ __forceinline__ int row_tiles(const PagedSeq& s) const {
        const int rows = s.len_q * group.d;
        return rows > most_rows ? 0 : (int)((uint32_t)(rows + (1 << log_r) - 1) >> log_r);
    }
    __device__ __forceinline__ int all_tiles(const PagedSeq& s) const {
        const int n = row_tiles(s);
        int sum = 0;
        for (int rt = 0; rt < n; ++rt) sum = add_up(sum, tiles(s, rt));
        return sum;
    }
};
struct PagedStepParams {
    PagedAttnParams a;
    float* part_out;          // [spans][KV heads][2][32 NT][128]
    float* part_lse;          // [spans][KV heads][2][32 NT]
    int32_t* prefix;          // [batch + 2]: steps of a KV head ahead of each sequence, and of all of them; the least steps of a span
    FastDiv n_spans;          // of a KV head
    FastDiv kv_heads;
    int32_t unit_rows;        // rows of a unit, as far as the host knows
    StepCut cut;              // most_rows: sequences with more rows are not this launch's (0x7fffffff: all are)
};
__device__ __forceinline__ int wave_prefix(int x) {      // inclusive
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int y = __shfl_up(x, d);
        if (lane >= d) x = add_up(x, y);
    }
    return x;
}
// A KV head's line of `total` steps in equal spans of at least `least`: the first `extra` of them have len + 1 steps.
struct StepSpans {
    int total, len, extra;
    __device__ __forceinline__ StepSpans(int steps, const FastDiv& n_spans, int least) : total(steps), len(n_spans.div(steps)), extra(0) {
        if (len >= least) extra = steps - len * n_spans.d;
        else len = least;
    }
    __device__ __forceinline__ int start(int i) const { return (int)min((int64_t)total, (int64_t)i * len + min(i, extra)); }
    __device__ __forceinline__ int of(int step) const {       // the span that the step falls into
        const int head = extra * (len + 1);
        return step < head ? step / (len + 1) : extra + (step - head) / max(1, len);
    }
};
// Steps that a span should have at least: a step more takes its wavefront 1.3 us (a trip to memory), while the merge is the
// shorter the fewer pieces there are, 1 us for 128 of the longest unit's, a step each, and what all rows' pieces take through
// memory and back at 4 TB/s.  With one step per span 8 sequences x 7 tokens x 5 heads on 1,924 tokens took 33 us and one of
// 17,126 tokens of 2 KV heads 27.
__device__ __forceinline__ int least_span(int total, int longest, int n_kv_heads, int unit_rows) {
    const float merge_us = (float)longest * (1.f / 128.f) + (float)total * (float)(n_kv_heads * unit_rows) * (1.f / 3900.f);
    return max(1, (int)__builtin_amdgcn_sqrtf(merge_us * (1.f / 1.3f)));
}

// Sequences laid end to end, `value` of a sequence being its length on that line.  Up to 64 of them sit in the lanes of every
// wavefront; of more, `chunk_sum` (LDS) keeps the sums of 64 at a time, which the wavefronts share out among themselves.
template <int WAVES, class Value>
struct PagedLine {
    const PagedBatch& bt;
    const Value value;
    int32_t* const chunk_sum;
    const int n_chunks, lane;
    PagedSeq lanes;
    int own, upto, total;
    __device__ __forceinline__ PagedSeq load(int b) const {
        PagedSeq s{0, 0, 0};
        if (b < bt.batch) s = paged_seq(bt, b);
        return s;
    }
    __device__ __forceinline__ PagedLine(const PagedBatch& batch, Value v, int32_t* sums, int wave)
        : bt(batch), value(v), chunk_sum(sums), n_chunks((batch.batch + 63) >> 6), lane(threadIdx.x & 63) {
        lanes = load(lane);
        own = value(lanes);
        upto = wave_prefix(own);
        if (n_chunks <= 1) {
            total = __builtin_amdgcn_readlane(upto, 63);
            return;
        }
        for (int c = wave; c < n_chunks; c += WAVES) {
            const int sum = wave_prefix(value(load(64 * c + lane)));
            if (lane == 63) chunk_sum[c] = sum;
        }
        __syncthreads();
        int sum = 0;
        for (int c = lane; c < n_chunks; c += 64) sum = add_up(sum, chunk_sum[c]);
        total = __builtin_amdgcn_readlane(wave_prefix(sum), 63);
    }
    __device__ __forceinline__ PagedSeq seq(int i) const {       // uniform
        PagedSeq s;
        if (n_chunks <= 1) {
            s.q0 = __builtin_amdgcn_readlane(lanes.q0, i);
            s.len_q = __builtin_amdgcn_readlane(lanes.len_q, i);
            s.len_k = __builtin_amdgcn_readlane(lanes.len_k, i);
        } else {
            s = paged_seq(bt, i);
            s.q0 = __builtin_amdgcn_readfirstlane(s.q0);
            s.len_q = __builtin_amdgcn_readfirstlane(s.len_q);
            s.len_k = __builtin_amdgcn_readfirstlane(s.len_k);
        }
        return s;
    }
    // The sequence that point `at` < total falls into, `at` becoming its place there; -1: none (never, unless the offsets change
    // under the launch).
    __device__ __forceinline__ int find(int& at) {
        int c0 = 0;
        if (n_chunks > 1) {
            for (;; c0 += 64) {
                if (c0 >= n_chunks) return -1;
                const int sum = c0 + lane < n_chunks ? chunk_sum[c0 + lane] : 0, all = wave_prefix(sum);
                const uint64_t behind = __ballot(all > at);
                if (behind != 0) {
                    const int l = __builtin_ctzll(behind);
                    at -= __shfl(all, l) - __shfl(sum, l);
                    c0 += l;
                    break;
                }
                at -= __shfl(all, 63);
            }
            c0 = __builtin_amdgcn_readfirstlane(c0);
            own = value(load(64 * c0 + lane));
            upto = wave_prefix(own);
        }
        const uint64_t behind = __ballot(upto > at);
        if (behind == 0) return -1;
        const int l = __builtin_ctzll(behind);
        at = __builtin_amdgcn_readfirstlane(at - __builtin_amdgcn_readlane(upto, l) + __builtin_amdgcn_readlane(own, l));
        return 64 * c0 + l;
    }
};

// Two ways to share out the work.  Spans (SHARED = false), as above.  Units (SHARED = true), for calls that are small all over:
// a workgroup per unit, whose wavefronts take every WAVES-th of its tiles and join their results in LDS; no workspace and no
// second launch, but nothing evens out units of different lengths.
template <int NT, int WAVES, int S, bool SHARED>
__global__ __launch_bounds__(WAVES * 64, 1) void paged_step_kernel(const PagedStepParams p) {
    constexpr int R = 32 * NT;
    constexpr int LOADS = 8;                 // load instructions (1 KiB each) per matrix and tile
    constexpr int STRIDE = SHARED ? WAVES : 1;
    constexpr int kStageBytes = WAVES * S * 2 * kStepTileBytes;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[kStageBytes];
    __shared__ int32_t chunk_sum[kPagedChunks];
    __shared__ float joint[SHARED ? 3 * WAVES * 32 : 1];
    static_assert(!SHARED || kStageBytes >= WAVES * 32 * kHeadDim * (int)sizeof(float), "the wavefronts' O of 32 rows is joined there");
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    const int l32 = lane & 31, hl = lane >> 5;
    const int g = p.a.group, causal = p.a.causal;
    const StepCut& cut = p.cut;
    const PagedBatch& bt = p.a.batch;

    auto length = [&](const PagedSeq& s) {
        return SHARED ? cut.row_tiles(s) : cut.all_tiles(s);
    };
    PagedLine<WAVES, decltype(length)> line(bt, length, chunk_sum, wave);
    if (!SHARED && blockIdx.x == 0) {       // steps of a KV head ahead of every sequence, for the merge
        for (int c = wave, ahead = 0, at = 0; c < line.n_chunks; c += WAVES) {
            for (; at < c; ++at) ahead = add_up(ahead, chunk_sum[at]);
            const int mine = length(line.load(64 * c + lane)), all = wave_prefix(mine);
            if (64 * c + lane < bt.batch) p.prefix[64 * c + lane] = add_up(ahead, all) - mine;
        }
        if (threadIdx.x == 0) p.prefix[bt.batch] = line.total == kTooMany ? 0 : line.total;
    }
    if (line.total == 0 || line.total == kTooMany) return;
    int least = 1;
    if constexpr (!SHARED) {
        int longest = line.total / 64;       // (of more than 64 sequences: that many alike)
        if (line.n_chunks <= 1) {
            longest = cut.row_tiles(line.lanes) > 0 ? (line.lanes.len_k + kStepTile - 1) / kStepTile : 0;
#pragma unroll
            for (int off = 32; off > 0; off >>= 1) longest = max(longest, __shfl_xor(longest, off));
        }
        least = __builtin_amdgcn_readfirstlane(least_span(line.total, longest, p.a.n_kv_heads, p.unit_rows));
        if (blockIdx.x == 0 && threadIdx.x == 0) p.prefix[bt.batch + 1] = least;
    }
    int at, left, kvh, w = 0;               // place on the line, tiles to work on
    if constexpr (SHARED) {
        const WorkOrder order(line.total, 1, p.a.n_kv_heads);
        const uint32_t block = blockIdx.y * kUnitsRow + blockIdx.x;
        if ((block >> 3) >= order.count || order.total > (int64_t)gridDim.x * gridDim.y) return;      // (more units than the rows make: as above)
        const int64_t unit = order.unit(block & 7, block >> 3);
        if (unit < 0) return;
        kvh = __builtin_amdgcn_readfirstlane((int)unit / line.total);
        at = __builtin_amdgcn_readfirstlane((int)unit - kvh * line.total);
    } else {
        const StepSpans spans(line.total, p.n_spans, least);
        // Neighbouring heads and spans on neighbouring wavefronts of one XCD; but short spans on as many compute units as there
        // are, whose memory paths are what a few tiles take (4 sequences of 540 tokens 14.4 -> 11.7 us, while 4 of 107,000
        // would take 288 instead of 277).
        const int group_no = (int)(blockIdx.x & 7) * (int)(gridDim.x >> 3) + (int)(blockIdx.x >> 3);
        w = spans.len < 8 ? wave * (int)gridDim.x + (int)blockIdx.x : group_no * WAVES + wave;
        const int span = p.kv_heads.div(w);
        kvh = w - span * p.a.n_kv_heads;
        at = spans.start(span);
        left = span < p.n_spans.d ? spans.start(span + 1) - at : 0;
        if (left <= 0) return;
    }

    // Row tile `rt` of sequence `seq`; uniform.
    struct Unit {
        PagedSeq s;
        int seq, rt, row0, rows, keys, tiles;
    };
    auto unit_of = [&](const PagedSeq& s, int seq, int rt) {
        Unit u;
        u.s = s;
        u.seq = seq;
        u.rt = rt;
        u.row0 = rt * R;
        u.rows = min(R, s.len_q * g - u.row0);
        u.keys = cut.keys(s, rt);
        u.tiles = max(SHARED ? 0 : 1, (u.keys + kStepTile - 1) / kStepTile);
        return u;
    };
    auto next_unit = [&](const Unit& u) {
        PagedSeq s = u.s;
        int seq = u.seq, rt = u.rt + 1;
        while (rt >= cut.row_tiles(s)) {
            rt = 0;
            if (++seq >= bt.batch) {       // (never, unless the offsets change under the launch: what is left has no rows and no keys)
                seq = 0;
                s = PagedSeq{0, 0, 0};
                break;
            }
            s = line.seq(seq);
        }
        return unit_of(s, seq, rt);
    };
    Unit unit;
    int tile;
    {
        const int seq = __builtin_amdgcn_readfirstlane(line.find(at));
        if (seq < 0) return;
        at = __builtin_amdgcn_readfirstlane(at);
        const PagedSeq s = line.seq(seq);
        const int n_rt = cut.row_tiles(s);
        int rt = 0;
        if constexpr (SHARED) {
            rt = n_rt - 1 - at;              // the longest first
        } else {
            for (; rt < n_rt; ++rt) {
                const int n = cut.tiles(s, rt);
                if (at < n) break;
                at -= n;
            }
        }
        if (rt < 0 || rt >= n_rt) return;    // (never, as above)
        unit = unit_of(s, seq, rt);
        tile = SHARED ? wave : at;
        if constexpr (SHARED) left = max(0, (unit.tiles - wave + WAVES - 1) / WAVES);
    }

    // ---- lane constants of the tile loads and operand reads
    const PagedKv& cache = p.a.cache;
    const int ld_row = lane >> 4, ld_pos = lane & 15;
    uint32_t ldk[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) ldk[i] = (uint32_t)ld_row * cache.row_b + (uint32_t)(ld_pos ^ (4 * i + ld_row)) * 16u;
    const uint32_t ldv = (uint32_t)ld_row * cache.row_b + (uint32_t)((((ld_pos >> 2) ^ ld_row) << 2) | (ld_pos & 3)) * 16u;
    const uint32_t k_off0 = k_lds_off(l32, hl);
    uint32_t v_off[4];
    {
        const int gi = l32 & 15, gg = l32 >> 4;
#pragma unroll
        for (int dt = 0; dt < 4; ++dt) v_off[dt] = v_lds_off(4 * hl + (gi >> 2), dt * 64 + gg * 32 + (gi & 3) * 8);
    }
    unsigned char* const stages = lds + wave * S * 2 * kStepTileBytes;
    auto k_stage = [&](int j) { return stages + (j % S) * 2 * kStepTileBytes; };
    auto v_stage = [&](int j) { return stages + (j % S) * 2 * kStepTileBytes + kStepTileBytes; };
    const float sl2 = p.a.scale_log2;

    // ---- requests: the tile after the last requested one, S tiles ahead of the one worked on, in the same unit or a later one
    Unit req = unit;
    int req_tile = tile, req_left = left;
    const int64_t head_off = (int64_t)kvh * cache.head_b;
    uint32_t number[4];      // page numbers of its four groups of eight keys (of keys past the end: the last key's),
    int64_t off[4];          // and byte offsets of the groups
    auto look_up = [&]() {
        const ConstInts table = (ConstInts)(uintptr_t)(bt.table + (int64_t)req.seq * bt.table_len);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            number[i] = req.keys == 0 ? 0 : (uint32_t)table[min(req_tile * kStepTile + 8 * i, req.keys - 1) >> cache.log_page];
    };
    auto locate = [&]() {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t slot = (uint32_t)(req_tile * kStepTile + 8 * i) & ((1u << cache.log_page) - 1);
            off[i] = min(number[i], cache.last_page) * cache.page_b + (uint64_t)slot * cache.row_b + head_off;
        }
    };
    // Keys past the end come along, from the slots behind the last one or from whatever page is at hand: their scores are masked
    // and their values zeroed in LDS.
    auto issue = [&](const unsigned char* pool, bool is_v, unsigned char* stage) {
        const uint32_t l0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)stage;
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
            dma16_once(pool + off[i >> 1] + (i & 1) * 4 * (int64_t)cache.row_b, is_v ? ldv : ldk[i & 3], l0 + i * 1024);
    };
    auto request_k = [&](unsigned char* stage) {
        locate();
        issue(cache.k, false, stage);
    };
    auto request_v = [&](unsigned char* stage) {
        issue(cache.v, true, stage);
        if (--req_left == 0) return;
        req_tile += STRIDE;
        if (!SHARED && req_tile == req.tiles) {
            req = next_unit(req);
            req_tile = 0;
        }
        look_up();
    };
    if (req_left > 0) look_up();
    int n = 0;               // tiles behind this wavefront, which stage j % S goes by
#pragma unroll
    for (int i = 0; i < S; ++i)
        if (req_left > 0) {
            request_k(k_stage(i));
            request_v(v_stage(i));
        }

    for (;;) {
        // ---- a piece: tiles [tile, end) of the unit
        const int row0 = unit.row0, rows = unit.rows, keys = unit.keys, last = keys - 1;
        const int piece0 = tile, end = SHARED ? unit.tiles : min(unit.tiles, tile + left);
        const int first_vis = causal ? unit.s.len_k - unit.s.len_q + cut.group.div(row0) : last;       // last key of the first row
        int pos[NT], head[NT], last_vis[NT];      // new token, query head and last key of this lane's rows
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int r = row0 + nt * 32 + l32;
            pos[nt] = cut.group.div(r);
            head[nt] = kvh * g + r - pos[nt] * g;
            last_vis[nt] = causal ? min(last, unit.s.len_k - unit.s.len_q + pos[nt]) : last;
        }

        // ---- Q fragments: rows without a query stay zero and are not stored
        bf16x8 qf[NT][8];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const __bf16* qrow = p.a.q + (unit.s.q0 + pos[nt]) * p.a.q_stride + (int64_t)head[nt] * kHeadDim + 8 * hl;
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                u32x4 raw = {0u, 0u, 0u, 0u};
                if (nt * 32 + l32 < rows) raw = *reinterpret_cast<const u32x4*>(qrow + 16 * t);
                qf[nt][t] = __builtin_bit_cast(bf16x8, raw);
            }
        }
        f32x16 o[NT][4];
        float m_run[NT], l_run[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            m_run[nt] = -INFINITY;
            l_run[nt] = 0.f;
#pragma unroll
            for (int dt = 0; dt < 4; ++dt)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[nt][dt][r] = 0.f;
        }
        // Q is used here, so that the compiler waits for it here and not in the loop, where its wait would be one for the tiles
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int t = 0; t < 8; ++t) asm volatile("" : "+v"(qf[nt][t]));
        for (; tile < end; tile += STRIDE, ++n) {
            const int ahead = --left;           // tiles of the span behind this one
            const int key0 = tile * kStepTile;
            unsigned char *const kst = k_stage(n), *const vst = v_stage(n);
            // K(j): behind it V(j) and, with two stages, K(j + 1) V(j + 1) may be on their way
            if (S == 1 || ahead == 0) asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
            else asm volatile("s_waitcnt vmcnt(24)" ::: "memory");
            f32x16 s[NT];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[nt][r] = 0.f;
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                const bf16x8 kf = *reinterpret_cast<const bf16x8*>(kst + (k_off0 ^ (t << 5)));
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) s[nt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[nt][t], s[nt], 0, 0, 0);
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // the K stage has been read
            if (ahead >= S) request_k(kst);

            // mask, softmax reference (kept lazily: it moves only for a score more than 2^8 ahead of it), weights
            const bool need_mask = key0 + kStepTile - 1 > min(first_vis, last);
            bf16x8 pp[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                if (need_mask) {
                    const int lim = last_vis[nt] - key0 - 4 * hl;   // compare against 8*(r/4) + r%4
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (8 * (r >> 2) + (r & 3) > lim) s[nt][r] = -INFINITY;
                }
                float mx = s[nt][0];
#pragma unroll
                for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[nt][r]);
                {
                    const uint32_t u = __builtin_bit_cast(uint32_t, mx);
                    const auto sw = __builtin_amdgcn_permlane32_swap(u, u, false, false);
                    mx = fmaxf(__builtin_bit_cast(float, (uint32_t)sw[0]), __builtin_bit_cast(float, (uint32_t)sw[1]));
                }
                const float mx2 = mx * sl2;
                const float m_new = (mx2 > m_run[nt] + 8.f) ? mx2 : m_run[nt];
                const float m_use = (m_new == -INFINITY) ? 0.f : m_new;   // a row that has seen no key yet
                const float alpha = __builtin_amdgcn_exp2f(m_run[nt] - m_use);
                m_run[nt] = m_new;
                float rs = 0.f;
#pragma unroll
                for (int t2 = 0; t2 < 2; ++t2) {
                    u32x4 packed;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const f32x2 x = {__builtin_amdgcn_exp2f(fmaf(s[nt][8 * t2 + 2 * e], sl2, -m_use)),
                                         __builtin_amdgcn_exp2f(fmaf(s[nt][8 * t2 + 2 * e + 1], sl2, -m_use))};
                        // The denominator from the unrounded weights; for the product they are bf16, as everywhere here: the matrix
                        // instructions take them so (results are 2.2e-3 off in the 2-norm, with fp32 weights 1.7e-3, bf16 both)
                        rs += x[0] + x[1];
                        packed[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
                    }
                    pp[nt][t2] = __builtin_bit_cast(bf16x8, packed);
                }
                l_run[nt] = l_run[nt] * alpha + rs;
                if (__any(alpha != 1.f)) {
#pragma unroll
                    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
                        for (int r = 0; r < 16; ++r) o[nt][dt][r] *= alpha;
                }
            }

            // V(j): behind it, with two stages, K(j + 1) V(j + 1), and K(j + S) just asked for
            if (S == 1) {
                if (ahead >= 1) asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
                else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            } else {
                if (ahead >= 2) asm volatile("s_waitcnt vmcnt(24)" ::: "memory");
                else if (ahead == 1) asm volatile("s_waitcnt vmcnt(16)" ::: "memory");
                else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            }
            if (key0 + kStepTile > keys) {      // values past the end: zero
                const u32x4 z = {0u, 0u, 0u, 0u};
#pragma unroll
                for (int i = 0; i < LOADS; ++i)
                    if (key0 + 4 * i + ld_row >= keys) *reinterpret_cast<u32x4*>(vst + i * 1024 + lane * 16) = z;
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            }
            // A value that some of the rows do not see reaches them as 0 x value, which an infinite or NaN one is not.  In
            // tiles that hold such keys these values are added by hand to the rows that see them and zeroed for the product.
            if (min(key0 + kStepTile - 1, last) > first_vis) {
                unsigned char* const mine = vst + lane * 128;      // half a key row
                bool odd = false;
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    const u32x4 x = *reinterpret_cast<const u32x4*>(mine + 16 * c);
#pragma unroll
                    for (int e = 0; e < 4; ++e) odd |= (x[e] & 0x7f80u) == 0x7f80u || (x[e] & 0x7f800000u) == 0x7f800000u;
                }
                if (__any(odd)) {
                    for (int key = 0; key < kStepTile; ++key) {
                        const unsigned char* const row = vst + key * kRowBytes;
#pragma unroll
                        for (int dt = 0; dt < 4; ++dt)
#pragma unroll
                            for (int b = 0; b < 4; ++b) {
                                const int at = v_lds_off(key, 64 * dt + 16 * b + 8 * hl) - key * kRowBytes;
                                const bf16x4 x = *reinterpret_cast<const bf16x4*>(row + at);
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    const float y = (float)x[i];
                                    if (!__builtin_isfinite(y)) {
#pragma unroll
                                        for (int nt = 0; nt < NT; ++nt)
                                            if (key0 + key <= last_vis[nt]) o[nt][dt][4 * b + i] += y;
                                    }
                                }
                            }
                    }
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        u32x4 x = *reinterpret_cast<const u32x4*>(mine + 16 * c);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            if ((x[e] & 0x7f80u) == 0x7f80u) x[e] &= 0xffff0000u;
                            if ((x[e] & 0x7f800000u) == 0x7f800000u) x[e] &= 0xffffu;
                        }
                        *reinterpret_cast<u32x4*>(mine + 16 * c) = x;
                    }
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                }
            }
#pragma unroll
            for (int k2 = 0; k2 < 2; ++k2)
#pragma unroll
                for (int dt = 0; dt < 4; ++dt) {
                    const unsigned char* src = vst + v_off[dt] + k2 * 16 * kRowBytes;
                    const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) bf16x4*)(src));
                    const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
                        (__attribute__((address_space(3))) bf16x4*)(src + 8 * kRowBytes));
                    const bf16x8 vf = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) o[nt][dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pp[nt][k2], o[nt][dt], 0, 0, 0);
                }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // the V stage has been read
            if (ahead >= S) request_v(vst);
        }

        if constexpr (SHARED) {
            // ---- the wavefronts' results of every row are joined, 32 rows at a time.  O goes to LDS in 16-byte chunks of 4
            // dims, chunk c of row r at slot c * 32 + (r ^ c): the writers (fixed c, one row per lane) and the readers (fixed
            // row, one chunk per lane, so that a row leaves as one 256- or 512-byte run) touch all banks evenly.
            float *const join_m = joint, *const join_l = joint + WAVES * 32, *const join_w = joint + 2 * WAVES * 32;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                __syncthreads();
                const float l_tot = l_run[nt] + __shfl_xor(l_run[nt], 32);
                if (hl == 0) {
                    join_m[wave * 32 + l32] = m_run[nt];
                    join_l[wave * 32 + l32] = l_tot;
                }
                f32x4* const po = reinterpret_cast<f32x4*>(lds) + wave * 1024;
#pragma unroll
                for (int dt = 0; dt < 4; ++dt)
#pragma unroll
                    for (int b = 0; b < 4; ++b) {
                        const int c = 8 * dt + 2 * b + hl;
                        f32x4 x;
#pragma unroll
                        for (int i = 0; i < 4; ++i) x[i] = o[nt][dt][4 * b + i];
                        po[c * 32 + (l32 ^ c)] = x;
                    }
                __syncthreads();
                if (threadIdx.x < WAVES * 32) {   // one thread per (row, wavefront): the wavefront's weight
                    const int r = threadIdx.x & 31, k = threadIdx.x >> 5;
                    float mx = -INFINITY, den = 0.f;
#pragma unroll
                    for (int i = 0; i < WAVES; ++i) mx = fmaxf(mx, join_m[i * 32 + r]);
                    const float ref = mx == -INFINITY ? 0.f : mx;
#pragma unroll
                    for (int i = 0; i < WAVES; ++i) den += join_l[i * 32 + r] * __builtin_amdgcn_exp2f(join_m[i * 32 + r] - ref);
                    const float inv = den == 0.f ? 0.f : 1.f / den;
                    join_w[k * 32 + r] = __builtin_amdgcn_exp2f(join_m[k * 32 + r] - ref) * inv;
                    const int flat = row0 + nt * 32 + r, at_pos = cut.group.div(flat);
                    if (k == 0 && nt * 32 + r < rows)
                        p.a.lse[(int64_t)(kvh * g + flat - at_pos * g) * bt.total_q + unit.s.q0 + at_pos] =
                            den == 0.f ? -INFINITY : (mx + __builtin_amdgcn_logf(den)) * kLn2;      // NaN from NaN weights
                }
                __syncthreads();
                const int c = threadIdx.x & 31;
#pragma unroll
                for (int pass = 0; pass < 16 / WAVES; ++pass) {
                    const int r = pass * 2 * WAVES + (threadIdx.x >> 5), flat = row0 + nt * 32 + r, at_pos = cut.group.div(flat);
                    f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int k = 0; k < WAVES; ++k) {
                        const float wgt = join_w[k * 32 + r];
                        const f32x4 y = reinterpret_cast<const f32x4*>(lds)[k * 1024 + c * 32 + (r ^ c)];
#pragma unroll
                        for (int i = 0; i < 4; ++i) x[i] = fmaf(wgt, y[i], x[i]);
                    }
                    if (nt * 32 + r < rows) {
                        const int64_t idx = ((int64_t)(unit.s.q0 + at_pos) * p.a.n_q_heads + kvh * g + flat - at_pos * g) * kHeadDim + 4 * c;
                        if (p.a.out_f32) *reinterpret_cast<f32x4*>(static_cast<float*>(p.a.out) + idx) = x;
                        else *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(p.a.out) + idx) = __builtin_convertvector(x, bf16x4);
                    }
                }
            }
            return;
        }

        // ---- the unit's result, or the piece's into its slot
        const bool whole = piece0 == 0 && end == unit.tiles;
        const int64_t slot_row = (int64_t)(2 * w + (piece0 == 0 ? 1 : 0)) * R;      // of n_spans x KV heads x 2
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const float l_tot = l_run[nt] + __shfl_xor(l_run[nt], 32);
            if (nt * 32 + l32 < rows) {
                const int token = unit.s.q0 + pos[nt];
                const bool none = l_tot == 0.f || keys == 0;       // (without keys the values may be anything, and the sums NaN)
                const float inv = none ? 0.f : 1.f / l_tot;
                const float lse = none ? -INFINITY : (m_run[nt] + __builtin_amdgcn_logf(l_tot)) * kLn2;     // NaN from NaN weights
                if (hl == 0) {
                    if (whole) p.a.lse[(int64_t)head[nt] * bt.total_q + token] = lse;
                    else p.part_lse[slot_row + nt * 32 + l32] = lse;
                }
                const int64_t at = whole ? ((int64_t)token * p.a.n_q_heads + head[nt]) * kHeadDim : (slot_row + nt * 32 + l32) * kHeadDim;
                float* const dst = whole ? static_cast<float*>(p.a.out) : p.part_out;
#pragma unroll
                for (int dt = 0; dt < 4; ++dt)
#pragma unroll
                    for (int b = 0; b < 4; b += 2) {
                        f32x4 x, y;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            x[i] = none ? 0.f : o[nt][dt][4 * b + i] * inv;
                            y[i] = none ? 0.f : o[nt][dt][4 * b + 4 + i] * inv;
                        }
                        const int64_t idx = at + 32 * dt + 8 * b;
                        if (!whole || p.a.out_f32) {
                            *reinterpret_cast<f32x4*>(dst + idx + 4 * hl) = x;
                            *reinterpret_cast<f32x4*>(dst + idx + 8 + 4 * hl) = y;
                        } else {      // two groups of eight dims swapped between the wavefront's halves: 16 bytes per store
                            const u32x2 px = __builtin_bit_cast(u32x2, __builtin_convertvector(x, bf16x4));
                            const u32x2 py = __builtin_bit_cast(u32x2, __builtin_convertvector(y, bf16x4));
                            const auto s0 = __builtin_amdgcn_permlane32_swap(px[0], py[0], false, false);
                            const auto s1 = __builtin_amdgcn_permlane32_swap(px[1], py[1], false, false);
                            *reinterpret_cast<u32x4*>(static_cast<__bf16*>(p.a.out) + idx + 8 * hl) = u32x4{s0[0], s1[0], s0[1], s1[1]};
                        }
                    }
            }
        }
        if (left <= 0) return;
        unit = next_unit(unit);
        tile = 0;
    }
}

// Merges the pieces of units that spans have cut: O = sum_i O_i exp(lse_i - L), L = ln sum_i exp(lse_i).  A few KB per row, so
// trips to memory are all there is to it: a half wavefront per piece, four dims a lane, with a running maximum of its own, four
// pieces requested at once.  WAVES wavefronts share a row (a new token of a query head): one where there are rows for every
// wavefront of the chip, which leaves no barrier between them, four or sixteen where there are fewer and more pieces each.
// `tokens`: workgroups per sequence and query head (times four for WAVES = 1), which share its new tokens.
template <int WAVES>
__global__ __launch_bounds__(WAVES == 1 ? 256 : WAVES * 64) void paged_merge_kernel(const PagedStepParams p, int tokens) {
    constexpr int N = 2 * WAVES, AHEAD = 4;
    __shared__ __attribute__((aligned(16))) float red[N][kHeadDim];
    __shared__ float red_mx[N], red_den[N];
    const PagedBatch& bt = p.a.batch;
    const int g = p.a.group, head = blockIdx.y, kvh = p.cut.group.div(head), in_group = head - kvh * g, log_r = p.cut.log_r;
    const int grp = (int)(threadIdx.x >> 5) % N, c = threadIdx.x & 31;
    const int per_head = p.prefix[bt.batch], least = p.prefix[bt.batch + 1];
    constexpr int PER_GROUP = WAVES == 1 ? 4 : 1;       // rows a workgroup works on at a time
    for (int x = blockIdx.x * PER_GROUP + (WAVES == 1 ? (int)(threadIdx.x >> 6) : 0); x < bt.batch * tokens; x += gridDim.x * PER_GROUP) {
        const int seq = x / tokens;
        const PagedSeq s = paged_seq(bt, seq);
        const int before = p.prefix[seq], n_rt = p.cut.row_tiles(s);
        if (per_head == 0 || n_rt == 0) continue;
        const StepSpans spans(per_head, p.n_spans, least);
        int rt = 0, at = before;       // the row tile in hand, and its first step
        for (int pos = x % tokens; pos < s.len_q; pos += tokens) {
            const int flat = pos * g + in_group;
            for (; rt < flat >> log_r; ++rt) at += p.cut.tiles(s, rt);
            const int w0 = spans.of(at), w1 = spans.of(at + p.cut.tiles(s, rt) - 1);
            if (w0 == w1) continue;
            const int row = flat - (rt << log_r);
            float mx = -INFINITY, den = 0.f;
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
            for (int w = w0 + grp; w <= w1; w += AHEAD * N) {
                float l[AHEAD];
                f32x4 o[AHEAD];
#pragma unroll
                for (int i = 0; i < AHEAD; ++i) {
                    l[i] = -INFINITY;
                    o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
                    if (w + i * N <= w1) {
                        const int64_t slot = ((int64_t)(w + i * N) * p.a.n_kv_heads + kvh) * 2 + (w + i * N == w0 ? 1 : 0);
                        const int64_t slot_row = (slot << log_r) + row;
                        l[i] = p.part_lse[slot_row];
                        o[i] = *reinterpret_cast<const f32x4*>(p.part_out + slot_row * kHeadDim + 4 * c);
                    }
                }
                float top = mx;
#pragma unroll
                for (int i = 0; i < AHEAD; ++i) top = fmaxf(top, l[i]);      // (NaN: as if it were not there)
                const float ref = top == -INFINITY ? 0.f : top, alpha = expf(mx - ref);
                den *= alpha;
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[e] *= alpha;
#pragma unroll
                for (int i = 0; i < AHEAD; ++i) {
                    const float wgt = expf(l[i] - ref);
                    den += wgt;
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[e] = fmaf(wgt, o[i][e], acc[e]);
                }
                mx = top;
            }
            const int token = s.q0 + pos;
            const int64_t out_row = ((int64_t)token * p.a.n_q_heads + head) * kHeadDim, lse_at = (int64_t)head * bt.total_q + token;
            if constexpr (WAVES == 1) {
                const float other = __shfl_xor(mx, 32), top = fmaxf(mx, other), ref = top == -INFINITY ? 0.f : top;
                const float mine = expf(mx - ref);
                den *= mine;
                den += __shfl_xor(den, 32);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    acc[e] *= mine;
                    acc[e] += __shfl_xor(acc[e], 32);
                    if (den != 0.f) acc[e] /= den;
                }
                if (grp == 0) {
                    if (p.a.out_f32) *reinterpret_cast<f32x4*>(static_cast<float*>(p.a.out) + out_row + 4 * c) = acc;
                    else
                        *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(p.a.out) + out_row + 4 * c) = __builtin_convertvector(acc, bf16x4);
                    if (c == 0) p.a.lse[lse_at] = den == 0.f ? -INFINITY : ref + logf(den);
                }
            } else {
                __syncthreads();                     // the row before has been read
                *reinterpret_cast<f32x4*>(&red[grp][4 * c]) = acc;
                if (c == 0) {
                    red_mx[grp] = mx;
                    red_den[grp] = den;
                }
                __syncthreads();
                if (threadIdx.x < kHeadDim) {
                    float top = -INFINITY, a = 0.f, dn = 0.f;
#pragma unroll
                    for (int i = 0; i < N; ++i) top = fmaxf(top, red_mx[i]);
                    const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        const float wgt = expf(red_mx[i] - ref);
                        a = fmaf(wgt, red[i][threadIdx.x], a);
                        dn = fmaf(wgt, red_den[i], dn);
                    }
                    if (dn != 0.f) a /= dn;
                    if (p.a.out_f32) static_cast<float*>(p.a.out)[out_row + threadIdx.x] = a;
                    else static_cast<__bf16*>(p.a.out)[out_row + threadIdx.x] = (__bf16)a;
                    if (threadIdx.x == 0) p.a.lse[lse_at] = dn == 0.f ? -INFINITY : ref + logf(dn);
                }
            }
        }
    }
}

}  // namespace pec
