// Attention over a paged cache in 4 bits for sequences with few new tokens: decode steps, drafted tokens, short chunks (gfx950).
//
// Units, lines and spans as in paged_step_kernel: a unit is up to R query rows that share a KV head, the units' 32-key tiles are one line
// for each KV head, cut into equal spans; pieces of units are merged by paged_merge_kernel.  Or, for small calls, a workgroup takes
// a unit, and nothing is left to merge.  Two things differ.  In 4 bits a tile is 4.25 KiB in the place of 16, so it goes from memory
// straight to registers, a tile ahead, with no LDS and no wait but the compiler's; and since a byte stands for two values, what
// is done per tile and what a piece's fp32 result costs count four times as much.  So a span belongs to a workgroup: its
// wavefronts take the tiles in turn and join their results in LDS, and a quarter as many pieces go through memory (with a span
// for every wavefront 24 x 5 drafted tokens behind 10,000 wrote and read 47 MB of them beside 280 MB of cache: 111 us).
//
// Products are 16 x 16 x 32 (lane l: m = l % 16, c = l / 16; A rows m, B columns m, k-slots 8 c ... 8 c + 7; C column m, rows 4 c + i).
// Scores, S^T = K Q^T: the contraction runs over dims in any order that K and Q agree on, so lane (m, c) takes dims 32 c ... 32 c + 31
// of key m, 16 bytes of codes in one load and exactly one scale group, eight dims for each of four products.  Of the tile's two
// halves of 16 keys lane c ends up with the scores of keys 4 c + i and 16 + 4 c + i, which are its eight k-slots of
// O^T += V^T P^T.  There row m of block j is dim 8 m + j: a lane needs of each of its eight keys the four bytes of dims
// 8 m ... 8 m + 7, converts them in pairs of dims and exchanges halves between neighbouring keys, two instructions for two values.
// Every load instruction stays inside 16 keys, so with pages of 16 keys and more its page is a scalar base and nothing about it is
// worked out per lane; pages of eight take a path of their own (SMALL).
//
// Weights are rounded to bf16 once, for their product with the values, as everywhere here; scores, sums, results and their merge are fp32.
//
// What bounds it: by heads memory, 4 sequences of 107,500 tokens, 64 / 8 heads (488 MB) 85 us with the merge, 120 of 3,300, 32 / 8 (435
// MB) 89, 5.2 TB/s while the spans run, where the loads alone take 82; by token half cache lines, 105 us for the former.  24 x 5 drafted tokens on
// 10,350, 64 / 8 heads, 48 rows: 81 us by heads, 89 by token, two wavefronts to a SIMD, each a chain of products, softmax, conversions
// and products.  270 instructions of the vector ALU and 48 matrix products for a tile keep the one busy for half of the time and the other
// for 28 %; of a wavefront's time 30 % goes for data that are not there and 31 % for its turn.  640 new tokens behind 1,000, 32 / 8, in
// units: 27 us.  4 of 540 in units: 8 us, latency.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "paged_mx_common.hpp"
#include "paged_step_kernel.hpp"

namespace pec {

// Steps that a span should have at least, as least_span(), a step taking its wavefront 0.6 us.
__device__ __forceinline__ int least_span_mx(int total, int longest, int n_kv_heads, int unit_rows) {
    const float merge_us = (float)longest * (1.f / 128.f) + (float)total * (float)(n_kv_heads * unit_rows) * (1.f / 3900.f);
    return max(1, (int)__builtin_amdgcn_sqrtf(merge_us * (1.f / 0.6f)));
}

// How a call's sequences are cut: R = 16, 32 or 48 rows a unit; as StepCut.
struct MxCut {
    static constexpr bool kSome = true;
    FastDiv group, rows;
    int causal;
    __device__ __forceinline__ int tile_of(int row) const { return rows.div(row); }
    __device__ __forceinline__ int64_t first_row(int64_t rt) const { return rt * rows.d; }
    __device__ __forceinline__ int keys(const PagedSeq& s, int rt) const {
        if (!causal) return s.len_k;
        const int last_row = min(s.len_q * group.d, (rt + 1) * rows.d) - 1;
        return max(0, min(s.len_k, s.len_k - s.len_q + group.div(last_row) + 1));
    }
    __device__ __forceinline__ int tiles(const PagedSeq& s, int rt) const { return max(1, (keys(s, rt) + kStepTile - 1) / kStepTile); }
    __device__ __forceinline__ int row_tiles(const PagedSeq& s) const { return rows.div(s.len_q * group.d + rows.d - 1); }
    __device__ __forceinline__ int all_tiles(const PagedSeq& s) const {
        const int n = row_tiles(s);
        int sum = 0;
        for (int rt = 0; rt < n; ++rt) sum = add_up(sum, tiles(s, rt));
        return sum;
    }
};
using PagedMxStepParams = PagedStepParamsOf<MxCut>;

constexpr float kNoKey = -0x1.fffffep127f;

struct MxTile {              // 32 keys, as lane (m, c) takes them
    u32x4 k[2];              // dims 32 c ... 32 c + 31 of key 16 u + m
    uint32_t v[8];           // dims 8 m ... 8 m + 7 of keys 16 u + 4 c + i at [4 u + i]
    uint32_t ks[2], vs[2];   // the scale byte of key 16 u + m for group c, those of keys 16 u + 4 c ... + 3 for group m / 4
};

// NT: row tiles of 16 to a unit.  WAVES: wavefronts of a span.  HEADS: KV heads whose spans share a workgroup: two where neighbouring
// heads' rows of a token lie side by side, 64 bytes each, half a cache line, which the compute unit then fetches once.  UNITS: a unit
// in the place of a span.  SMALL: pages of eight keys.
template <int NT, int WAVES, int HEADS, bool UNITS, bool SMALL>
__global__ __launch_bounds__(HEADS * WAVES * 64, 2) void paged_mx_step_kernel(const PagedMxStepParams p, const PagedMx cache) {
    constexpr int R = 16 * NT;
    constexpr bool QLDS = NT > 2;
    __shared__ __attribute__((aligned(1024))) float joint_all[HEADS][WAVES > 1 ? WAVES * 16 * kHeadDim : 1];
    __shared__ float joint_sums[HEADS][3 * WAVES * 16];
    __shared__ u32x4 lds_q[HEADS][QLDS ? NT * 4 * 64 : 1];
    __shared__ int32_t chunk_sum[kPagedChunks];
    const int wave_no = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), side = wave_no / WAVES, wave = wave_no % WAVES;
    const int lane = threadIdx.x & 63, m = lane & 15, c = lane >> 4, tid = threadIdx.x % (WAVES * 64);
    float *const joint_o = joint_all[side], *const joint = joint_sums[side];
    const int g = p.a.group, causal = p.a.causal;
    const MxCut& cut = p.cut;
    const PagedBatch& bt = p.a.batch;

    auto length = [&](const PagedSeq& s) { return UNITS ? cut.row_tiles(s) : cut.all_tiles(s); };
    PagedLine<HEADS * WAVES, true, decltype(length)> line(bt, length, chunk_sum, wave_no);
    if (!UNITS && blockIdx.x == 0) {       // steps of a KV head ahead of every sequence, for the merge
        for (int ch = wave_no, ahead = 0, at = 0; ch < line.n_chunks; ch += HEADS * WAVES) {
            for (; at < ch; ++at) ahead = add_up(ahead, chunk_sum[at]);
            const int mine = length(line.load(64 * ch + lane)), all = wave_prefix(mine);
            if (64 * ch + lane < bt.batch) p.prefix[64 * ch + lane] = add_up(ahead, all) - mine;
        }
        if (threadIdx.x == 0) p.prefix[bt.batch] = line.total == kTooMany ? 0 : line.total;
    }
    if (line.total == 0 || line.total == kTooMany) return;
    int least = 1;
    if constexpr (!UNITS) {
        int longest = line.total / 64;       // (of more than 64 sequences: that many alike)
        if (line.n_chunks <= 1) {
            longest = cut.row_tiles(line.lanes) > 0 ? (line.lanes.len_k + kStepTile - 1) / kStepTile : 0;
#pragma unroll
            for (int off = 32; off > 0; off >>= 1) longest = max(longest, __shfl_xor(longest, off));
        }
        least = __builtin_amdgcn_readfirstlane(least_span_mx(line.total, longest, p.a.n_kv_heads, p.unit_rows));
        if (blockIdx.x == 0 && threadIdx.x == 0) p.prefix[bt.batch + 1] = least;
    }
    int at, len, kvh, w = 0;                // place on the line, tiles from there on; slots are numbered 2 w, 2 w + 1
    if constexpr (UNITS) {
        const WorkOrder order(line.total, 1, p.kv_heads.d);
        const uint32_t block = blockIdx.y * kUnitsRow + blockIdx.x;
        if ((block >> 3) >= order.count || order.total > (int64_t)gridDim.x * gridDim.y) return;      // (more units than the rows make: as in paged_step_kernel)
        const int64_t unit = order.unit(block & 7, block >> 3);
        if (unit < 0) return;
        kvh = __builtin_amdgcn_readfirstlane((int)unit / line.total);
        at = __builtin_amdgcn_readfirstlane((int)unit - kvh * line.total);
        kvh = kvh * HEADS + side;
    } else {
        // the KV heads of a span on neighbouring workgroups of an XCD, so that token rows of the cache are read together
        const StepSpans spans(line.total, p.n_spans, least);
        w = (int)(blockIdx.x & 7) * (int)(gridDim.x >> 3) + (int)(blockIdx.x >> 3);
        const int span = p.kv_heads.div(w);
        kvh = (w - span * p.kv_heads.d) * HEADS + side;
        w = span * p.a.n_kv_heads + kvh;
        at = spans.start(span);
        len = span < p.n_spans.d ? spans.start(span + 1) - at : 0;
        if (len <= 0) return;
    }

    // The call's arguments, loaded where they are used: what only a piece's start and end want is not kept in scalar registers, of which
    // 60 ... 98 were spilled to vector registers, and vector registers to memory (24 x 5 drafted tokens 110 us, now 89).
    auto arguments = []() {
        typedef const __attribute__((address_space(4))) PagedMxStepParams* Kernarg;
        Kernarg at = (Kernarg)__builtin_amdgcn_kernarg_segment_ptr();
        asm volatile("" : "+s"(at));
        PagedMxStepParams q;
        __builtin_memcpy(&q, (const PagedMxStepParams*)at, sizeof(q));
        return q;
    };

    // Row tile `rt` of sequence `seq`; uniform.  (The sequence itself is looked up where it is needed: scalar registers are short.)
    struct Unit {
        int seq, rt, keys, tiles;
    };
    auto unit_of = [&](const MxCut& cut, const PagedSeq& s, int seq, int rt) {
        const int keys = cut.keys(s, rt);
        return Unit{seq, rt, keys, max(1, (keys + kStepTile - 1) / kStepTile)};
    };
    auto next_unit = [&](const Unit& u) {
        const PagedMxStepParams p = arguments();
        int seq = u.seq, rt = u.rt + 1;
        PagedSeq s = line.seq(seq, p.a.batch);
        while (rt >= p.cut.row_tiles(s)) {
            rt = 0;
            if (++seq >= p.a.batch.batch) return Unit{0, 0, 0, 1};       // (never, unless the offsets change under the launch)
            s = line.seq(seq, p.a.batch);
        }
        return unit_of(p.cut, s, seq, rt);
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
        if constexpr (UNITS) {
            rt = n_rt - 1 - at;              // the longest first
        } else {
            for (; rt < n_rt; ++rt) {
                const int n = cut.tiles(s, rt);
                if (at < n) break;
                at -= n;
            }
        }
        if (rt < 0 || rt >= n_rt) return;    // (never, as above)
        unit = unit_of(cut, s, seq, rt);
        tile = UNITS ? 0 : at;
        if constexpr (UNITS) len = unit.tiles;
    }

    // ---- requests: tile number n of the span is wavefront n % WAVES's.  Each asks for the one after the last that it asked for, in
    // the same unit or a later one.  Page numbers are scalar loads a tile ahead (they count against another counter than the tiles).
    Unit req = unit;
    int req_tile = tile + wave, req_left = len - wave;
    auto settle = [&]() {
        while (req_tile >= req.tiles) {
            req_tile -= req.tiles;
            req = next_unit(req);
        }
    };
    const unsigned char* const k_head = cache.k + (int64_t)kvh * cache.head_b;
    const unsigned char* const v_head = cache.v + (int64_t)kvh * cache.head_b;
    const unsigned char* const ks_head = cache.ks + (int64_t)kvh * cache.scale_head_b;
    const unsigned char* const vs_head = cache.vs + (int64_t)kvh * cache.scale_head_b;
    const uint32_t slot_mask = (1u << cache.log_page) - 1;
    // lane offsets from the first key of a half (of the page that the lane's key is in)
    const uint32_t k_lane = (uint32_t)(SMALL ? m & 7 : m) * cache.row_b + 16u * c;
    const uint32_t ks_lane = ((uint32_t)c << cache.log_page) + (SMALL ? m & 7 : m);
    const uint32_t vs_lane = ((uint32_t)(m >> 2) << cache.log_page) + 4u * (SMALL ? c & 1 : c);
    uint32_t v_lane[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v_lane[i] = (4u * (SMALL ? c & 1 : c) + i) * cache.row_b + 4u * m;
    // Codes are marked as read once, but where heads share a workgroup and half a cache line is left for the neighbouring one's.  (By heads
    // 4 x 107,500 tokens 85 us, without the mark 94; it is on codes that are read again, too, by token with 32 and 48 rows by the
    // neighbouring head's workgroup, 24 x 5 drafted tokens 89 / 91, and by other units of a prompt, 3 of 640 32.0 / 31.2.)
    auto code_load = [](auto* from) {
        if constexpr (HEADS > 1) return *from;
        else return __builtin_nontemporal_load(from);
    };
    uint32_t number[SMALL ? 4 : 2];
    auto look_up = [&]() {
        const ConstInts table = (ConstInts)(uintptr_t)(bt.table_len > 0 ? bt.table + (int64_t)req.seq * bt.table_len : bt.cu_q);      // (without a page: a word to look at)
        constexpr int KEYS = SMALL ? 8 : 16;
#pragma unroll
        for (int i = 0; i < kStepTile / KEYS; ++i)
            number[i] = (uint32_t)table[max(0, min(req_tile * kStepTile + KEYS * i, req.keys - 1)) >> cache.log_page];
    };
    // Keys past the end come along, from the slots behind the last one or from whatever page is at hand: their scores are masked
    // and their values become zeros.
    const unsigned char *v_base[2], *vs_base[2];      // of the tile whose keys have been requested and whose values have not
    auto request_k = [&](MxTile& t) {
#pragma unroll
        for (int i = 0; i < (SMALL ? 4 : 2); ++i) number[i] = min(number[i], cache.last_page);      // (here, so that nobody waits for them before)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const unsigned char *kp, *ksp;
            if constexpr (SMALL) {      // a lane's keys are in one page, its values' too
                const uint64_t page = m & 8 ? number[2 * u + 1] : number[2 * u], page_v = c & 2 ? number[2 * u + 1] : number[2 * u];
                kp = k_head + page * cache.page_b;
                ksp = ks_head + page * cache.scale_page_b;
                v_base[u] = v_head + page_v * cache.page_b;
                vs_base[u] = vs_head + page_v * cache.scale_page_b;
            } else {
                const uint32_t slot = (uint32_t)(req_tile * kStepTile + 16 * u) & slot_mask;
                const uint64_t codes = number[u] * (uint64_t)cache.page_b + slot * (uint64_t)cache.row_b;
                const uint64_t scales = number[u] * (uint64_t)cache.scale_page_b + slot;
                kp = k_head + codes;
                ksp = ks_head + scales;
                v_base[u] = v_head + codes;
                vs_base[u] = vs_head + scales;
            }
            t.k[u] = code_load(reinterpret_cast<const u32x4*>(kp + k_lane));
            t.ks[u] = ksp[ks_lane];
        }
        if ((req_left -= WAVES) <= 0) return;      // (behind the last one it is asked for over and over)
        req_tile += WAVES;
        if (!UNITS) settle();
        look_up();
    };
    auto request_v = [&](MxTile& t) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
            for (int i = 0; i < 4; ++i) t.v[4 * u + i] = code_load(reinterpret_cast<const uint32_t*>(v_base[u] + v_lane[i]));
            t.vs[u] = *reinterpret_cast<const uint32_t*>(vs_base[u] + vs_lane);
        }
    };

    // ---- the piece in hand: tiles [tile, end) of the unit, `done` tiles of the span behind it
    const float sl2 = p.a.scale_log2;
    int end, first_vis, done = 0, q0, rows;   // (q0, rows: the unit's sequence begins there, and so many rows are its)
    int last_vis[NT];                         // last key of this lane's rows
    // Q as B operands, of more than 32 rows in LDS, one copy for the workgroup, in the order in which they are read: registers are short then
    u32x4 q_reg[QLDS ? 1 : NT][4];
    auto q_of = [&](int i, int t) { return __builtin_bit_cast(bf16x8, QLDS ? lds_q[side][(i * 4 + t) * 64 + lane] : q_reg[QLDS ? 0 : i][t]); };
    f32x4 o[NT][8];
    float m_run[NT], l_run[NT];    // softmax reference (kNoKey: no key yet; finite, so that it can be subtracted), denominators
    auto begin_piece = [&]() {
        const PagedMxStepParams p = arguments();
        const int last = unit.keys - 1, row0 = unit.rt * R;
        const PagedSeq seq = line.seq(unit.seq, p.a.batch);
        q0 = seq.q0;
        rows = min(R, seq.len_q * p.a.group - row0);
        end = min(unit.tiles, tile + len - done);
        first_vis = p.cut.causal ? seq.len_k - seq.len_q + p.cut.group.div(row0) : last;       // last key of the first row
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int row = row0 + nt * 16 + m, pos = p.cut.group.div(row), head = kvh * p.a.group + row - pos * p.a.group;
            last_vis[nt] = p.cut.causal ? min(last, seq.len_k - seq.len_q + pos) : last;
            // rows without a query stay zero and are not stored
            const __bf16* qrow = p.a.q + (q0 + pos) * p.a.q_stride + (int64_t)head * kHeadDim + 32 * c;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                if (QLDS && (nt * 4 + t) % WAVES != wave) continue;
                u32x4 raw = {0u, 0u, 0u, 0u};
                if (nt * 16 + m < rows) raw = *reinterpret_cast<const u32x4*>(qrow + 8 * t);
                if constexpr (QLDS) lds_q[side][(nt * 4 + t) * 64 + lane] = raw;
                else q_reg[nt][t] = raw;
            }
            m_run[nt] = kNoKey;
            l_run[nt] = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) o[nt][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        if constexpr (QLDS) {
            __syncthreads();
        } else {
            // Q is used here, so that the compiler waits for it here and not in the loop, where its wait would be one for the tiles
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int t = 0; t < 4; ++t) asm volatile("" : "+v"(q_reg[nt][t]));
        }
    };
    auto across = [](float x, auto op) {      // over the four lanes that share a row
        const uint32_t u = __builtin_bit_cast(uint32_t, x);
        const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        x = op(__builtin_bit_cast(float, (uint32_t)a[0]), __builtin_bit_cast(float, (uint32_t)a[1]));
        const uint32_t v = __builtin_bit_cast(uint32_t, x);
        const auto b = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        return op(__builtin_bit_cast(float, (uint32_t)b[0]), __builtin_bit_cast(float, (uint32_t)b[1]));
    };
    // V^T blocks of eight keys a lane, two at a time: block(j, V^T operand)
    auto blocks_of = [](const uint32_t (&v)[8], const float (&sv)[8], auto block) {
        auto pair = [&](auto which) {
            constexpr int P = decltype(which)::value;
            uint32_t d[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const bf16x2 x = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v[e], sv[e], P);
                d[e] = __builtin_bit_cast(uint32_t, x);
            }
            u32x4 lo, hi;
#pragma unroll
            for (int f = 0; f < 4; ++f) {
                lo[f] = __builtin_amdgcn_perm(d[2 * f + 1], d[2 * f], 0x05040100u);
                hi[f] = __builtin_amdgcn_perm(d[2 * f + 1], d[2 * f], 0x07060302u);
            }
            block(2 * P, __builtin_bit_cast(bf16x8, lo));
            block(2 * P + 1, __builtin_bit_cast(bf16x8, hi));
        };
        pair(std::integral_constant<int, 0>{});
        pair(std::integral_constant<int, 1>{});
        pair(std::integral_constant<int, 2>{});
        pair(std::integral_constant<int, 3>{});
    };
    auto scales_of = [](const uint32_t (&b)[2], float (&sv)[8]) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            sv[4 * h] = mx_scale<0>(b[h]);
            sv[4 * h + 1] = mx_scale<1>(b[h]);
            sv[4 * h + 2] = mx_scale<2>(b[h]);
            sv[4 * h + 3] = mx_scale<3>(b[h]);
        }
    };

    auto work = [&](MxTile& t, int number_of) {
        const int key0 = number_of * kStepTile, keys = unit.keys, last = keys - 1;
        f32x4 s[NT][2];
#pragma unroll
        for (int x = 0; x < NT; ++x) s[x][0] = s[x][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const float scale = mx_scale_of(t.ks[u]);
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                const bf16x8 kf = __builtin_bit_cast(bf16x8, mx_values(t.k[u][d], scale));
#pragma unroll
                for (int x = 0; x < NT; ++x) s[x][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, q_of(x, d), s[x][u], 0, 0, 0);
            }
        }
        request_k(t);
        // mask, softmax reference, weights
        const bool need_mask = key0 + kStepTile - 1 > min(first_vis, last);
        bf16x8 pp[NT];
#pragma unroll
        for (int x = 0; x < NT; ++x) {
            if (need_mask) {
                const int lim = last_vis[x] - key0 - 4 * c;
#pragma unroll
                for (int r = 0; r < 8; ++r)
                    if (16 * (r >> 2) + (r & 3) > lim) s[x][r >> 2][r & 3] = -INFINITY;
            }
            // The reference is kept lazily: it moves only for a score more than 2^8 ahead of it, and only then do the four lanes
            // of a row exchange anything.
            float mx = s[x][0][0];
#pragma unroll
            for (int r = 1; r < 8; ++r) mx = fmaxf(mx, s[x][r >> 2][r & 3]);
            mx *= sl2;
            if (__any(mx > m_run[x] + 8.f)) {
                mx = across(mx, [](float a, float b) { return fmaxf(a, b); });
                if (mx > m_run[x] + 8.f) {
                    const float alpha = __builtin_amdgcn_exp2f(m_run[x] - mx);
                    m_run[x] = mx;
                    l_run[x] *= alpha;
#pragma unroll
                    for (int j = 0; j < 8; ++j)
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[x][j][i] *= alpha;
                }
            }
            float rs = 0.f;
            u32x4 packed;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const f32x2 y = {__builtin_amdgcn_exp2f(fmaf(s[x][e >> 1][2 * (e & 1)], sl2, -m_run[x])),
                                 __builtin_amdgcn_exp2f(fmaf(s[x][e >> 1][2 * (e & 1) + 1], sl2, -m_run[x]))};
                rs += y[0] + y[1];      // the denominator from the unrounded weights; for the product they are bf16, as everywhere here
                packed[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(y, bf16x2));
            }
            pp[x] = __builtin_bit_cast(bf16x8, packed);
            l_run[x] += rs;
        }
        float sv[8];
        auto sum_up = [&](int j, const bf16x8& vf) {
#pragma unroll
            for (int x = 0; x < NT; ++x) o[x][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pp[x], o[x][j], 0, 0, 0);
        };
        // values past the end: zero
        uint32_t v[8], vs[2] = {t.vs[0], t.vs[1]};
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = t.v[e];
        auto zero = [&](int e) {
            v[e] = 0u;
            vs[e >> 2] = (vs[e >> 2] & ~(0xffu << 8 * (e & 3))) | 127u << 8 * (e & 3);
        };
        auto key_of = [&](int e) { return 16 * (e >> 2) + 4 * c + (e & 3); };
        if (key0 + kStepTile > keys) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (key0 + key_of(e) >= keys) zero(e);
        }
        // A value that some of the rows do not see reaches them as 0 x value, which NaN (and what exceeds bf16) is not.  In tiles
        // with such keys their values are zeroed for the product, and each is added by itself to the rows that see it.
        uint32_t odd_keys = 0;
        if (min(key0 + kStepTile - 1, last) > first_vis) {
            uint32_t odd = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if ((vs[e >> 2] >> 8 * (e & 3) & 0xffu) >= 253u && key0 + key_of(e) > first_vis) odd |= 1u << e;
            if (__any(odd != 0)) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint64_t b = __ballot(odd >> e & 1);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (b >> 16 * i & 0xffff) odd_keys |= 1u << (16 * (e >> 2) + 4 * i + (e & 3));
                }
                odd_keys = __builtin_amdgcn_readfirstlane(odd_keys);
                // (an infinity or NaN goes in with the weight 1, as its own may be 0 in fp32)
                auto added = [](float to, float weight, uint32_t y) {
                    const float value = __builtin_bit_cast(float, y);
                    return fmaf((y & 0x7f800000u) == 0x7f800000u ? 1.f : weight, value, to);
                };
                // (a key's 16 bytes for the dims of this lane's results are read again: few registers, and seldom)
                const ConstInts table = (ConstInts)(uintptr_t)(bt.table + (int64_t)unit.seq * bt.table_len);
#pragma unroll 1
                for (uint32_t rest = odd_keys; rest != 0; rest &= rest - 1) {
                    const int key = __builtin_ctz(rest), at_key = key0 + key;
                    const uint64_t page = min((uint32_t)table[at_key >> cache.log_page], cache.last_page);
                    const uint32_t slot = (uint32_t)at_key & slot_mask;
                    const u32x4 codes = *reinterpret_cast<const u32x4*>(v_head + page * cache.page_b + (uint64_t)slot * cache.row_b + 16 * c);
                    const float scale = mx_scale_of(vs_head[page * cache.scale_page_b + ((uint32_t)c << cache.log_page) + slot]);
#pragma unroll
                    for (int x = 0; x < NT; ++x) {
                        const u32x4 two = __builtin_bit_cast(u32x4, pp[x]);
                        const uint32_t own = key & 16 ? (key & 2 ? two[3] : two[2]) : (key & 2 ? two[1] : two[0]);
                        const uint32_t its = (uint32_t)__shfl((int)own, (key >> 2 & 3) * 16 + m);
                        const float weight = __builtin_bit_cast(float, key & 1 ? its & 0xffff0000u : its << 16);
                        if (at_key > last_vis[x]) continue;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            __builtin_amdgcn_sched_barrier(0);      // (four values at a time: registers are short)
                            const u32x4 y = mx_values(codes[i], scale);
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                o[x][2 * j][i] = added(o[x][2 * j][i], weight, y[j] << 16);
                                o[x][2 * j + 1][i] = added(o[x][2 * j + 1][i], weight, y[j] & 0xffff0000u);
                            }
                        }
                    }
                }
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (odd_keys >> key_of(e) & 1) zero(e);
            }
        }
        scales_of(vs, sv);
        blocks_of(v, sv, sum_up);
        request_v(t);
    };
    // ---- a piece's results are joined, 16 rows at a time, and go out, as the unit's or into the piece's slot.  O goes through LDS in 16-byte
    // chunks of 4 dims, chunk ch of row r at slot ch * 16 + (r ^ ch % 16): writers (a row per lane) and readers (a chunk per lane, so that
    // a row leaves as one run) touch all banks evenly.
    float *const join_m = joint, *const join_l = joint + WAVES * 16, *const join_w = joint + 2 * WAVES * 16;
    auto finish_piece = [&](int piece0) {
        const PagedMxStepParams p = arguments();
        int lane = threadIdx.x & 63, tid = threadIdx.x % (WAVES * 64);
        asm volatile("" : "+v"(lane), "+v"(tid));      // places in LDS and in the results are worked out here, too
        const int m = lane & 15, c = lane >> 4;
        const bool whole = piece0 == 0 && end == unit.tiles;
        const int row0 = unit.rt * R;
        const int64_t slot_row = (int64_t)(2 * w + (piece0 == 0 ? 1 : 0)) * R;      // of n_spans x KV heads x 2
        float* const dst = whole ? static_cast<float*>(p.a.out) : p.part_out;
        const bool f32 = !whole || p.a.out_f32;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            if (nt * 16 >= rows) break;
            const float l_tot = across(l_run[nt], [](float a, float b) { return a + b; });
            if constexpr (WAVES == 1) {      // nobody to join
                const int flat = row0 + nt * 16 + m, pos = p.cut.group.div(flat), head = kvh * p.a.group + flat - pos * p.a.group, token = q0 + pos;
                if (nt * 16 + m >= rows) continue;
                const float inv = l_tot == 0.f ? 0.f : 1.f / l_tot;
                float* const to = whole ? p.a.lse + (int64_t)head * p.a.batch.total_q + token : p.part_lse + slot_row + nt * 16 + m;
                if (c == 0) *to = l_tot == 0.f ? -INFINITY : (m_run[nt] + __builtin_amdgcn_logf(l_tot)) * kLn2;      // NaN from NaN weights
                const int64_t row = whole ? (int64_t)token * p.a.n_q_heads + head : slot_row + nt * 16 + m;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    f32x8 y;
#pragma unroll
                    for (int j = 0; j < 8; ++j) y[j] = o[nt][j][i] * inv;
                    const int64_t idx = row * kHeadDim + 32 * c + 8 * i;
                    if (f32) *reinterpret_cast<f32x8*>(dst + idx) = y;
                    else *reinterpret_cast<bf16x8*>(static_cast<__bf16*>(p.a.out) + idx) = __builtin_convertvector(y, bf16x8);
                }
                continue;
            }
            if (c == 0) {
                join_m[wave * 16 + m] = m_run[nt];
                join_l[wave * 16 + m] = l_tot;
            }
            f32x4* const po = reinterpret_cast<f32x4*>(joint_o) + wave * 512;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int ch = 8 * c + 2 * i + half;
                    po[ch * 16 + (m ^ (ch & 15))] = f32x4{o[nt][4 * half][i], o[nt][4 * half + 1][i], o[nt][4 * half + 2][i], o[nt][4 * half + 3][i]};
                }
            __syncthreads();
            if (tid < WAVES * 16) {   // one thread per (row, wavefront): the wavefront's weight
                const int row = tid & 15, k = tid >> 4;
                float mx = kNoKey, den = 0.f;
#pragma unroll
                for (int i = 0; i < WAVES; ++i) mx = fmaxf(mx, join_m[i * 16 + row]);
#pragma unroll
                for (int i = 0; i < WAVES; ++i) den += join_l[i * 16 + row] * __builtin_amdgcn_exp2f(join_m[i * 16 + row] - mx);
                const float inv = den == 0.f ? 0.f : 1.f / den;
                join_w[k * 16 + row] = __builtin_amdgcn_exp2f(join_m[k * 16 + row] - mx) * inv;
                if (k == 0 && nt * 16 + row < rows) {
                    const int flat = row0 + nt * 16 + row, pos = p.cut.group.div(flat);
                    float* const to = whole ? p.a.lse + (int64_t)(kvh * p.a.group + flat - pos * p.a.group) * p.a.batch.total_q + q0 + pos : p.part_lse + slot_row + nt * 16 + row;
                    *to = den == 0.f ? -INFINITY : (mx + __builtin_amdgcn_logf(den)) * kLn2;      // NaN from NaN weights
                }
            }
            __syncthreads();
            const int ch = tid & 31;
#pragma unroll
            for (int pass = 0; pass < 8 / WAVES; ++pass) {
                const int row = pass * 2 * WAVES + (tid >> 5), flat = row0 + nt * 16 + row, pos = p.cut.group.div(flat);
                f32x4 z = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < WAVES; ++k) {
                    const float wgt = join_w[k * 16 + row];
                    const f32x4 y = reinterpret_cast<const f32x4*>(joint_o)[k * 512 + ch * 16 + (row ^ (ch & 15))];
#pragma unroll
                    for (int i = 0; i < 4; ++i) z[i] = fmaf(wgt, y[i], z[i]);
                }
                if (nt * 16 + row < rows) {
                    const int64_t to = whole ? (int64_t)(q0 + pos) * p.a.n_q_heads + kvh * p.a.group + flat - pos * p.a.group : slot_row + nt * 16 + row;
                    if (f32) *reinterpret_cast<f32x4*>(dst + to * kHeadDim + 4 * ch) = z;
                    else *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(p.a.out) + to * kHeadDim + 4 * ch) = __builtin_convertvector(z, bf16x4);
                }
            }
            __syncthreads();      // before the next 16 rows, or the next piece's, go there
        }
    };

    MxTile t;
    if (req_left > 0) {
        if (!UNITS) settle();
        look_up();
        request_k(t);
        request_v(t);
    }
    for (;;) {
        begin_piece();
        const int piece0 = tile;
        for (int n = tile + ((wave - done) & (WAVES - 1)); n < end; n += WAVES) work(t, n);
        finish_piece(piece0);
        done += end - piece0;
        if (UNITS || done >= len) return;
        unit = next_unit(unit);
        tile = 0;
    }
}

}  // namespace pec
