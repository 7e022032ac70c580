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
// NT = 1: eight wavefronts per workgroup, one stage.  NT = 2 (up to 64 rows): four wavefronts with 512 registers each, two stages.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "paged_common.hpp"
#include "paged_simple_kernel.hpp"

namespace pec {

constexpr int kPagedWaves1 = 8, kPagedWaves2 = 4;     // wavefronts per workgroup of up to 32 and up to 64 rows a unit
constexpr int kStepTile = 32;
constexpr int kStepTileBytes = kStepTile * kRowBytes;
constexpr int kPagedChunks = 1024;                     // sequences are added up 64 at a time: up to 65,536 of them

struct PagedStepParams {
    PagedAttnParams a;
    float* part_out;          // [spans][KV heads][2][32 NT][128]
    float* part_lse;          // [spans][KV heads][2][32 NT]
    int32_t* prefix;          // [batch + 1]: steps of a KV head ahead of each sequence, and of all of them
    int32_t n_spans;          // of a KV head
    int32_t most_rows;        // sequences with more rows than this are not this launch's (0x7fffffff: all are)
};

// Steps (tiles of 32 keys, at least one) of row tile `rt` of `s`, R rows each, and of all of its row tiles.
__device__ __forceinline__ int step_keys(const PagedSeq& s, int group, int causal, int r, int rt) {
    if (!causal) return s.len_k;
    const int64_t rows = min((int64_t)s.len_q * group, (int64_t)(rt + 1) * r);
    return max(0, min(s.len_k, s.len_k - s.len_q + (int)((rows - 1) / group) + 1));
}
__device__ __forceinline__ int step_tiles(const PagedSeq& s, int group, int causal, int r, int rt) {
    return max(1, (step_keys(s, group, causal, r, rt) + kStepTile - 1) / kStepTile);
}
__device__ __forceinline__ int step_row_tiles(const PagedSeq& s, int group, int r, int most_rows) {
    const int64_t rows = (int64_t)s.len_q * group;
    return rows > most_rows ? 0 : (int)((rows + r - 1) / r);
}
__device__ __forceinline__ int step_tiles_of(const PagedSeq& s, int group, int causal, int r, int most_rows) {
    const int n = step_row_tiles(s, group, r, most_rows);
    int sum = 0;
    for (int rt = 0; rt < n; ++rt) sum += step_tiles(s, group, causal, r, rt);
    return sum;
}
__device__ __forceinline__ int wave_prefix(int x) {      // inclusive
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int y = __shfl_up(x, d);
        if (lane >= d) x += y;
    }
    return x;
}
struct StepSpans {
    int len, extra;              // the first `extra` spans have len + 1 steps
    __device__ __forceinline__ StepSpans(int steps, int n_spans) : len(steps / n_spans), extra(steps % n_spans) {}
    __device__ __forceinline__ int start(int i) const { return i * len + min(i, extra); }
    __device__ __forceinline__ int of(int step) const {       // the span that the step falls into
        const int head = extra * (len + 1);
        return step < head ? step / (len + 1) : extra + (step - head) / max(1, len);
    }
};

template <int NT, int WAVES, int S>
__global__ __launch_bounds__(WAVES * 64, 1) void paged_step_kernel(const PagedStepParams p) {
    constexpr int R = 32 * NT;
    constexpr int LOADS = 8;                 // load instructions (1 KiB each) per matrix and tile
    __shared__ __attribute__((aligned(1024))) unsigned char lds[WAVES * S * 2 * kStepTileBytes];
    __shared__ int32_t chunk_sum[kPagedChunks];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    const int l32 = lane & 31, hl = lane >> 5;
    const int g = p.a.group, causal = p.a.causal;

    // ---- all steps of a KV head, and where this wavefront's span begins.  Up to 64 sequences sit in the lanes of every wavefront.
    const PagedBatch& bt = p.a.batch;
    const int n_chunks = (bt.batch + 63) >> 6;
    auto load = [&](int b) {
        PagedSeq s{0, 0, 0};
        if (b < bt.batch) s = paged_seq(bt, b);
        return s;
    };
    auto tiles_of = [&](const PagedSeq& s) { return step_tiles_of(s, g, causal, R, p.most_rows); };
    PagedSeq lanes = load(lane);
    int own = tiles_of(lanes), upto = wave_prefix(own), per_head;
    if (n_chunks <= 1) {
        per_head = __builtin_amdgcn_readlane(upto, 63);
    } else {
        for (int c = wave; c < n_chunks; c += WAVES) {
            const int sum = wave_prefix(tiles_of(load(64 * c + lane)));
            if (lane == 63) chunk_sum[c] = sum;
        }
        __syncthreads();
        int sum = 0;
        for (int c = lane; c < n_chunks; c += 64) sum += chunk_sum[c];
        per_head = __builtin_amdgcn_readlane(wave_prefix(sum), 63);
    }
    if (blockIdx.x == 0) {       // for the merge
        for (int c = wave, ahead = 0, at = 0; c < n_chunks; c += WAVES) {
            for (; at < c; ++at) ahead += chunk_sum[at];
            const int mine = tiles_of(load(64 * c + lane)), all = wave_prefix(mine);
            if (64 * c + lane < bt.batch) p.prefix[64 * c + lane] = ahead + all - mine;
        }
        if (threadIdx.x == 0) p.prefix[bt.batch] = per_head;
    }
    if (per_head == 0) return;
    const StepSpans spans(per_head, p.n_spans);
    const int group_no = (int)(blockIdx.x & 7) * (int)(gridDim.x >> 3) + (int)(blockIdx.x >> 3);     // neighbours on one XCD
    const int w = group_no * WAVES + wave, span = w / p.a.n_kv_heads, kvh = w % p.a.n_kv_heads;
    const int start = spans.start(span);
    int left = span < p.n_spans ? spans.start(span + 1) - start : 0;       // tiles to work on
    if (left <= 0) return;

    // Row tile `rt` of sequence `seq`; uniform.
    struct Unit {
        PagedSeq s;
        int seq, rt, row0, rows, keys, tiles;
    };
    auto seq_of = [&](int i) {
        PagedSeq s;
        if (n_chunks <= 1) {
            s.q0 = __builtin_amdgcn_readlane(lanes.q0, i);
            s.len_q = __builtin_amdgcn_readlane(lanes.len_q, i);
            s.len_k = __builtin_amdgcn_readlane(lanes.len_k, i);
        } else {
            s = paged_seq(bt, i);
        }
        return s;
    };
    auto unit_of = [&](const PagedSeq& s, int seq, int rt) {
        Unit u;
        u.s = s;
        u.seq = seq;
        u.rt = rt;
        u.row0 = rt * R;
        u.rows = (int)min((int64_t)R, (int64_t)s.len_q * g - u.row0);
        u.keys = step_keys(s, g, causal, R, rt);
        u.tiles = max(1, (u.keys + kStepTile - 1) / kStepTile);
        return u;
    };
    auto next_unit = [&](const Unit& u) {
        PagedSeq s = u.s;
        int seq = u.seq, rt = u.rt + 1;
        while (rt >= step_row_tiles(s, g, R, p.most_rows)) {
            rt = 0;
            if (++seq >= bt.batch) {       // (never, unless the offsets change under the launch)
                seq = 0;
                break;
            }
            s = seq_of(seq);
        }
        return unit_of(s, seq, rt);
    };
    Unit unit;
    int tile;
    {
        int at = start, c0 = 0;
        if (n_chunks > 1) {              // the chunk of 64 sequences
            for (;; c0 += 64) {
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
            own = tiles_of(load(64 * c0 + lane));
            upto = wave_prefix(own);
        }
        const uint64_t behind = __ballot(upto > at);     // the sequence
        if (behind == 0) return;         // (never, unless the offsets change under the launch)
        const int l = __builtin_ctzll(behind);
        at = __builtin_amdgcn_readfirstlane(at - __builtin_amdgcn_readlane(upto, l) + __builtin_amdgcn_readlane(own, l));
        const int seq = 64 * c0 + l;
        const PagedSeq s = seq_of(seq);
        const int n_rt = step_row_tiles(s, g, R, p.most_rows);
        int rt = 0;                      // the row tile
        for (; rt < n_rt; ++rt) {
            const int n = step_tiles(s, g, causal, R, rt);
            if (at < n) break;
            at -= n;
        }
        if (rt >= n_rt) return;          // (the same)
        unit = unit_of(s, seq, rt);
        tile = at;
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
    uint32_t number[4];      // page numbers of its four groups of eight keys (keys past the end: the last key's),
    int64_t off[4];          // and byte offsets of the groups
    auto look_up = [&]() {
        if (req.keys == 0) return;
        const ConstInts table = (ConstInts)(uintptr_t)(bt.table + (int64_t)req.seq * bt.table_len);
#pragma unroll
        for (int i = 0; i < 4; ++i) number[i] = (uint32_t)table[min(req_tile * kStepTile + 8 * i, req.keys - 1) >> cache.log_page];
    };
    auto locate = [&]() {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int key = min(req_tile * kStepTile + 8 * i, (req.keys - 1) & ~7);
            off[i] = min(number[i], cache.last_page) * cache.page_b + (uint64_t)(uint32_t)(key & ((1 << cache.log_page) - 1)) * cache.row_b + head_off;
        }
    };
    // (a unit without keys is one tile whose loads fetch whatever is at the start of the cache; everything of it is masked)
    auto issue = [&](const unsigned char* pool, bool is_v, unsigned char* stage) {
        const uint32_t l0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)stage;
        if ((req_tile + 1) * kStepTile <= req.keys) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i)
                dma16_once(pool + off[i >> 1] + (i & 1) * 4 * (int64_t)cache.row_b, is_v ? ldv : ldk[i & 3], l0 + i * 1024);
        } else {      // keys past the end re-read the last one: their weights are zero
            const int last = max(0, req.keys - 1);
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const int key = 4 * i + ld_row;
                const uint32_t col = is_v ? (uint32_t)((((ld_pos >> 2) ^ (key & 3)) << 2) | (ld_pos & 3)) * 16u
                                          : (uint32_t)(ld_pos ^ (key & 15)) * 16u;
                const int from = min(req_tile * kStepTile + key, last) - min(req_tile * kStepTile + 8 * (i >> 1), last & ~7);
                dma16_once(pool + off[i >> 1], (uint32_t)from * cache.row_b + col, l0 + i * 1024);
            }
        }
    };
    auto request_k = [&](unsigned char* stage) {
        if (req.keys == 0) {
#pragma unroll
            for (int i = 0; i < 4; ++i) off[i] = 0;
        } else {
            locate();
        }
        issue(cache.k, false, stage);
    };
    auto request_v = [&](unsigned char* stage) {
        issue(cache.v, true, stage);
        if (--req_left == 0) return;
        if (++req_tile == req.tiles) {
            req = next_unit(req);
            req_tile = 0;
        }
        look_up();
    };
    look_up();
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
        const int piece0 = tile, end = min(unit.tiles, tile + left);
        const int first_vis = causal ? unit.s.len_k - unit.s.len_q + row0 / g : last;       // last key of the first row
        int last_vis[NT];                                                                  // ... of this lane's rows
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) last_vis[nt] = causal ? min(last, unit.s.len_k - unit.s.len_q + (row0 + nt * 32 + l32) / g) : last;

        // ---- Q fragments: rows without a query stay zero and are not stored
        bf16x8 qf[NT][8];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int r = row0 + nt * 32 + l32;
            const __bf16* qrow = p.a.q + (unit.s.q0 + r / g) * p.a.q_stride + ((int64_t)kvh * g + r % g) * kHeadDim + 8 * hl;
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
        for (; tile < end; ++tile, ++n) {
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
                        rs += x[0] + x[1];   // the denominator from the unrounded weights; for the product they are bf16
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
                                const bf16x4 x = *reinterpret_cast<const bf16x4*>(row + (v_lds_off(key, 64 * dt + 16 * b + 8 * hl) - key * kRowBytes));
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

        // ---- the unit's result, or the piece's into its slot
        const bool whole = piece0 == 0 && end == unit.tiles;
        const int64_t slot_row = (int64_t)(2 * w + (piece0 == 0 ? 1 : 0)) * R;      // of n_spans x KV heads x 2
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const float l_tot = l_run[nt] + __shfl_xor(l_run[nt], 32);
            if (nt * 32 + l32 < rows) {
                const int r = row0 + nt * 32 + l32, head = kvh * g + r % g, token = unit.s.q0 + r / g;
                const bool none = l_tot == 0.f || keys == 0;       // (without keys the values may be anything, and the sums NaN)
                const float inv = none ? 0.f : 1.f / l_tot;
                const float lse = none ? -INFINITY : (m_run[nt] + __builtin_amdgcn_logf(l_tot)) * kLn2;     // NaN from NaN weights
                if (hl == 0) {
                    if (whole) p.a.lse[(int64_t)head * bt.total_q + token] = lse;
                    else p.part_lse[slot_row + nt * 32 + l32] = lse;
                }
                const int64_t at = whole ? ((int64_t)token * p.a.n_q_heads + head) * kHeadDim : (slot_row + nt * 32 + l32) * kHeadDim;
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
// wavefront of the chip, which leaves no barrier between them, four where there are fewer and more pieces each.  `tokens`:
// workgroups per sequence and query head (times four for WAVES = 1), which share its new tokens.
constexpr int kPagedMergeThreads = 256;
template <int WAVES>
__global__ __launch_bounds__(kPagedMergeThreads) void paged_merge_kernel(const PagedStepParams p, int r_unit, int tokens) {
    constexpr int N = 2 * WAVES, AHEAD = 4;
    __shared__ __attribute__((aligned(16))) float red[N][kHeadDim];
    __shared__ float red_mx[N], red_den[N];
    const PagedBatch& bt = p.a.batch;
    const int g = p.a.group, head = blockIdx.y, kvh = head / g, grp = (threadIdx.x >> 5) % N, c = threadIdx.x & 31;
    const int per_head = p.prefix[bt.batch];
    constexpr int PER_GROUP = WAVES == 1 ? 4 : 1;       // rows a workgroup works on at a time
    for (int x = blockIdx.x * PER_GROUP + (WAVES == 1 ? (int)(threadIdx.x >> 6) : 0); x < bt.batch * tokens; x += gridDim.x * PER_GROUP) {
        const int seq = x / tokens;
        const PagedSeq s = paged_seq(bt, seq);
        const int before = p.prefix[seq], n_rt = step_row_tiles(s, g, r_unit, p.most_rows);
        if (per_head == 0 || n_rt == 0) continue;
        const StepSpans spans(per_head, p.n_spans);
        int rt = 0, at = before;       // the row tile in hand, and its first step
        for (int pos = x % tokens; pos < s.len_q; pos += tokens) {
            const int64_t flat = (int64_t)pos * g + head % g;
            for (; rt < (int)(flat / r_unit); ++rt) at += step_tiles(s, g, p.a.causal, r_unit, rt);
            const int w0 = spans.of(at), w1 = spans.of(at + step_tiles(s, g, p.a.causal, r_unit, rt) - 1);
            if (w0 == w1) continue;
            const int row = (int)(flat - (int64_t)rt * r_unit);
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
                        const int64_t slot_row = (((int64_t)(w + i * N) * p.a.n_kv_heads + kvh) * 2 + (w + i * N == w0 ? 1 : 0)) * r_unit + row;
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
                    else *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(p.a.out) + out_row + 4 * c) = __builtin_convertvector(acc, bf16x4);
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
