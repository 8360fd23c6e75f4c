// Attention of many new tokens over the paged cache on the tensor cores (tcgen05.mma, accumulators in tensor memory): prompt chunks and
// single tokens of one batch in one launch, causal, with an optional sliding window and first tokens that stay visible.
//
// Mathematics: one pass with a running maximum and sum.  For a tile of up to 128 query rows (a token's heads of one KV head are rows of the same tile) and
// steps of 80 tokens,
//     S = Q K^T (128 x 80),   p = 2^(S scale - m),   l += sum p,   O += P V (128 x 128),
// with a lazy reference m: it moves only when a step's maximum exceeds it by more than 8 (weights stay below 256), and then l and O are rescaled.  P is
// rounded to bf16 for the product (the tensor core's operand type; 2^-8 of each weight, averaged by the sum); l adds the unrounded weights in fp32.
// Parts of a unit leave (m, l, O) in fp32, and states of the same row join as M = max m, l = sum 2^(m_i - M) l_i, O likewise.  No part is longer than 2048 steps
// (see kChunkPartSteps), so l is off by at most 2^-24 (2048 + 22 + the number of parts) of itself, and by far less where errors average.
//
// A unit is two tiles of one sequence and KV head (256 rows, a pair), or its last rows if they fit one tile (solo), over the pages that they see: all
// up to the last row's own, or the sinks' pages and those from the first row's window on.  A pair gives each of two streams a tile and both the same K and V;
// a solo unit alternates its steps between the streams.  One CTA per SM, 12 warps:
//   warps 0-3, 4-7  softmax of stream 0 and stream 1: one query row per thread (TMEM lane), 80 scores at a time
//   warp 8, 11      copies: query tiles and K; V.  A ring of four steps; a page's K (or V) is one copy of 4 KiB
//   warp 9, 10      the products of stream 0 and of stream 1
// Tensor memory, 256 of the 512 columns per stream: S (80), P (40), O (128).  Steps of 80 tokens are the longest whose weights fit beside the scores, so that
// S of the next step runs as soon as the scores have been read.
//
// Bounds.  Single tokens (64 x 16K, 32 / 8 heads): memory, 642 us, 6.69 TB/s; what it took is a short way round the ring (copies of V that do not stand in
// K's way, satisfied barriers that cost little).  Chunks: the softmax of the two warps that share a scheduler.  A pair's step takes 2400 cycles (512 rows behind
// 64K), of a stream's 1180 for the weights, 350 for the maximum, 140 for reading the scores, 310 waiting for products; the products of both streams alone would take 1432
// (128 x 80 x 16 reads 6.5 KiB of shared memory, 52 cycles, and P V 64).  Under load the board's power limit adds to that (2048 rows behind 128K: 3.6 to 3.9 ms in a
// burst, 4.2 ms at 1.6 GHz sustained, 1.04 to 1.09 PFLOP/s of 1.37 that a plain product sustains).  Sixteen softmax warps with half a row each took the
// same time, sixteen with quarter rows (16-lane loads) 1.6 times as long.  A unit costs about 5.2 us beyond its steps of 1.3.
//
// Every wait on an mbarrier is bounded, anew for each part of a segment; when one runs out the CTA sets KAP_ERR_TIMEOUT, later waits return at once, the roles run
// to their end inside this CTA's shared and tensor memory, copies and products in flight are waited for (bounded again), tensor memory is freed and
// the kernel returns.
#pragma once

#include "kap_ptx.cuh"

namespace kap {

constexpr int kChunkSoftmaxWarps = 8;                                 // 4 a stream
constexpr int kChunkThreads = 32 * (kChunkSoftmaxWarps + 4);
constexpr int kChunkTileRows = 128;                                    // query rows of one tile (TMEM lanes)
constexpr int kChunkUnitRows = 2 * kChunkTileRows;
// Solo units of up to 64 rows use products of 64 rows, which take half the energy, and single tokens run into the board's power limit, too (windowed batch
// sustained 970 us, with 128 rows 1040).  Row r of such a tile is lane r % 16 of the quarter r / 16.
constexpr int kChunkSmallRows = 64;
constexpr int kChunkStepPages = 5;
constexpr int kChunkStepTokens = kChunkStepPages * kPageSize;          // 80
constexpr int kChunkSlots = 8;                                         // step n: K in slot 2 n, V in slot 2 n + 1 (mod 8)
// A slot holds the step's pages one after the other, each as [two groups of 8 tokens][columns 0-63, 64-127][token]: one copy a page, and the
// groups of all pages lie 2 KiB apart, as the products' operands want it.
constexpr int kChunkSlotBytes = kChunkStepPages * kTileBytes;          // 20 KiB
constexpr int kChunkGroupBytes = 2048, kChunkHalfBytes = 1024;
constexpr int kChunkQHalfBytes = kChunkTileRows * 128;                 // 128 rows x 64 columns: 16 KiB
constexpr int kChunkQBytes = 2 * kChunkQHalfBytes;
constexpr int kChunkTmemP = 80, kChunkTmemO = 128;                     // columns of a stream's 256; S from 0
constexpr int kChunkMaxSegments = 72;                                  // planned at a time
// A sequence's tokens: a whole unit of so many takes a CTA two seconds, and steps stay far below the sentinel of chunk_in_step.
constexpr int kChunkMostTokens = 1 << 26;
// What a unit costs, to place the cuts and for nothing else: its tokens and, for the first products and the epilogue, some more, times 2 with two
// tiles.  (Windowed batch 835 us, with 5 : 3 910, 3 : 1 895; 2 x 4096 on the tape 316 us, with 320 tokens more 327, with 240 341.)
constexpr int kChunkUnitCost = 400, kChunkPairCost = 2, kChunkSoloCost = 1;
// Of a CTA's share: fewer CTAs work when there is little to do.  (32 / 8 heads, with 320, 640 and 1280: one token at 100 14.4, 17.8, 22.6 us, at 1K 16.9, 20.3, 22.0, at 4K
// 23.1, 21.6, 25.6; 16 tokens at 1K 26.6, 26.4, 27.2; 50 rows of 500 21.4, 23.9, 27.3, behind 4K 28.4, 28.5, 31.2.)
constexpr int kChunkLeastCost = 640;

// One sum over all steps of a long context would lose what is small beside it (2^24 equal weights of 0.37 in a pair: l 0.13 % off, and O, whose products the
// tensor core adds without rounding to nearest, 9 %; 128K of them 0.0014 % and 0.04 %).  So a segment is done in parts of at most so many steps (163840 tokens),
// each with fresh sums, whose states join one after the other in memory: l and O are then off by no more than those of 128K, the time is the same to 0.5 %, and
// waits have their limits for a part of some milliseconds, not for a unit, which may take seconds.
// (Joined in a function that the loop over the steps calls, prompts took 2 to 3 % longer.)
constexpr int kChunkPartSteps = 2048;

struct alignas(16) ChunkSegment {                                      // what one CTA does of one unit (query tile pair, KV head)
    int32_t list_at;                                                   // the sequence's first entry in bt_pages
    int32_t tok0, lo;                                                  // first token row of q, its logical position (negative: sees nothing)
    int32_t rows_head;                                                 // query rows | KV head << 16
    int32_t step_begin, step_end;
    int32_t length;                                                    // tokens of the sequence
    int32_t slot;                                                      // of its partial state; -1: the whole unit, writes the output
};
struct ChunkCut { long long unit; int32_t inside, tok0, rows_head, pad; };   // where a CTA begins; inside: in the middle of this unit
// In step (see chunk_in_step): units of one sequence, the first ones whole, the last n_cut cut into `pieces` each; pieces = 0: not in step.
// Dealt (see chunk_deal): seq = -1, pieces = 1, `whole` units, none cut.
struct ChunkInStep { int32_t pieces, n_cut, whole, seq; };
constexpr int kChunkDealSeqs = 16, kChunkDealRounds = 3;               // dealing: sequences at most, units for each CTA at least
constexpr int kChunkStates = 4;                                        // states a CTA, 256 rows each, that the workspace holds
constexpr int kChunkMostPieces = 16, kChunkPieceCost = 8;              // cost of a piece beyond its steps (products to fill, state), in steps
constexpr long long kChunkInStepBytes = 48ll << 20;
static_assert(kChunkMostTokens / kChunkStepTokens + 10 * kChunkMostPieces < (INT32_MAX >> 8), "the sentinel of chunk_in_step");

struct ChunkControl {
    unsigned long long full[kChunkSlots], free[kChunkSlots];
    unsigned long long q_full[2], q_free[2];
    unsigned long long s_ready[2], s_free[2], p_ready[2], pv_done[2];  // [stream]
    unsigned long long drained;
    uint32_t tmem_base;
    int32_t timed_out;
    int32_t n_segments, more;                                          // of this round; another round follows
    int32_t active, active_seq;                                        // sequences with rows, one of them
    uint32_t has_rows[kChunkThreads / 32];                             // a bit for each sequence, in batches of up to kChunkThreads
    ChunkInStep in_step;
    // plan: this CTA's range of the tape
    int32_t seq, unit, step, end_seq, end_unit, end_step, first_done;
    long long warp_sum[kChunkThreads / 32];
    int32_t cut_seq[2];
    long long cut_rest[2];
};
struct ChunkShared {
    ChunkControl c;
    alignas(16) ChunkSegment segments[kChunkMaxSegments];
};
// The next part of segment k, of which `done` steps have been dealt with; moves both on.
__device__ __forceinline__ ChunkSegment chunk_next_part(const ChunkShared& sh, int& k, int& done) {
    ChunkSegment s = sh.segments[k];
    s.step_begin += done;
    if (s.step_end - s.step_begin > kChunkPartSteps) {
        s.step_end = s.step_begin + kChunkPartSteps;
        done += kChunkPartSteps;
    } else {
        done = 0;
        ++k;
    }
    return s;
}
constexpr int kChunkCtlBytes = 3 * 1024;
constexpr int kChunkSmemBytes = 2 * kChunkQBytes + kChunkSlots * kChunkSlotBytes + kChunkCtlBytes;
static_assert(sizeof(ChunkShared) <= kChunkCtlBytes && kChunkSmemBytes <= 232448, "shared memory");

struct ChunkParams {
    const int32_t *q_indptr, *bt_indptr, *bt_pages, *ctx_len;
    float *part_o, *part_ml;
    ChunkCut* cuts;                                                    // [gridDim.x + 1]
    ChunkInStep* in_step;
    __nv_bfloat16* out;
    float* lse;
    int32_t* status;
    long long num_pool_pages;
    int32_t batch, total_rows, hq, hkv, G, log2_g, window, n_sink, wide_out;      // wide_out: out lies on a 32-byte boundary
    float scale_log2;
};

// ------------------------------------------------------------------------------------------------------------------ plan
// All units of the batch, ordered by sequence, KV head and tile, lie on a tape whose length is their cost; CTA i of n takes the tape from
// i / n to (i + 1) / n of it.  Every CTA finds its two ends by itself, from closed forms, so that lengths may live on the device (4 us from the start of
// the kernel to the first copy; a unit is cut at most as often as CTAs share it, two states a CTA).
struct ChunkSeq { int32_t row0, n, length, list_at; };                 // first row of q, rows, tokens, block table

__device__ __forceinline__ ChunkSeq chunk_seq(const ChunkParams& p, int b, bool& bad) {
    const int r0 = p.q_indptr[b], r1 = p.q_indptr[b + 1], L = p.ctx_len[b], l0 = p.bt_indptr[b], l1 = p.bt_indptr[b + 1];
    const long long listed = max(0ll, (long long)l1 - l0) * kPageSize;
    ChunkSeq s;
    s.row0 = min(max(r0, 0), p.total_rows);
    s.n = max(min(r1, p.total_rows) - s.row0, 0);
    s.length = l0 < 0 ? 0 : (int)min((long long)min(max(L, 0), kChunkMostTokens), listed);
    s.list_at = l0;
    bad = r0 != s.row0 || r1 != s.row0 + s.n || (s.n > 0 && L != s.length);      // (a sequence without rows may have any length)
    return s;
}
__device__ __forceinline__ int chunk_tiles(const ChunkParams& p, int n) {
    return (n + (kChunkUnitRows >> p.log2_g) - 1) >> (8 - p.log2_g);
}
// cost of the first k tiles of a sequence, for one KV head
__device__ __forceinline__ long long chunk_cost(const ChunkParams& p, const ChunkSeq& s, int k) {
    if (k <= 0) return 0;
    const int R = kChunkUnitRows >> p.log2_g, t = chunk_tiles(p, s.n), whole = min(k, t - 1);
    const long long lo = max(0, s.length - s.n), knee = (long long)p.window + p.n_sink;   // where the window begins to leave tokens out
    const long long m = p.window ? min((long long)whole, max(0ll, (knee - lo + R - 1) >> (8 - p.log2_g))) : whole;
    long long c = kChunkPairCost * (whole * (long long)kChunkUnitCost + m * lo + R * (m * (m + 1) / 2) + (whole - m) * (knee + R));
    if (k == t) {
        const int rest = s.n - (t - 1) * R;
        const long long at = lo + (long long)(t - 1) * R, seen = p.window && at >= knee ? knee + rest : at + rest;
        c += (rest * p.G > kChunkTileRows ? kChunkPairCost : kChunkSoloCost) * (kChunkUnitCost + seen);
    }
    return c;
}
struct ChunkPages { int32_t head, first, n; };                         // logical pages 0 .. head-1 and first .. first + n - head - 1
__device__ __forceinline__ ChunkPages chunk_pages(const ChunkParams& p, int lo, int hi) {
    ChunkPages g;
    const int end = hi < 0 ? 0 : hi / kPageSize + 1;
    g.first = p.window ? (int)(max(0ll, (long long)lo - p.window + 1) / kPageSize) : 0;
    g.first = min(g.first, end);
    g.head = min(g.first, (int)(((long long)p.n_sink + kPageSize - 1) / kPageSize));
    g.n = g.head + end - g.first;
    return g;
}
__device__ __forceinline__ int chunk_steps(const ChunkParams& p, const ChunkSeq& s, int tile) {
    const int R = (kChunkUnitRows >> p.log2_g), lo = s.length - s.n + tile * R, hi = min(lo + R, s.length) - 1;
    return (chunk_pages(p, lo, hi).n + kChunkStepPages - 1) / kChunkStepPages;
}

// How one sequence whose rows all see a long context is divided: instead of a range of the tape, which begins anywhere in a unit, CTA i takes the
// units i, i + n, ... as far as they go round, and of the rest, each cut into pieces, the pieces i, i + n, ... in the order of the context.  All CTAs
// then walk the same tokens at about the same time, tiles of one head next to each other, so that K and V come from L2, which could not hold the
// 512 MB of 128K tokens (2048 rows behind them sustained 4.87 ms on the tape, 4.06 so).  Around the limits, bursts, tape / in step: 512 rows behind 12000 (47 MiB of K and
// V) 117 / 114 us, behind 32K 275 / 285, 64K 551 / 524; 2048 behind 16K 468 / 497, 32K 983 / 961, 64K 2032 / 1864; with eight tokens for each row 4096
// rows behind 32K 1897 / 1947, with four 8192 rows 3765 / 3819: up to 6 % either way, until the context is well beyond L2.  Called by one warp.
__device__ __forceinline__ void chunk_in_step(const ChunkParams& p, ChunkControl& c) {
    const int lane = threadIdx.x & 31, n_cta = gridDim.x;
    bool bad;
    const ChunkSeq s = chunk_seq(p, c.active_seq, bad);
    const int t = chunk_tiles(p, s.n), units = t * p.hkv, rest = units % n_cta, steps = chunk_steps(p, s, t - 1);
    const long long seen = p.window ? min((long long)s.length, (long long)p.window + p.n_sink + s.n) : s.length;
    ChunkInStep v{0, rest, units - rest, c.active_seq};
    if (t >= 2 && s.length / 8 >= s.n && seen * p.hkv * (4 * kHeadDim) >= kChunkInStepBytes) {
        // the number of pieces that ends first
        const int k = lane + 1, rounds = (rest * k + n_cta - 1) / n_cta;
        int cost = k > kChunkMostPieces || rest * k > kChunkStates * n_cta ? INT32_MAX >> 8 : rounds * ((steps + k - 1) / k + (k > 1 ? kChunkPieceCost : 0));
        cost = (cost << 5 | lane);                                     // (steps: below 2^20)
        v.pieces = (__reduce_min_sync(0xffffffffu, cost) & 31) + 1;
    }
    if (lane == 0) {
        c.in_step = v;
        if (blockIdx.x == 0) *p.in_step = v;
        c.unit = 0;                                                    // segments planned so far
    }
}

// Whole units dealt out: where there are many of falling cost, prompts above all, a range of the tape each leaves CTAs with cut units (states, and the join)
// and with no more even shares than the costs are right.  Instead units are sorted by the tokens that they see, a counting sort in closed form: tile k of a
// sequence is in class lo / R + 1 + k (lo: its cached tokens, R: tokens of a tile), a solo unit in that of a pair of its cost; and CTA i takes the units at
// i, 2 n - 1 - i, 2 n + i, ... .  (Prompts of 3 x 5000 231 us, on the tape 250; 2 x 4096 286 and 310; 1 x 4096 143 and 161.)  Not where whole units cannot
// be shared evenly: the last, incomplete round has to cost less than an eighth of a share, the dearest unit less than 3 / 5.  Inside these limits dealing took 0.85 to
// 1.00 of the tape's time in 20 batches of all kinds.  Outside it may gain or lose.  Last round: 1 x 4400 (0.13 of a share) tape 180, dealt 160 us; 2 x 2048 behind 1K
// (0.20) 161, 151; behind 4K (0.25) 327, 345; behind 8K (0.27) 559, 604.  Dearest unit: 1 x 2600 (0.78) 85, 72; 64 rows behind 16K beside short prompts (2.1) 148, 344.
struct ChunkDealt { int32_t base, pairs, solo; };                      // of a lane's sequence: first class and number of pairs, class of the solo unit or -1
__device__ __forceinline__ ChunkDealt chunk_dealt(const ChunkParams& p, const ChunkControl& c, ChunkSeq& s) {
    int b = -1, rank = threadIdx.x & 31;                               // the rank-th sequence with rows
    if (rank < c.active) {
#pragma unroll 1
        for (int w = 0; w < kChunkThreads / 32; ++w) {
            uint32_t has = c.has_rows[w];
            const int n = __popc(has);
            if (rank >= n) { rank -= n; continue; }
            while (rank--) has &= has - 1u;
            b = w * 32 + __ffs(has) - 1;
            break;
        }
    }
    ChunkDealt d{0, 0, -1};
    s = ChunkSeq{0, 0, 0, 0};
    if (b >= 0) {
        bool bad;
        s = chunk_seq(p, b, bad);
        const int R = kChunkUnitRows >> p.log2_g, t = chunk_tiles(p, s.n), rest = s.n - (t - 1) * R, lo = max(0, s.length - s.n);
        const long long knee = (long long)p.window + p.n_sink + rest, seen = p.window ? min((long long)s.length, knee) : s.length;
        d.base = lo / R + 1;
        d.pairs = t;
        if (rest * p.G <= kChunkTileRows) { --d.pairs; d.solo = (int)max(0ll, seen / 2 - kChunkUnitCost / 2) / R; }
    }
    return d;
}
// of the sequences' units (of one KV head) those in class h and above
__device__ __forceinline__ int chunk_dealt_from(const ChunkDealt& d, int active, int h) {
    int n = 0;
    for (int i = 0; i < active; ++i) {
        const int base = __shfl_sync(0xffffffffu, d.base, i), pairs = __shfl_sync(0xffffffffu, d.pairs, i), solo = __shfl_sync(0xffffffffu, d.solo, i);
        n += min(max(base + pairs - h, 0), pairs) + (solo >= h && solo >= 0 ? 1 : 0);
    }
    return n;
}
// the q-th of them, in falling classes: (lane of its sequence, tile); every lane has a q of its own
__device__ __forceinline__ int2 chunk_dealt_at(const ChunkDealt& d, int active, int q) {
    int lo = 0, hi = __reduce_max_sync(0xffffffffu, max(d.base + d.pairs, d.solo + 1));      // from(lo) > q >= from(hi)
    for (int left = hi; left > 0; left >>= 1) {
        const int mid = (lo + hi) >> 1;
        const bool more = chunk_dealt_from(d, active, mid) > q;
        if (hi - lo > 1) { if (more) lo = mid; else hi = mid; }
    }
    int rest = q - chunk_dealt_from(d, active, lo + 1);
    int2 at = make_int2(0, 0);
    bool found = false;
    for (int i = 0; i < active; ++i) {
        const int base = __shfl_sync(0xffffffffu, d.base, i), pairs = __shfl_sync(0xffffffffu, d.pairs, i), solo = __shfl_sync(0xffffffffu, d.solo, i);
        if (lo >= base && lo < base + pairs) {
            if (!found && rest == 0) { at = make_int2(i, lo - base); found = true; }
            --rest;
        }
        if (solo == lo) {
            if (!found && rest == 0) { at = make_int2(i, pairs); found = true; }
            --rest;
        }
    }
    return at;
}
// whether to deal; called by one warp
__device__ __forceinline__ void chunk_deal(const ChunkParams& p, ChunkControl& c) {
    const int lane = threadIdx.x & 31, n_cta = gridDim.x, active = c.active;
    ChunkSeq s;
    const ChunkDealt d = chunk_dealt(p, c, s);
    const int units = __reduce_add_sync(0xffffffffu, chunk_tiles(p, s.n)) * p.hkv;
    if (units < kChunkDealRounds * n_cta) return;
    // the dearest unit, and the dearest of the last, incomplete round
    const int last = units / n_cta * n_cta, q = lane == 0 || last == units ? 0 : last / p.hkv;
    const int2 at = chunk_dealt_at(d, active, q);
    ChunkSeq o;
    o.row0 = 0; o.list_at = 0;
    o.n = __shfl_sync(0xffffffffu, s.n, at.x); o.length = __shfl_sync(0xffffffffu, s.length, at.x);
    const long long cost = chunk_cost(p, o, at.y + 1) - chunk_cost(p, o, at.y);
    const long long dearest = __shfl_sync(0xffffffffu, cost, 0), tail = last == units ? 0 : __shfl_sync(0xffffffffu, cost, 1);
    long long share = 0;
    for (int w = 0; w < kChunkThreads / 32; ++w) share += c.warp_sum[w];
    share /= n_cta;
    if (8 * tail > share || 5 * dearest > 3 * share) return;
    if (lane == 0) {
        const ChunkInStep v{1, 0, units, -1};
        c.in_step = v;
        if (blockIdx.x == 0) *p.in_step = v;
        c.unit = 0;
    }
}

// this CTA's ends; called by all threads
__device__ __forceinline__ void chunk_plan(const ChunkParams& p, ChunkControl& c) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, per = (p.batch + kChunkThreads - 1) / kChunkThreads;
    long long mine = 0;
    bool rows = false;
    for (int i = 0; i < per; ++i) {
        const int b = tid * per + i;
        if (b >= p.batch) break;
        bool bad;
        const ChunkSeq s = chunk_seq(p, b, bad);
        if (bad && blockIdx.x == 0) atomicOr(p.status, 1 << KAP_ERR_DEVICE_INDEX);
        if (s.n > 0) { atomicAdd(&c.active, 1); c.active_seq = b; rows = true; }
        mine += chunk_cost(p, s, chunk_tiles(p, s.n)) * p.hkv;
    }
    const uint32_t has_rows = __ballot_sync(0xffffffffu, rows);
    if (lane == 0) c.has_rows[warp] = has_rows;
    long long upto = mine;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const long long o = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += o;
    }
    if (lane == 31) c.warp_sum[warp] = upto;
    if (tid < 2) c.cut_seq[tid] = p.batch;                             // the tape's end
    __syncthreads();
    const bool deals = c.active > 0 && c.active <= kChunkDealSeqs && per == 1;
    if (c.active == 1 || deals) {
        if (warp == 0) {
            if (c.active == 1) chunk_in_step(p, c);
            __syncwarp();
            if (deals && !c.in_step.pieces) chunk_deal(p, c);
        }
        __syncthreads();
        if (c.in_step.pieces) return;
    }
    if (tid == 0 && blockIdx.x == 0) p.in_step->pieces = 0;
    long long total = 0, before = 0;
#pragma unroll
    for (int w = 0; w < kChunkThreads / 32; ++w) {
        if (w == warp) before = total;
        total += c.warp_sum[w];
    }
    before += upto - mine;
    const long long parts = max(1ll, min((long long)gridDim.x, total / kChunkLeastCost));
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const long long i = min((long long)blockIdx.x + e, parts), x = i == parts ? total : (long long)((double)total * ((double)i / (double)parts));
        if (x < before || x >= before + mine) continue;
        long long rest = x - before;
        for (int k = 0; k < per; ++k) {
            const int b = tid * per + k;
            bool bad;
            const ChunkSeq s = chunk_seq(p, b, bad);
            const long long cost = chunk_cost(p, s, chunk_tiles(p, s.n)) * p.hkv;
            if (rest < cost || k == per - 1 || b == p.batch - 1) {
                c.cut_seq[e] = b;
                c.cut_rest[e] = rest;
                break;
            }
            rest -= cost;
        }
    }
    __syncthreads();
    if (warp < 2) {                                                    // unit and step of each end
        const int b = c.cut_seq[warp];
        int unit = 0, step = 0, tok0 = 0, rows_head = 0, inside = 0;
        if (b < p.batch) {
            bool bad;
            const ChunkSeq s = chunk_seq(p, b, bad);
            const int t = chunk_tiles(p, s.n), R = (kChunkUnitRows >> p.log2_g);
            const long long one = chunk_cost(p, s, t);
            int head = min((int)((double)c.cut_rest[warp] / (double)one), p.hkv - 1);
            if (head * one > c.cut_rest[warp]) --head;                 // (a quotient that was rounded up)
            const long long y = c.cut_rest[warp] - head * one;
            int k = 0, hi = t;                                         // cost(k) <= y < cost(hi)
            while (hi - k > 1) {
                const int stride = (hi - k + 31) / 32, probe = k + lane * stride;
                const uint32_t below = __ballot_sync(0xffffffffu, probe < hi && chunk_cost(p, s, probe) <= y);
                const int at = k + max(31 - __clz(below), 0) * stride;
                hi = min(hi, at + stride);
                k = at;
            }
            const int steps = chunk_steps(p, s, k), rows = min(R, s.n - k * R) * p.G;
            const int z = (int)((y - chunk_cost(p, s, k)) / (rows > kChunkTileRows ? kChunkPairCost : kChunkSoloCost)) - kChunkUnitCost;     // (below 2^31: a context's tokens and a tile's)
            step = min(steps, max(0, (z + kChunkStepTokens / 2) / kChunkStepTokens));
            unit = head * t + k;
            inside = step > 0 && step < steps;
            tok0 = s.row0 + k * R;
            rows_head = rows | head << 16;
            if (step == steps && steps > 0) { ++unit; step = 0; }      // (unit = t hkv: the next sequence's first)
        }
        if (lane == 0) {
            if (warp == 0) { c.seq = b; c.unit = unit; c.step = step; c.first_done = 0; }
            else { c.end_seq = b; c.end_unit = unit; c.end_step = step; }
            if (warp == 0 || blockIdx.x == gridDim.x - 1) {
                ChunkCut cut;
                cut.unit = (long long)b << 32 | (unsigned)unit;
                cut.inside = inside ? step : 0; cut.tok0 = tok0; cut.rows_head = rows_head; cut.pad = 0;
                p.cuts[blockIdx.x + warp] = cut;
            }
        }
    }
    __syncthreads();
}

// the next segments of this CTA; called by one warp
__device__ __forceinline__ void chunk_segments(const ChunkParams& p, ChunkShared& sh) {
    ChunkControl& c = sh.c;
    const int lane = threadIdx.x & 31, R = (kChunkUnitRows >> p.log2_g);
    if (c.in_step.pieces) {
        const ChunkInStep v = c.in_step;
        if (v.seq < 0) {
            ChunkSeq s;
            const ChunkDealt d = chunk_dealt(p, c, s);
            const int n_cta = gridDim.x, cta = blockIdx.x, first = c.unit, rounds = v.whole / n_cta, turn = rounds & 1 ? n_cta - 1 - cta : cta;
            const int all = rounds + (rounds * n_cta + turn < v.whole ? 1 : 0), take = min(all - first, kChunkMaxSegments);
            for (int k0 = 0; k0 < take; k0 += 32) {
                const int k = first + min(k0 + lane, take - 1), q = k * n_cta + (k & 1 ? n_cta - 1 - cta : cta);
                const int2 at = chunk_dealt_at(d, c.active, q / p.hkv);
                ChunkSeq o;
                o.row0 = __shfl_sync(0xffffffffu, s.row0, at.x); o.n = __shfl_sync(0xffffffffu, s.n, at.x);
                o.length = __shfl_sync(0xffffffffu, s.length, at.x); o.list_at = __shfl_sync(0xffffffffu, s.list_at, at.x);
                ChunkSegment g;
                g.list_at = o.list_at; g.tok0 = o.row0 + at.y * R; g.lo = o.length - o.n + at.y * R;
                g.rows_head = (min(R, o.n - at.y * R) << p.log2_g) | (q % p.hkv) << 16;
                g.step_begin = 0; g.step_end = chunk_steps(p, o, at.y);
                g.length = o.length;
                g.slot = -1;
                if (k0 + lane < take) sh.segments[k0 + lane] = g;
            }
            __syncwarp();
            if (lane == 0) { c.n_segments = take; c.more = first + take < all; c.unit = first + take; }
            return;
        }
        bool bad;
        const ChunkSeq s = chunk_seq(p, v.seq, bad);
        const int t = chunk_tiles(p, s.n), n_cta = gridDim.x, first = c.unit, rounds = v.whole / n_cta, cut = v.n_cut * v.pieces;
        const int all = rounds + ((int)blockIdx.x < cut ? (cut - 1 - (int)blockIdx.x) / n_cta + 1 : 0), take = min(all - first, kChunkMaxSegments);
        for (int k = lane; k < take; k += 32) {
            const int at = first + k, q = (at - rounds) * n_cta + (int)blockIdx.x;      // q: of the pieces
            const bool whole = at < rounds;
            const int piece = whole ? 0 : q / v.n_cut, u = whole ? at * n_cta + (int)blockIdx.x : v.whole + q % v.n_cut, head = u / t, tile = u % t;
            const int steps = chunk_steps(p, s, tile), pieces = whole ? 1 : v.pieces;
            ChunkSegment g;
            g.list_at = s.list_at; g.tok0 = s.row0 + tile * R; g.lo = s.length - s.n + tile * R;
            g.rows_head = (min(R, s.n - tile * R) << p.log2_g) | head << 16;
            g.step_begin = (int)((long long)steps * piece / pieces);
            g.step_end = (int)((long long)steps * (piece + 1) / pieces);
            g.length = s.length;
            g.slot = pieces == 1 ? -1 : q;
            sh.segments[k] = g;
        }
        __syncwarp();
        if (lane == 0) { c.n_segments = take; c.more = first + take < all; c.unit = first + take; }
        return;
    }
    int seq = c.seq, unit = c.unit, step = c.step, first_done = c.first_done, n = 0;
    const int end_seq = c.end_seq, end_unit = c.end_unit, end_step = c.end_step;
    const int last_seq = end_unit > 0 || end_step > 0 ? end_seq : end_seq - 1;
    while (n < kChunkMaxSegments && seq <= last_seq) {
        const int b = seq + lane;
        ChunkSeq s{0, 0, 0, 0};
        bool bad;
        if (b <= last_seq) s = chunk_seq(p, b, bad);
        const int t = chunk_tiles(p, s.n), skip = lane == 0 ? unit : 0;
        const int units = (b == end_seq ? end_unit + (end_step > 0 ? 1 : 0) : t * p.hkv) - skip;
        int upto = max(units, 0);
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const int o = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= d) upto += o;
        }
        const int all = __shfl_sync(0xffffffffu, upto, 31), take = min(all, kChunkMaxSegments - n);
        int next_seq = seq + 32, next_unit = 0;
        for (int k0 = 0; k0 < take; k0 += 32) {
            const int k = min(k0 + lane, take - 1);
            int owner = 0;                                             // lanes whose units all come before k
#pragma unroll
            for (int d = 16; d > 0; d /= 2)
                if (__shfl_sync(0xffffffffu, upto, owner + d - 1) <= k) owner += d;
            ChunkSeq o;
            o.row0 = __shfl_sync(0xffffffffu, s.row0, owner); o.n = __shfl_sync(0xffffffffu, s.n, owner);
            o.length = __shfl_sync(0xffffffffu, s.length, owner); o.list_at = __shfl_sync(0xffffffffu, s.list_at, owner);
            const int prior = __shfl_sync(0xffffffffu, upto, max(owner - 1, 0)), before = owner ? prior : 0;
            const int ot = chunk_tiles(p, o.n), u = k - before + (owner == 0 ? unit : 0), head = u / ot, tile = u % ot;
            const int steps = chunk_steps(p, o, tile);
            ChunkSegment g;
            g.list_at = o.list_at; g.tok0 = o.row0 + tile * R; g.lo = o.length - o.n + tile * R;
            g.rows_head = min(R, o.n - tile * R) * p.G | head << 16;
            const bool cta_first = !first_done && n + k == 0, cta_last = seq + owner == end_seq && u == end_unit;
            g.step_begin = cta_first ? step : 0;
            g.step_end = cta_last ? end_step : steps;
            g.length = o.length;
            g.slot = g.step_begin == 0 && g.step_end == steps ? -1 : (int)blockIdx.x * 2 + (g.step_end < steps ? 1 : 0);
            if (k0 + lane < take) sh.segments[n + k] = g;
            if (k0 + 32 >= take) {                                     // where the next round goes on, if these were not all
                const int src = take - 1 - k0;
                const int nu = __shfl_sync(0xffffffffu, u + 1, src), no = __shfl_sync(0xffffffffu, owner, src), nt = __shfl_sync(0xffffffffu, ot * p.hkv, src);
                if (take < all) { next_seq = seq + no + (nu == nt); next_unit = nu == nt ? 0 : nu; }
            }
        }
        n += take;
        if (take == all) { next_seq = seq + 32; next_unit = 0; }
        seq = next_seq; unit = next_unit;
    }
    if (lane == 0) {
        c.n_segments = n;
        c.more = seq < last_seq || (seq == last_seq && (seq != end_seq || unit < end_unit + (end_step > 0 ? 1 : 0)));
        c.seq = seq; c.unit = unit; c.first_done = first_done || n > 0;
    }
}

// --------------------------------------------------------------------------------------------------------------- softmax
__device__ __forceinline__ void chunk_load_scores(uint32_t at, float (&s)[kChunkStepTokens]) {
    uint32_t u[kChunkStepPages][16];
#pragma unroll
    for (int i = 0; i < kChunkStepPages; ++i) tmem_ld16_nowait(at + i * 16, u[i]);
    tmem_wait_ld();
#pragma unroll
    for (int i = 0; i < kChunkStepTokens; ++i) s[i] = __uint_as_float(u[i >> 4][i & 15]);
}
__device__ __forceinline__ float chunk_row_max(const float (&s)[kChunkStepTokens]) {
    float mx[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
    for (int i = 4; i + 8 <= kChunkStepTokens; i += 8)
#pragma unroll
        for (int e = 0; e < 4; ++e) mx[e] = max3(mx[e], s[i + e], s[i + 4 + e]);
#pragma unroll
    for (int e = 0; e < 4; ++e) mx[e] = fmaxf(mx[e], s[kChunkStepTokens - 4 + e]);
    return fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
}
// The weights 2^(s scale - mu) as packed bf16; returns their fp32 sum.  With kPoly one pair in four is computed on the FMA pipe (512 rows
// behind 64K 523 us, with none 546, one in eight 535, one in three 527, one in two 553), which
// gives at least 2^-126 where 2^-inf = 0 is wanted, so steps with masked scores do without it.
template <bool kPoly>
__device__ __forceinline__ float chunk_weights(const float (&s)[kChunkStepTokens], float scale, float mu, uint32_t (&w)[kChunkStepTokens / 2]) {
    const uint64_t sc2 = pack_f32x2(scale, scale), mu2 = pack_f32x2(-mu, -mu);
    uint64_t sum[2] = {0ull, 0ull};
#pragma unroll
    for (int e = 0; e < kChunkStepTokens / 2; ++e) {
        const uint64_t x = fma_f32x2(pack_f32x2(s[2 * e], s[2 * e + 1]), sc2, mu2);
        float a, b;
        if (kPoly && e % 4 == 3) {
            exp2_poly(x, a, b);
        } else {
            unpack_f32x2(x, a, b);
            a = ex2(a);
            b = ex2(b);
        }
        sum[e & 1] = add_f32x2(sum[e & 1], pack_f32x2(a, b));
        w[e] = pack_bf16(a, b);
    }
    float a, b;
    unpack_f32x2(add_f32x2(sum[0], sum[1]), a, b);
    return a + b;
}
// The waiting is done in a function of its own: with its loop at every wait, a barrier that had long been passed cost 50 cycles more (a group of eight
// products and two such waits 525 cycles, 435 with this and both barriers tried together).
__device__ __noinline__ bool wait_slowly(uint32_t bar, uint32_t parity, uint64_t deadline, volatile int32_t* late) { return mbar_wait(bar, parity, deadline, late); }
__device__ __forceinline__ bool both_passed(uint32_t bar0, uint32_t parity0, uint32_t bar1, uint32_t parity1) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p, q;\n\t"
                 "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tmbarrier.try_wait.parity.shared::cta.b64 q, [%3], %4;\n\t"
                 "and.pred p, p, q;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(bar0), "r"(parity0), "r"(bar1), "r"(parity1) : "memory");
    return ok != 0;
}
__device__ __forceinline__ void pair_barrier(int id) { asm volatile("bar.sync %0, 64;" ::"r"(id) : "memory"); }

template <bool kNhd>
__global__ void __launch_bounds__(kChunkThreads, 1)
kap_chunk_kernel(const __grid_constant__ CUtensorMap kv_map, const __grid_constant__ CUtensorMap q_map, const ChunkParams p)
{
    extern __shared__ unsigned char smem_raw[];
    if (smem_u32(smem_raw) & 1023u) {                                  // the tiles need it; no static shared memory, so it holds
        if (threadIdx.x == 0) atomicOr(p.status, 1 << KAP_ERR_DEVICE_INDEX);
        pdl_wait();
        return;
    }
    unsigned char* const q_tiles = smem_raw;
    unsigned char* const slots = smem_raw + 2 * kChunkQBytes;
    ChunkShared& sh = *reinterpret_cast<ChunkShared*>(slots + kChunkSlots * kChunkSlotBytes);
    ChunkControl* const c = &sh.c;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    if (tid == 0) {
        for (int i = 0; i < kChunkSlots; ++i) { mbar_init(smem_u32(&c->full[i]), 1); mbar_init(smem_u32(&c->free[i]), 2); }   // free: both issuers
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&c->q_full[i]), 1);
            mbar_init(smem_u32(&c->q_free[i]), 2);
            mbar_init(smem_u32(&c->s_ready[i]), 1);
            mbar_init(smem_u32(&c->s_free[i]), 4);                     // the stream's softmax warps
            mbar_init(smem_u32(&c->p_ready[i]), 4);
            mbar_init(smem_u32(&c->pv_done[i]), 1);
        }
        mbar_init(smem_u32(&c->drained), 2);
        c->timed_out = 0;
        c->active = 0;
        c->in_step.pieces = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&kv_map) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&q_map) : "memory");
    }
    __syncwarp();
    if (warp == 0) {                                                   // one CTA per SM: never waits
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&c->tmem_base)), "n"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = c->tmem_base;
    pdl_wait();                                                        // nothing of the caller's is read above
    pdl_launch_dependents();
    chunk_plan(p, *c);
    uint64_t deadline = global_ns() + kWaitBudgetNs;                   // of a part's waits; every role sets it anew
    volatile int32_t* const late = &c->timed_out;
    auto wait = [&](unsigned long long& bar, uint32_t parity) {
        return mbar_try_wait(smem_u32(&bar), parity) || wait_slowly(smem_u32(&bar), parity, deadline, late);
    };
    auto wait_both = [&](unsigned long long& bar0, uint32_t parity0, unsigned long long& bar1, uint32_t parity1) {
        if (both_passed(smem_u32(&bar0), parity0, smem_u32(&bar1), parity1)) return;
        wait_slowly(smem_u32(&bar0), parity0, deadline, late);
        wait_slowly(smem_u32(&bar1), parity1, deadline, late);
    };

    // state of the roles, kept over the rounds
    int loads = 0, q_use[2] = {0, 0}, q_slot = 0, step0 = 0, count = 0;
    uint32_t q_parity = 0;
    bool ok = true;
    uint64_t keep;
    asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(keep));

    for (;;) {
    if (warp == kChunkSoftmaxWarps + 3) chunk_segments(p, sh);
    __syncthreads();
    const int n_segments = c->n_segments, more_rounds = c->more;
    if (warp == kChunkSoftmaxWarps || warp == kChunkSoftmaxWarps + 3) {
        // ---- copies: one warp brings the query tiles and K, another V, which is needed later, so that neither waits for the other's slots.  Up
        // to five a step, issued by one elected lane with warp-uniform coordinates.
        const int v = warp == kChunkSoftmaxWarps ? 0 : 1;
        for (int k = 0, done = 0; k < n_segments && ok;) {
            const ChunkSegment s = chunk_next_part(sh, k, done);
            deadline = global_ns() + kWaitBudgetNs;
            const int rows = s.rows_head & 0xffff, kv_head = s.rows_head >> 16;
            const ChunkPages g = chunk_pages(p, s.lo, s.lo + (rows >> p.log2_g) - 1);
            const int n_steps = s.step_end - s.step_begin, page0 = s.step_begin * kChunkStepPages;
            const int n_pages = min(g.n - page0, n_steps * kChunkStepPages);
            const bool pair = rows > kChunkTileRows;
            if (n_steps <= 0) continue;
            auto fetch = [&](int i) {                                  // physical page of the segment's i-th
                if (i >= n_pages) return 0;
                const int at = page0 + i;
                return p.bt_pages[s.list_at + (at < g.head ? at : at - g.head + g.first)];
            };
            constexpr int kBatch = 30 / kChunkStepPages;               // page ids, 30 at a time and one batch ahead
            int32_t ids = 0, next_ids = lane < 30 ? fetch(lane) : 0;
            if (v == 0) {
                for (int t = 0; t < (pair ? 2 : 1) && ok; ++t) {
                    const int to = pair ? t : q_slot;
                    ok = __all_sync(0xffffffffu, q_use[to] == 0 || wait(c->q_free[to], (uint32_t)(q_use[to] - 1) & 1u));
                    if (!ok) break;
                    if (elect_one()) {
                        const uint32_t bar = smem_u32(&c->q_full[to]), dst = smem_u32(q_tiles) + to * kChunkQBytes;
                        const int tok = s.tok0 + t * (kChunkTileRows >> p.log2_g), head = kv_head << p.log2_g;
                        mbar_expect_tx(bar, kChunkQBytes);
                        tma_load_3d(dst, &q_map, 0, head, tok, bar, keep);
                        tma_load_3d(dst + kChunkQHalfBytes, &q_map, 64, head, tok, bar, keep);
                    }
                    __syncwarp();
                    ++q_use[to];
                }
                if (!pair) q_slot ^= 1;
            }
            int in_batch = 0;
            for (int j = 0; j < n_steps && ok; ++j, ++loads) {
                if (in_batch == 0) {
                    ids = next_ids;
                    next_ids = lane < 30 ? fetch((j + kBatch) * kChunkStepPages + lane) : 0;
                    if (ids < 0 || ids >= p.num_pool_pages) { ids = 0; atomicOr(p.status, 1 << KAP_ERR_DEVICE_INDEX); }
                }
                const int n = min(kChunkStepPages, n_pages - j * kChunkStepPages), slot = 2 * (loads % (kChunkSlots / 2)) + v;
                int32_t row[kChunkStepPages];                          // first token row of each page's K or V, in groups of 8
#pragma unroll
                for (int i = 0; i < kChunkStepPages; ++i) {
                    const int page = __shfl_sync(0xffffffffu, ids, in_batch * kChunkStepPages + i);
                    row[i] = (kNhd ? page * 2 + v : (page * 2 + v) * p.hkv + kv_head) * (kPageSize / 8);
                }
                if (++in_batch == kBatch) in_batch = 0;
                ok = __all_sync(0xffffffffu, wait(c->free[slot], ((uint32_t)(loads / (kChunkSlots / 2)) & 1u) ^ 1u));      // (the first round does not wait)
                if (!ok) break;
                if (elect_one()) {
                    const uint32_t bar = smem_u32(&c->full[slot]), dst = smem_u32(slots) + slot * kChunkSlotBytes;
                    mbar_expect_tx(bar, (uint32_t)n * kTileBytes);
#pragma unroll
                    for (int i = 0; i < kChunkStepPages; ++i)
                        if (i < n) tma_load_5d(dst + i * kTileBytes, &kv_map, row[i], kNhd ? kv_head : 0, bar, keep);
                }
                __syncwarp();
            }
        }
    } else if (warp == kChunkSoftmaxWarps + 1 || warp == kChunkSoftmaxWarps + 2) {
        // ---- tensor core: an issuer for each stream, so that neither waits for the other's softmax: S of its next step, then O += P V of the one
        // before.  One elected lane runs through a whole segment, waits included, with warp-uniform operands.  Both arrive on a tile's
        // free barrier, with their products or, where the tile is not theirs, as soon as it is there (its last use is then over).
        const int t = warp - (kChunkSoftmaxWarps + 1);
        const uint64_t q_desc = umma_smem_desc(smem_u32(q_tiles), 16, 1024), k_desc = umma_smem_desc(smem_u32(slots), 16, kChunkGroupBytes);
        // V: 16 tokens (K) x 128 columns (N), N contiguous; columns 64-127 in the other half of a group
        const uint64_t v_desc = umma_smem_desc(smem_u32(slots), kChunkHalfBytes, kChunkGroupBytes);
        for (int k = 0, done = 0; k < n_segments;) {
            const ChunkSegment seg = chunk_next_part(sh, k, done);
            deadline = global_ns() + kWaitBudgetNs;
            const int rows = __shfl_sync(0xffffffffu, seg.rows_head & 0xffff, 0);
            const ChunkPages g = chunk_pages(p, seg.lo, seg.lo + (rows >> p.log2_g) - 1);
            const int n_steps = __shfl_sync(0xffffffffu, seg.step_end - seg.step_begin, 0);
            const int n_pages = __shfl_sync(0xffffffffu, g.n - seg.step_begin * kChunkStepPages, 0);
            const int pair = rows > kChunkTileRows ? 1 : 0, stride = pair ? 1 : 2, first = pair ? 0 : t;       // this stream's steps
            if (n_steps <= 0) continue;
            const int base = step0, work0 = count, q_at = pair ? t : q_slot;
            const uint32_t idesc_o = rows <= kChunkSmallRows ? umma_idesc(kChunkSmallRows, kHeadDim, true) : umma_idesc(kChunkTileRows, kHeadDim, true);
            const uint32_t idesc_page = rows <= kChunkSmallRows ? umma_idesc(kChunkSmallRows, kPageSize, false) : umma_idesc(kChunkTileRows, kPageSize, false);
            if (elect_one()) {
                auto slot_of = [&](int j) { return 2 * ((base + j) % (kChunkSlots / 2)); };
                auto phase_of = [&](int j) { return (uint32_t)((base + j) / (kChunkSlots / 2)) & 1u; };
                // of a step that is the other stream's
                auto pass = [&](int j, int v) {
                    wait(c->full[slot_of(j) + v], phase_of(j));
                    mbar_arrive(smem_u32(&c->free[slot_of(j) + v]));
                };
                auto issue_s = [&](int j, int n) {                     // of step j, work n of the stream
                    const int slot = slot_of(j);
                    // the tile is there, and the softmax warps have read the scores before (a barrier's phase before its first has passed)
                    wait_both(c->full[slot], phase_of(j), c->s_free[t], (uint32_t)(n - 1) & 1u);
                    tc_fence_after();
                    const uint64_t q = q_desc + (uint32_t)q_at * (kChunkQBytes / 16), kd = k_desc + (uint32_t)slot * (kChunkSlotBytes / 16);
                    const int pages = min(kChunkStepPages, n_pages - j * kChunkStepPages);
                    const uint32_t idesc_s = idesc_page + ((uint32_t)(pages - 1) * (kPageSize >> 3) << 17);
#pragma unroll
                    for (int ks = 0; ks < 8; ++ks)
                        umma_ss(tmem + t * 256, q + ((ks >> 2) * kChunkQHalfBytes + (ks & 3) * 32) / 16,
                                kd + ((ks >> 2) * kChunkHalfBytes + (ks & 3) * 32) / 16, idesc_s, ks > 0);
                    umma_commit(smem_u32(&c->s_ready[t]));
                    umma_commit(smem_u32(&c->free[slot]));
                };
                auto issue_pv = [&](int j, int n) {
                    const int slot = slot_of(j) + 1;
                    wait_both(c->full[slot], phase_of(j), c->p_ready[t], (uint32_t)n & 1u);
                    tc_fence_after();
                    const uint64_t v = v_desc + (uint32_t)slot * (kChunkSlotBytes / 16);
                    const uint32_t o = tmem + t * 256 + kChunkTmemO, w = tmem + t * 256 + kChunkTmemP;
                    const int pages = min(kChunkStepPages, n_pages - j * kChunkStepPages);
#pragma unroll
                    for (int pg = 0; pg < kChunkStepPages; ++pg)
                        if (pg < pages) umma_ts(o, w + pg * 8, v + pg * (kTileBytes / 16), idesc_o, n > work0 || pg > 0);
                    umma_commit(smem_u32(&c->pv_done[t]));
                    umma_commit(smem_u32(&c->free[slot]));
                };
                wait(c->q_full[q_at], q_parity >> q_at & 1u);
                int n = work0, passed = 0;                             // passed: steps of the other stream up to here have been passed for V
                auto pass_v = [&](int upto) {
                    if (!pair)
                        for (; passed < upto; ++passed)
                            if ((passed & 1) != t) pass(passed, 1);
                };
                for (int j = first; j < n_steps; j += stride, ++n) {
                    if (!pair && j > 0) pass(j - 1, 0);
                    issue_s(j, n);
                    if (j + stride >= n_steps) umma_commit(smem_u32(&c->q_free[q_at]));
                    if (n > work0) { pass_v(j - stride); issue_pv(j - stride, n - 1); }
                }
                if (!pair && ((n_steps - 1) & 1) != t) pass(n_steps - 1, 0);
                if (n > work0) { const int last = first + (n - 1 - work0) * stride; pass_v(last); issue_pv(last, n - 1); }
                else mbar_arrive(smem_u32(&c->q_free[q_at]));          // (one step: nothing for the second stream)
                pass_v(n_steps);
                if (pair) {                                            // the other stream's query tile
                    wait(c->q_full[t ^ 1], q_parity >> (t ^ 1) & 1u);
                    mbar_arrive(smem_u32(&c->q_free[t ^ 1]));
                }
            }
            __syncwarp();
            step0 += n_steps;
            count += pair ? n_steps : (n_steps + 1 - t) >> 1;
            q_parity ^= pair ? 3u : 1u << q_slot;
            if (!pair) q_slot ^= 1;
        }
    } else if (warp < kChunkSoftmaxWarps) {
        // ---- softmax: stream = warp group, one query row per thread
        const int stream = warp >> 2;
        const uint32_t t_lane = tmem + ((uint32_t)((warp & 3) * 32) << 16), t_s = t_lane + stream * 256, t_p = t_s + kChunkTmemP, t_o = t_s + kChunkTmemO;
        const float sc = p.scale_log2;
        for (int k = 0, done = 0; k < n_segments;) {
            const bool joins = done > 0;                               // to the state that the parts before have left
            ChunkSegment seg = chunk_next_part(sh, k, done);
            const bool whole = seg.slot < 0 && done == 0;              // the unit's results, not a state
            // (of a unit that is not cut: a state that this CTA does not use otherwise, or not before)
            if (seg.slot < 0) seg.slot = (int)(c->in_step.pieces ? blockIdx.x : 2 * gridDim.x + blockIdx.x);
            deadline = global_ns() + kWaitBudgetNs;
            const int rows = seg.rows_head & 0xffff, kv_head = seg.rows_head >> 16;
            const bool pair = rows > kChunkTileRows;
            const int n_steps = seg.step_end - seg.step_begin;
            const bool small = rows <= kChunkSmallRows;
            const int first_row = (pair ? stream * kChunkTileRows : 0) + (warp & 3) * (small ? 16 : 32), R = first_row + lane;
            const bool valid = R < rows && (!small || lane < 16), any_valid = first_row < rows;
            // The row sees tokens [0, sink_end) and [from, to), counted along the segment's pages
            int sink_end = 0, from = 0, to = 0;
            const int hi = seg.lo + (rows >> p.log2_g) - 1;
            const ChunkPages g = chunk_pages(p, seg.lo, hi);
            // the last step holds the page in which the sequence ends
            const bool tail = g.n - seg.step_begin * kChunkStepPages <= n_steps * kChunkStepPages && seg.length % kPageSize != 0 && hi / kPageSize == (seg.length - 1) / kPageSize;
            if (valid) {
                const int pos = seg.lo + (R >> p.log2_g), shift = (g.first - g.head) * kPageSize;
                to = pos + 1 - shift;
                if (p.window) {
                    from = (int)max((long long)pos - p.window + 1, 0ll) - shift;
                    sink_end = min(p.n_sink, to);
                    if (from <= sink_end) from = 0;
                }
            }
            float m_ref = -INFINITY, l = 0.f;
            int mine = 0;                                              // works of this stream in the segment
            for (int j = pair ? 0 : stream; j < n_steps; j += pair ? 1 : 2) {
                const int at = (seg.step_begin + j) * kChunkStepTokens;
                wait(c->s_ready[stream], (uint32_t)count & 1u);
                __syncwarp();
                tc_fence_after();
                if (any_valid) {
                    float s[kChunkStepTokens];
                    chunk_load_scores(t_s, s);
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&c->s_free[stream]));
                    const bool masked = __any_sync(0xffffffffu, valid && (to - at < kChunkStepTokens || (from > at && sink_end - at < kChunkStepTokens)));
                    if (masked) {
                        const int n_to = to - at, n_from = from - at, n_sink = sink_end - at;
#pragma unroll
                        for (int i = 0; i < kChunkStepTokens; ++i) s[i] = i < n_to && (i >= n_from || i < n_sink) ? s[i] : -INFINITY;
                    }
                    const float m_step = chunk_row_max(s) * sc;        // -inf: the row sees nothing here
                    const bool lift = m_step > m_ref + kLazyMax;       // always so for the first visible step
                    if (__any_sync(0xffffffffu, lift)) {
                        const float m_new = lift ? m_step : m_ref;
                        const float factor = m_new == -INFINITY ? 1.f : ex2(m_ref - m_new);
                        if (mine > 0) {                                // O follows, once the products issued so far are in it
                            wait(c->pv_done[stream], (uint32_t)(count - 1) & 1u);
                            __syncwarp();
                            tc_fence_after();
#pragma unroll 1
                            for (int i = 0; i < kHeadDim; i += 16) {
                                uint32_t o[16];
                                tmem_ld16(t_o + i, o);
#pragma unroll
                                for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * factor);
                                tmem_st16(t_o + i, o);
                            }
                        }
                        l *= factor;
                        m_ref = m_new;
                    }
                    const float mu = m_ref == -INFINITY ? 0.f : m_ref;
                    uint32_t w[kChunkStepTokens / 2];
                    l += masked ? chunk_weights<false>(s, sc, mu, w) : chunk_weights<true>(s, sc, mu, w);
                    if (count > 0) {                                   // the weights before have been multiplied
                        wait(c->pv_done[stream], (uint32_t)(count - 1) & 1u);
                        __syncwarp();
                        tc_fence_after();
                    }
                    tmem_st16(t_p, *reinterpret_cast<uint32_t(*)[16]>(&w[0]));
                    tmem_st16(t_p + 16, *reinterpret_cast<uint32_t(*)[16]>(&w[16]));
                    tmem_st8(t_p + 32, *reinterpret_cast<uint32_t(*)[8]>(&w[32]));
                    tmem_wait_st();
                } else {
                    if (lane == 0) mbar_arrive(smem_u32(&c->s_free[stream]));
                    // a warp without rows must not run ahead either: its p_ready arrival would count for the step before
                    if (count > 0) wait(c->pv_done[stream], (uint32_t)(count - 1) & 1u);
                }
                if (tail && j == n_steps - 1 && (warp & 3) == 0) {
                    // Rows of V behind the sequence's end may hold anything, and 0 x NaN is NaN: they are set to zero in shared memory before
                    // the product (in a pair by both streams, each before its own).
                    const int v_step = step0 + j, v_slot = (2 * v_step) % kChunkSlots + 1;
                    wait(c->full[v_slot], (uint32_t)(v_step / (kChunkSlots / 2)) & 1u);
                    __syncwarp();
                    unsigned char* v = slots + v_slot * kChunkSlotBytes + (g.n - 1) % kChunkStepPages * kTileBytes;
                    for (int i = lane; i < kTileBytes / 16; i += 32) {         // (group, half of the columns, token of the group, 16 bytes)
                        const int tok = (i >> 7) * 8 + (i >> 3 & 7);
                        if (tok >= seg.length % kPageSize) *reinterpret_cast<uint4*>(v + i * 16) = make_uint4(0, 0, 0, 0);
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&c->p_ready[stream]));
                ++count; ++mine;
            }
            // ---- the part's result: the output of a whole unit, or a state
            if (mine > 0) {
                wait(c->pv_done[stream], (uint32_t)(count - 1) & 1u);
                __syncwarp();
                tc_fence_after();
            }
            float factor0 = 1.f, factor1 = 0.f;                        // of this stream's O and, in solo segments, of the other's
            int col0 = 0, col1 = kHeadDim;
            if (!pair) {
                // both streams hold a part of the rows' state: each warp takes half of the columns of its 32 rows
                tmem_st2(t_p, __float_as_uint(m_ref), __float_as_uint(l));
                tmem_wait_st();
                tc_fence_before();
                pair_barrier(1 + (warp & 3));
                tc_fence_after();
                float2 other;
                tmem_ld2(t_lane + (stream ^ 1) * 256 + kChunkTmemP, other.x, other.y);
                const float m = fmaxf(m_ref, other.x), mu = m == -INFINITY ? 0.f : m;
                factor0 = ex2(m_ref - mu); factor1 = ex2(other.x - mu);
                const float l0 = l * factor0, l1 = other.y * factor1;
                l = stream ? l1 + l0 : l0 + l1;
                m_ref = m;
                col0 = stream * (kHeadDim / 2); col1 = col0 + kHeadDim / 2;
            }
            const long long state = (long long)seg.slot * kChunkUnitRows + R;
            float factor2 = 0.f;                                       // of the state that it joins
            if (joins) {
                float2 prior = make_float2(-INFINITY, 0.f);
                if (valid) prior = *reinterpret_cast<const float2*>(p.part_ml + state * 2);
                if (!pair) pair_barrier(1 + (warp & 3));               // both streams have read it
                const float m = fmaxf(m_ref, prior.x), mu = m == -INFINITY ? 0.f : m, factor = ex2(m_ref - mu);
                factor2 = ex2(prior.x - mu);
                factor0 *= factor; factor1 *= factor;
                l = l * factor + prior.y * factor2;
                m_ref = m;
            }
            if (any_valid) {
                const bool own = mine > 0, both = !pair && n_steps > 1, have = pair ? own : n_steps > 0;
                const uint32_t t_first = pair ? t_o : t_lane + kChunkTmemO, t_second = t_lane + 256 + kChunkTmemO;
                const float f0 = pair || stream == 0 ? factor0 : factor1, f1 = stream == 0 ? factor1 : factor0;
                const bool empty = l == 0.f;                           // (the sum of a query that is not finite is NaN, and so is its result)
                const float inv = !whole ? 1.f : empty ? 0.f : 1.f / l;
                const int tok = seg.tok0 + (R >> p.log2_g), h = (kv_head << p.log2_g) + (R & (p.G - 1));
                const long long cell = (long long)tok * p.hq + h;
#pragma unroll 1
                for (int i = col0; i < col1; i += 32) {
                    float o[32];
                    if (have) {
                        uint32_t u[2][16];
                        tmem_ld16_nowait(t_first + i, u[0]);
                        tmem_ld16_nowait(t_first + i + 16, u[1]);
                        tmem_wait_ld();
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] = __uint_as_float(u[e >> 4][e & 15]) * f0;
                        if (both) {
                            tmem_ld16_nowait(t_second + i, u[0]);
                            tmem_ld16_nowait(t_second + i + 16, u[1]);
                            tmem_wait_ld();
#pragma unroll
                            for (int e = 0; e < 32; ++e) o[e] += __uint_as_float(u[e >> 4][e & 15]) * f1;
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] = 0.f;
                    }
                    if (joins && valid) {
                        const float4* const prior = reinterpret_cast<const float4*>(p.part_o + state * kHeadDim + i);
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float4 x = prior[e];
                            o[4 * e] += x.x * factor2; o[4 * e + 1] += x.y * factor2; o[4 * e + 2] += x.z * factor2; o[4 * e + 3] += x.w * factor2;
                        }
                    }
                    if (valid && whole) {
                        uint32_t v[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) v[e] = empty ? 0u : pack_bf16(o[2 * e] * inv, o[2 * e + 1] * inv);
                        __nv_bfloat16* dst = p.out + cell * kHeadDim + i;
                        if (p.wide_out) {                              // (every lane has a row of its own: the fewer instructions, the better)
                            store_32b(dst, &v[0]);
                            store_32b(dst + 16, &v[8]);
                        } else {
#pragma unroll
                            for (int e = 0; e < 4; ++e) reinterpret_cast<uint4*>(dst)[e] = make_uint4(v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]);
                        }
                    } else if (valid) {
                        // 32-byte stores: each lane has a row of its own, so an instruction touches 32 lines whatever its width
#pragma unroll
                        for (int e = 0; e < 4; ++e) store_32b(p.part_o + state * kHeadDim + i + 8 * e, reinterpret_cast<const uint32_t*>(&o[8 * e]));
                    }
                }
                if (valid && (pair || stream == 0)) {
                    if (!whole) *reinterpret_cast<float2*>(p.part_ml + state * 2) = make_float2(m_ref, l);
                    else if (p.lse) p.lse[cell] = empty ? -INFINITY : (m_ref + log2f(l)) * 0.6931471805599453f;
                }
            }
            tc_fence_before();                                         // O has been read: the next segment's products may replace it
            if (!pair) pair_barrier(1 + (warp & 3));
            __syncwarp();
            step0 += n_steps;
        }
    }
    if (!more_rounds) break;
    __syncthreads();                                                   // everybody has read this round's segments
    }

    if ((warp == kChunkSoftmaxWarps || warp == kChunkSoftmaxWarps + 3) && *late) {      // copies in flight must land before the CTA ends
        const uint64_t last = global_ns() + kWaitBudgetNs;
        int32_t more = 0;
        const int v = warp == kChunkSoftmaxWarps ? 0 : 1;
        for (int i = max(0, loads - kChunkSlots / 2); i < loads; ++i)
            mbar_wait(smem_u32(&c->full[2 * (i % (kChunkSlots / 2)) + v]), (uint32_t)(i / (kChunkSlots / 2)) & 1u, last, &more);
        for (int s = 0; s < 2; ++s)
            if (q_use[s]) mbar_wait(smem_u32(&c->q_full[s]), (uint32_t)(q_use[s] - 1) & 1u, last, &more);
    }
    if (warp == kChunkSoftmaxWarps + 1 || warp == kChunkSoftmaxWarps + 2) {
        if (elect_one()) umma_commit(smem_u32(&c->drained));           // everything issued, whatever happened
        int32_t more = 0;
        mbar_wait(smem_u32(&c->drained), 0, global_ns() + kWaitBudgetNs, &more);
        __syncwarp();
    }
    if (lane == 0 && *late) atomicOr(p.status, 1 << KAP_ERR_TIMEOUT);
    tc_fence_before();
    __syncthreads();
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(512) : "memory");
}

// ---- joins the states of the units that were cut: those of a unit are the last of CTA c - 1, which began it, and the ones of the CTAs from c on as
// long as their cuts lie in it; in step, one for each piece.  A warp takes a row at a time, a lane four columns.
constexpr int kChunkMergeThreads = 256;
struct ChunkStates { long long first, stride, last; int32_t n; };      // slots of a unit's states: first + i stride, the last one apart
__device__ __forceinline__ ChunkStates cut_states(int c, int cuts) {   // cuts c .. c + cuts - 1 lie in the unit
    return {2ll * (c - 1) + 1, 2, 2ll * (c - 1 + cuts), cuts + 1};
}
__device__ __forceinline__ ChunkStates piece_states(const ChunkInStep& v, int of) {
    return {of, v.n_cut, of + (long long)(v.pieces - 1) * v.n_cut, v.pieces};
}
// kRows rows from R on, every `apart`-th, with kBatch states of each in flight; rows from `end` on are left out.
template <int kRows, int kBatch>
__device__ __forceinline__ void chunk_merge_rows(const ChunkParams& p, const ChunkStates& of, int R, int apart, int end, int tok0, int head) {
    const int lane = threadIdx.x & 31;
    Merged acc[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) { acc[r].m = -INFINITY; acc[r].l = 0.f; acc[r].o = make_float4(0.f, 0.f, 0.f, 0.f); }
    for (int i0 = 0; i0 < of.n; i0 += kBatch) {
        float2 ml[kRows][kBatch];
        float4 o[kRows][kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const int i = i0 + j;
            const long long state = (i < of.n - 1 ? of.first + i * of.stride : of.last) * kChunkUnitRows;
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                ml[r][j] = make_float2(-INFINITY, 0.f);
                if (i < of.n && R + r * apart < end) {
                    const long long row = state + R + r * apart;
                    ml[r][j] = __ldcg(reinterpret_cast<const float2*>(p.part_ml + row * 2));
                    o[r][j] = __ldcg(reinterpret_cast<const float4*>(p.part_o + row * kHeadDim) + lane);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
#pragma unroll
            for (int r = 0; r < kRows; ++r)
                if (ml[r][j].y != 0.f) merge_into(acc[r], ml[r][j].x, ml[r][j].y, o[r][j]);
    }
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        const int at = R + r * apart;
        if (at >= end) break;
        const long long cell = (long long)(tok0 + (at >> p.log2_g)) * p.hq + (head << p.log2_g) + (at & (p.G - 1));
        const float inv = acc[r].l == 0.f ? 0.f : 1.f / acc[r].l;
        uint2 v;
        v.x = pack_bf16(acc[r].o.x * inv, acc[r].o.y * inv);
        v.y = pack_bf16(acc[r].o.z * inv, acc[r].o.w * inv);
        *reinterpret_cast<uint2*>(p.out + cell * kHeadDim + lane * 4) = v;
        if (p.lse && lane == 0) p.lse[cell] = acc[r].l == 0.f ? -INFINITY : (acc[r].m + log2f(acc[r].l)) * 0.6931471805599453f;
    }
}

// Many rows: most are in units that one CTA finished.  Block (c, part): 32 rows of the unit in which CTA c begins, if no CTA before it begins in its
// middle (in step: of the c-th unit cut).
constexpr int kChunkMergeRows = 32;
__global__ void __launch_bounds__(kChunkMergeThreads)
kap_chunk_merge_kernel(const ChunkParams p, const int n_cta)
{
    constexpr int kParts = kChunkUnitRows / kChunkMergeRows;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = 1 + blockIdx.x / kParts, row0 = blockIdx.x % kParts * kChunkMergeRows;
    pdl_wait();
    const ChunkInStep in_step = *p.in_step;
    int rows, head, tok0;                                              // the unit's query rows, its KV head and first token row
    ChunkStates states;
    if (in_step.pieces) {
        if (in_step.pieces == 1 || c > in_step.n_cut) return;
        bool bad;
        const ChunkSeq s = chunk_seq(p, in_step.seq, bad);
        const int t = chunk_tiles(p, s.n), u = in_step.whole + c - 1, R = kChunkUnitRows >> p.log2_g, tile = u % t;
        head = u / t; tok0 = s.row0 + tile * R; rows = min(R, s.n - tile * R) << p.log2_g;
        states = piece_states(in_step, c - 1);
    } else {
        const ChunkCut cut = p.cuts[c];
        if (!cut.inside) return;
        const ChunkCut prior = p.cuts[c - 1];
        if (prior.inside && prior.unit == cut.unit) return;
        int n = 1;                                                     // cuts inside the unit
        for (;;) {
            const int i = c + n + lane;
            const bool same = i < n_cta && p.cuts[i].inside && p.cuts[i].unit == cut.unit;
            const uint32_t m = __ballot_sync(0xffffffffu, same);
            const int more = m == 0xffffffffu ? 32 : __ffs(~m) - 1;
            n += more;
            if (more < 32) break;
        }
        rows = cut.rows_head & 0xffff; head = cut.rows_head >> 16; tok0 = cut.tok0;
        states = cut_states(c, n);
    }
    constexpr int kWarps = kChunkMergeThreads / 32, kEach = kChunkMergeRows / kWarps;
    const int end = min(rows, row0 + kChunkMergeRows);
    if (states.n == 2) {                                               // the usual cut: all rows of the warp at once
        chunk_merge_rows<kEach, 2>(p, states, row0 + warp, kWarps, end, tok0, head);
    } else {
        for (int R = row0 + warp; R < end; R += kWarps) chunk_merge_rows<1, 8>(p, states, R, 0, end, tok0, head);
    }
}

// Few rows, most of them in units cut many times: a warp for each (row, head), which finds its unit's states itself.  (50 rows at 4K: the call 27.5 us,
// with blocks for all places where a unit could be cut 31.)
__global__ void __launch_bounds__(kChunkMergeThreads)
kap_chunk_merge_rows_kernel(const ChunkParams p, const int n_cta)
{
    const int lane = threadIdx.x & 31, cell = blockIdx.x * (kChunkMergeThreads / 32) + (threadIdx.x >> 5), row = cell / p.hq, h = cell % p.hq;
    pdl_wait();
    if (row >= p.total_rows) return;
    const ChunkInStep in_step = *p.in_step;
    int lo = 0, hi = p.batch;                                          // the sequence that owns the row, 32 probes at a time
    while (hi - lo > 1) {
        const int step = (hi - lo + 31) / 32, probe = lo + lane * step;
        const uint32_t below = __ballot_sync(0xffffffffu, probe < hi && p.q_indptr[probe] <= row);
        lo += max(31 - __clz(below), 0) * step;
        hi = min(hi, lo + step);
    }
    bool bad;
    const ChunkSeq s = chunk_seq(p, lo, bad);
    if (row < s.row0 || row >= s.row0 + s.n) return;                   // nobody's
    const int R = kChunkUnitRows >> p.log2_g, t = chunk_tiles(p, s.n), tile = (row - s.row0) / R, head = h >> p.log2_g, unit = head * t + tile;
    ChunkStates states;
    if (in_step.pieces) {
        if (in_step.pieces == 1 || unit < in_step.whole) return;
        states = piece_states(in_step, unit - in_step.whole);
    } else {
        int first = 0, n = 0;
        for (int c0 = 1; c0 < n_cta; c0 += 32) {
            const int c = c0 + lane;
            const bool same = c < n_cta && p.cuts[c].inside && p.cuts[c].unit == ((long long)lo << 32 | (unsigned)unit);
            const uint32_t m = __ballot_sync(0xffffffffu, same);
            if (m && n == 0) first = c0 + __ffs(m) - 1;
            n += __popc(m);
        }
        if (n == 0) return;                                            // one CTA did the whole unit
        states = cut_states(first, n);
    }
    const int tok0 = s.row0 + tile * R;
    const int at = ((row - tok0) << p.log2_g) + (h & (p.G - 1));
    chunk_merge_rows<1, 8>(p, states, at, 0, at + 1, tok0, head);
}

}  // namespace kap
