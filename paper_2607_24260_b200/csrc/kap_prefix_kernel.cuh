// Attention over shared prefixes and the sequences' own pages on the tensor cores (tcgen05.mma, accumulators in tensor
// memory): the kernel behind kap_shared_prefix_attn, and the pass that joins its partial states.
//
// Mathematics: flash decoding.  For a tile of up to 128 query rows and steps of 64 tokens,
//     S = Q K^T (128 x 64),   p = 2^(S scale - m),   l += sum p,   O += P V (128 x 128),
// with a lazy reference m: it moves only when a step's maximum exceeds it by more than 8 (weights stay below 256),
// and then l and O are rescaled.  P is rounded to bf16 for the product (the tensor core's operand type; 2^-8 of each weight,
// averaged by the sum); l adds the unrounded weights in fp32, so lse keeps fp32 accuracy.  Segments leave (m, l, O)
// un-normalised in fp32, and states of the same row join as M = max m, l = sum 2^(m_i - M) l_i, O likewise.
//
// Why this split: a prefix unit has up to 256 query rows (64 sequences x 4 heads), 4 x 256 x 128 operations for each 512
// bytes of K and V: 256 operations a byte, right at the B200's balance point, so every K / V byte must be used by both
// row tiles from one copy in shared memory, and the two tiles' softmax must overlap the other's products.  One CTA per SM:
//   warps 0-3, 4-7  softmax of stream 0 and stream 1: one query row per thread (TMEM lane), 64 scores at a time
//   warp 8          TMA: query tiles, then K / V steps through a ring of five 32 KiB stages
//   warps 9, 11     issue the MMAs of stream 0 and stream 1: S of a work before O += P V of the one before it, so scores are
//                   ready before the softmax warps ask for them
//   warp 10         reads the CTA's segment list ahead and hands it to the others through shared memory
// A pair segment gives each stream its own row tile and both the same K / V stage; a solo segment (at most 128 rows)
// alternates its steps between the streams.  Tensor memory: 512 columns, per stream two S / P buffers of 64 columns (the
// weights overwrite the scores they came from) and O (128).
//
// Bounds on one step of a pair: 8 S products of 128 x 64 x 16 read 6 KiB of shared memory each, 48 cycles at 128 B a
// cycle, and 4 P V products of 128 x 128 x 16 take 64 cycles: 640 cycles a tile, 1280 a pair (6550 operations a cycle, 80 % of
// the dense rate); 2 x 128 x 64 exponentials take 1024 cycles of the SM's 16 a cycle.
//
// Every wait on an mbarrier is bounded; when one runs out the CTA sets KAP_ERR_TIMEOUT, the roles drain, copies and
// products in flight are waited for (bounded again), tensor memory is freed and the kernel returns.
#pragma once

#include "kap_prefix.h"
#include "kap_ptx.cuh"

namespace kap {

constexpr int kPfxThreads = 384;
constexpr int kPfxStages = 5;
constexpr int kPfxPlaneBytes = kPrefixStepTokens * 128;                // 64 tokens x 64 columns: 8 KiB
constexpr int kPfxStageBytes = 4 * kPfxPlaneBytes;                     // K columns 0-63 | 64-127 | V likewise
constexpr int kPfxQHalfBytes = kPrefixTileRows * 128;                  // 128 rows x 64 columns: 16 KiB
constexpr int kPfxQBytes = 2 * kPfxQHalfBytes;
constexpr int kPfxSegRing = 16, kPfxSegHalf = 8;

struct PfxDesc {                                                       // a segment as the roles use it
    int32_t kv_head, flags, tok_row0, rows;
    int32_t n_steps;                                                   // steps to do (the context may be shorter than the list)
    int32_t first_token, end_token;                                    // of the segment's first step; end of what may be seen
    int32_t list_at, n_pages;                                          // block-table entries from list_at on
    int32_t own_seen;                                                  // own parts: tokens that the sequence's first row sees
    int32_t state_row0;
    int32_t ctx;                                                       // own parts: ctx_len (V rows from there on are cleared)
    int32_t pad[4];
};
struct PfxControl {
    PfxDesc seg[kPfxSegRing];
    unsigned long long seg_full[2], seg_free[2];
    unsigned long long kv_full[kPfxStages], kv_free[kPfxStages];
    unsigned long long q_full[2], q_free[2];
    unsigned long long s_ready[4], p_ready[4], pv_done[4];             // [stream * 2 + buffer]
    unsigned long long drained[2];
    uint32_t tmem_base;
    int32_t timed_out;
};
constexpr int kPfxCtlBytes = 2048;
static_assert(sizeof(PfxControl) <= kPfxCtlBytes, "control block too large");
constexpr int kPfxSmemBytes = 2 * kPfxQBytes + kPfxStages * kPfxStageBytes + kPfxCtlBytes;
static_assert(kPfxSmemBytes <= 232448, "more than 227 KiB of shared memory");

struct PfxParams {
    const PrefixSegment* segments;
    const int32_t* cta_begin;
    const PrefixSeq* seqs;
    const PrefixRow* row_map;
    const PrefixUnit* units;
    const int32_t *q_indptr, *bt_indptr, *bt_pages, *ctx_len;
    float *part_o, *part_ml;
    __nv_bfloat16* out;
    float* lse;
    int32_t* status;
    long long num_pool_pages;
    int32_t batch, total_rows, hq, hkv, G, nhd;
    float scale_log2;
};

// Which stream a segment begins with: not the one that the segment before it ended with, so that runs of short segments keep
// both streams busy.
struct PfxOrder {
    int last = 1;
    __device__ __forceinline__ int begin() const { return last ^ 1; }
    __device__ __forceinline__ void done(bool pair, int n_steps) {     // after a segment
        if (n_steps > 0) last = pair ? begin() ^ 1 : begin() ^ ((n_steps - 1) & 1);
    }
};

template <bool kNhd>
__global__ void __launch_bounds__(kPfxThreads, 1)
kap_prefix_kernel(const __grid_constant__ CUtensorMap kv_map, const __grid_constant__ CUtensorMap q_map, const PfxParams p)
{
    extern __shared__ unsigned char smem_raw[];
    if (smem_u32(smem_raw) & 1023u) {                                  // the tiles need it; no static shared memory, so it holds
        if (threadIdx.x == 0) atomicOr(p.status, 1 << KAP_ERR_DEVICE_INDEX);
        return;
    }
    unsigned char* const q_tiles = smem_raw;
    unsigned char* const stages = smem_raw + 2 * kPfxQBytes;
    PfxControl* const c = reinterpret_cast<PfxControl*>(stages + kPfxStages * kPfxStageBytes);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&c->seg_full[i]), 1);
            mbar_init(smem_u32(&c->seg_free[i]), 11);                  // eight softmax warps, the TMA warp, two MMA warps
            mbar_init(smem_u32(&c->q_full[i]), 1);
            mbar_init(smem_u32(&c->q_free[i]), 2);                     // both MMA warps
            mbar_init(smem_u32(&c->drained[i]), 1);
        }
        for (int i = 0; i < kPfxStages; ++i) { mbar_init(smem_u32(&c->kv_full[i]), 1); mbar_init(smem_u32(&c->kv_free[i]), 2); }
        for (int i = 0; i < 4; ++i) {
            mbar_init(smem_u32(&c->s_ready[i]), 1);
            mbar_init(smem_u32(&c->p_ready[i]), 4);
            mbar_init(smem_u32(&c->pv_done[i]), 1);
        }
        c->timed_out = 0;
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
    const uint64_t deadline = global_ns() + kWaitBudgetNs;
    volatile int32_t* const late = &c->timed_out;
    const int seg0 = p.cta_begin[blockIdx.x], n_seg = p.cta_begin[blockIdx.x + 1] - seg0;
    auto wait = [&](unsigned long long& bar, uint32_t parity) { return mbar_wait(smem_u32(&bar), parity, deadline, late); };
    // segment k of this CTA, for the warps that consume the list (whole warps, converged)
    auto open_segment = [&](int k, PfxDesc& d) {
        const bool ok = (k & (kPfxSegHalf - 1)) != 0 || wait(c->seg_full[(k / kPfxSegHalf) & 1], (uint32_t)(k / kPfxSegRing) & 1u);
        if (__all_sync(0xffffffffu, ok)) d = c->seg[k % kPfxSegRing];
        return __all_sync(0xffffffffu, ok) != 0;
    };
    auto close_segment = [&](int k) {
        __syncwarp();
        if (lane == 0 && ((k & (kPfxSegHalf - 1)) == kPfxSegHalf - 1 || k == n_seg - 1)) mbar_arrive(smem_u32(&c->seg_free[(k / kPfxSegHalf) & 1]));
    };

    if (warp == 10) {
        // ---- segment list: eight at a time, one per lane
        for (int k0 = 0; k0 < n_seg; k0 += kPfxSegHalf) {
            const int half = (k0 / kPfxSegHalf) & 1;
            bool ok = k0 < kPfxSegRing || wait(c->seg_free[half], (uint32_t)(k0 / kPfxSegRing - 1) & 1u);
            if (!__all_sync(0xffffffffu, ok)) break;
            if (lane < kPfxSegHalf && k0 + lane < n_seg) {
                const PrefixSegment s = p.segments[seg0 + k0 + lane];
                const int at = p.bt_indptr[s.seq], listed = p.bt_indptr[s.seq + 1] - at;
                const int ctx = p.ctx_len[s.seq];
                const bool prefix = s.flags & kSegPrefix;
                int n_pages = min(s.n_pages, listed - s.first_page);
                if (!prefix)                                           // pages that hold nothing yet are not read
                    n_pages = min(n_pages, max(ctx, 0) / kPageSize + (max(ctx, 0) % kPageSize ? 1 : 0) - s.first_page);
                else if (n_pages < s.n_pages)
                    atomicOr(p.status, 1 << KAP_ERR_DEVICE_INDEX);
                n_pages = max(n_pages, 0);
                PfxDesc d;
                d.kv_head = s.kv_head; d.flags = s.flags; d.tok_row0 = s.tok_row0; d.rows = s.rows;
                d.n_steps = max(0, min(s.step_end, (n_pages + kPrefixStepPages - 1) / kPrefixStepPages) - s.step_begin);
                d.first_token = (s.first_page + s.step_begin * kPrefixStepPages) * kPageSize;
                d.list_at = at + s.first_page + s.step_begin * kPrefixStepPages;
                d.n_pages = max(0, min(n_pages, s.step_end * kPrefixStepPages) - s.step_begin * kPrefixStepPages);
                d.end_token = d.first_token + d.n_pages * kPageSize;
                d.own_seen = ctx - s.n_q + 1; d.ctx = ctx;
                d.state_row0 = s.state_row0;
                d.pad[0] = d.pad[1] = d.pad[2] = d.pad[3] = 0;
                c->seg[(k0 + lane) % kPfxSegRing] = d;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&c->seg_full[half]));
        }
    } else if (warp == 8) {
        // ---- TMA: lane 2 i + h copies columns 64 h .. of page i of the step (K, then V)
        uint64_t once, keep;
        asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(once));
        asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(keep));
        int step = 0, q_use[2] = {0, 0}, q_slot = 0;
        bool ok = true;
        for (int k = 0; k < n_seg && ok; ++k) {
            PfxDesc d;
            if (!(ok = open_segment(k, d))) break;
            if (d.n_steps > 0) {
                const bool pair = d.flags & kSegPair;
                const uint64_t policy = d.flags & kSegPrefix ? keep : once;
                for (int t = 0; t < (pair ? 2 : 1) && ok; ++t) {
                    const int slot = pair ? t : q_slot;
                    ok = q_use[slot] == 0 || wait(c->q_free[slot], (uint32_t)(q_use[slot] - 1) & 1u);
                    ok = __all_sync(0xffffffffu, ok);
                    if (ok && lane == 0) {
                        const uint32_t bar = smem_u32(&c->q_full[slot]), dst = smem_u32(q_tiles + slot * kPfxQBytes);
                        const int tok = d.tok_row0 + t * (kPrefixTileRows / p.G);
                        mbar_expect_tx(bar, kPfxQBytes);
                        tma_load_3d(dst, &q_map, 0, d.kv_head * p.G, tok, bar, keep);
                        tma_load_3d(dst + kPfxQHalfBytes, &q_map, 64, d.kv_head * p.G, tok, bar, keep);
                    }
                    ++q_use[slot];
                }
                if (!pair) q_slot ^= 1;
                int32_t ids = 0, next_ids = lane < d.n_pages ? p.bt_pages[d.list_at + lane] : 0;   // 32 pages at a time, one batch ahead
                for (int j = 0; j < d.n_steps && ok; ++j, ++step) {
                    if ((j & 7) == 0) {
                        ids = next_ids;
                        const int ahead = (j + 8) * kPrefixStepPages + lane;
                        next_ids = ahead < d.n_pages ? p.bt_pages[d.list_at + ahead] : 0;
                        if (ids < 0 || ids >= p.num_pool_pages) { ids = 0; atomicOr(p.status, 1 << KAP_ERR_DEVICE_INDEX); }
                    }
                    const int stage = step % kPfxStages, use = step / kPfxStages;
                    ok = use == 0 || wait(c->kv_free[stage], (uint32_t)(use - 1) & 1u);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    const int n = min(kPrefixStepPages, d.n_pages - j * kPrefixStepPages);
                    const uint32_t bar = smem_u32(&c->kv_full[stage]);
                    if (lane == 0) mbar_expect_tx(bar, (uint32_t)n * kPageHeadBytes);
                    const int i = (lane >> 1) & 3, h = lane & 1, v = lane >> 3;        // page, half, K or V
                    const int32_t page = __shfl_sync(0xffffffffu, ids, (j & 7) * kPrefixStepPages + i);
                    __syncwarp();
                    if (lane < 16 && i < n) {
                        const uint32_t dst = smem_u32(stages + stage * kPfxStageBytes + (2 * v + h) * kPfxPlaneBytes + i * kHalfTileBytes);
                        if (kNhd) tma_load_3d(dst, &kv_map, h * 64, d.kv_head, (page * 2 + v) * kPageSize, bar, policy);
                        else tma_load_2d(dst, &kv_map, h * 64, ((page * 2 + v) * p.hkv + d.kv_head) * kPageSize, bar, policy);
                    }
                }
            }
            close_segment(k);
        }
        if (*late) {                                                   // copies in flight must land before the CTA ends
            const uint64_t last = global_ns() + kWaitBudgetNs;
            int32_t more = 0;
            for (int s = max(0, step - kPfxStages); s < step; ++s) mbar_wait(smem_u32(&c->kv_full[s % kPfxStages]), (uint32_t)(s / kPfxStages) & 1u, last, &more);
            for (int s = 0; s < 2; ++s)
                if (q_use[s]) mbar_wait(smem_u32(&c->q_full[s]), (uint32_t)(q_use[s] - 1) & 1u, last, &more);
        }
    } else if (warp == 9 || warp == 11) {
        // ---- tensor core: one warp per stream, because a group of products keeps its issuer waiting for about as long as
        // they take (the queue is short), so whatever the issuer does in between is lost unless another one issues then.
        // The whole warp walks along with warp-uniform values (operands computed by a single lane have to be moved to the
        // uniform registers for every product); one elected lane issues.
        const int stream = warp == 9 ? 0 : 1;
        constexpr uint32_t idesc_s = umma_idesc(kPrefixTileRows, kPrefixStepTokens, false), idesc_o = umma_idesc(kPrefixTileRows, kHeadDim, true);
        // descriptors of the first query tile, of K and of V in the first stage; other places add their distance / 16
        const uint64_t q_desc = umma_smem_desc(smem_u32(q_tiles), 16, 1024), k_desc = umma_smem_desc(smem_u32(stages), 16, 1024);
        // V: 16 tokens (K) x 128 columns (N), N contiguous; columns 64-127 one plane further, 8 tokens = 1 KiB
        const uint64_t v_desc = umma_smem_desc(smem_u32(stages) + 2 * kPfxPlaneBytes, kPfxPlaneBytes, 1024);
        const uint32_t t_s = tmem + stream * 256, t_o = t_s + 128;
        int stage = 0, q_slot = 0, count = 0;
        uint32_t stage_parity = 0, q_parity = 0;                       // of the ring; bit i: of query slot i
        int held = -1, held_pages = 0, held_first = 0;                 // stage of the work whose P V is still to be issued
        bool ok = true;
        PfxOrder order;
        auto all_wait = [&](unsigned long long& bar, uint32_t parity) { return __all_sync(0xffffffffu, wait(bar, parity)) != 0; };
        auto issue_pv = [&](int n) {                                   // of work n, the held one
            const int b = stream * 2 + (n & 1);
            if (!all_wait(c->p_ready[b], (uint32_t)(n >> 1) & 1u)) return false;
            tc_fence_after();
            const uint64_t v = v_desc + (uint32_t)held * (kPfxStageBytes / 16);
            const uint32_t s = t_s + (n & 1) * 64;
            if (elect_one()) {
#pragma unroll
                for (int pg = 0; pg < kPrefixStepPages; ++pg)
                    if (pg < held_pages) umma_ts(t_o, s + pg * 8, v + pg * (kHalfTileBytes / 16), idesc_o, !held_first || pg > 0);
                umma_commit(smem_u32(&c->pv_done[b]));
                umma_commit(smem_u32(&c->kv_free[held]));
            }
            __syncwarp();
            held = -1;
            return true;
        };
        auto issue_s = [&](int n, int slot) {
            const int b = stream * 2 + (n & 1);
            // the weights of work n - 2 lie over this buffer: its products must be done
            if (n >= 2 && !all_wait(c->pv_done[b], (uint32_t)((n - 2) >> 1) & 1u)) return false;
            tc_fence_after();
            const uint64_t q = q_desc + (uint32_t)slot * (kPfxQBytes / 16), kd = k_desc + (uint32_t)stage * (kPfxStageBytes / 16);
            const uint32_t s = t_s + (n & 1) * 64;
            if (elect_one()) {
#pragma unroll
                for (int ks = 0; ks < 8; ++ks)
                    umma_ss(s, q + ((ks >> 2) * kPfxQHalfBytes + (ks & 3) * 32) / 16, kd + ((ks >> 2) * kPfxPlaneBytes + (ks & 3) * 32) / 16,
                            idesc_s, ks > 0);
                umma_commit(smem_u32(&c->s_ready[b]));
            }
            __syncwarp();
            return true;
        };
        for (int k = 0; k < n_seg && ok; ++k) {
            PfxDesc d;
            if (!(ok = open_segment(k, d))) break;
            const int n_steps = __shfl_sync(0xffffffffu, d.n_steps, 0), n_pages = __shfl_sync(0xffffffffu, d.n_pages, 0);
            const int pair = __shfl_sync(0xffffffffu, d.flags & kSegPair, 0) ? 1 : 0;
            if (n_steps > 0) {
                const int start = order.begin(), slot = pair ? stream : q_slot, used = pair ? 3 : 1 << q_slot;
                // both issuers wait for every query tile and every stage, and both give each back: what one does not use
                // itself it gives back at once
                for (int i = 0; i < 2 && ok; ++i)
                    if (used >> i & 1) ok = all_wait(c->q_full[i], (q_parity >> i) & 1u);
                int mine = 0;
                for (int j = 0; j < n_steps && ok; ++j) {
                    ok = all_wait(c->kv_full[stage], stage_parity);
                    if (!ok) break;
                    if (pair || (start ^ (j & 1)) == stream) {
                        ok = issue_s(count, slot);
                        if (ok && held >= 0) ok = issue_pv(count - 1);
                        if (!ok) break;
                        held = stage; held_pages = min(kPrefixStepPages, n_pages - j * kPrefixStepPages); held_first = mine == 0;
                        ++count; ++mine;
                    } else if (elect_one()) {
                        mbar_arrive(smem_u32(&c->kv_free[stage]));
                    }
                    __syncwarp();
                    if (++stage == kPfxStages) { stage = 0; stage_parity ^= 1u; }
                }
                if (ok && elect_one()) {                               // the query tiles may be replaced when these products are done
                    umma_commit(smem_u32(&c->q_free[slot]));
                    if (pair) umma_commit(smem_u32(&c->q_free[slot ^ 1]));
                }
                __syncwarp();
                if (ok && held >= 0) ok = issue_pv(count - 1);         // nothing of the next segment can be scored meanwhile: O is read first
                q_parity ^= used;
                if (!pair) q_slot ^= 1;
                order.done(pair, n_steps);
            }
            close_segment(k);
        }
        if (elect_one()) umma_commit(smem_u32(&c->drained[stream]));   // everything issued, whatever happened
        int32_t more = 0;
        mbar_wait(smem_u32(&c->drained[stream]), 0, global_ns() + kWaitBudgetNs, &more);
        __syncwarp();
    } else if (warp < 8) {
        // ---- softmax: stream = warp group, one query row per thread
        const int stream = warp >> 2, r = (warp & 3) * 32 + lane;
        const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16) + stream * 256;
        const float sc = p.scale_log2;
        int step = 0, count = 0;
        bool ok = true;
        PfxOrder order;
        for (int k = 0; k < n_seg && ok; ++k) {
            PfxDesc d;
            if (!(ok = open_segment(k, d))) break;
            const bool pair = d.flags & kSegPair;
            const int start = order.begin();
            const int tile = pair ? stream : 0;                        // pair segments: tile t belongs to stream t
            const int R = tile * kPrefixTileRows + r;
            const bool valid = R < d.rows, any_valid = tile * kPrefixTileRows + (warp & 3) * 32 < d.rows;
            // tokens below `seen` are visible to this row
            int seen = 0;
            if (valid) {
                if (d.flags & kSegPrefix) {
                    const PrefixRow row = p.row_map[d.tok_row0 + R / p.G];
                    seen = p.ctx_len[row.seq] + row.back;
                } else {
                    seen = d.own_seen + R / p.G;
                }
                seen = min(seen, d.end_token);
            }
            float m_ref = -INFINITY, l = 0.f;
            int mine = 0;                                              // works of this stream in the segment
            for (int j = 0; j < d.n_steps && ok; ++j, ++step) {
                if (!pair && (start ^ (j & 1)) != stream) continue;
                const int b = stream * 2 + (count & 1);
                const uint32_t s_at = lanes + (count & 1) * 64;
                const int tok0 = d.first_token + j * kPrefixStepTokens;
                ok = wait(c->s_ready[b], (uint32_t)(count >> 1) & 1u);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc_fence_after();
                if (!(d.flags & kSegPrefix) && (warp & 3) == 0 && tok0 + kPrefixStepTokens > d.ctx) {
                    // value rows behind the context may hold anything (even NaN, which 0 x NaN would spread): clear those of
                    // the last page (later pages are not multiplied)
                    const int from = d.ctx - tok0, to = min(kPrefixStepTokens, (from + kPageSize - 1) / kPageSize * kPageSize);
                    const int stage = step % kPfxStages;
                    ok = wait(c->kv_full[stage], (uint32_t)(step / kPfxStages) & 1u);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    unsigned char* v = stages + stage * kPfxStageBytes + 2 * kPfxPlaneBytes + (lane >> 3 & 1) * kPfxPlaneBytes + (lane & 7) * 16;
                    for (int t = max(from, 0) + (lane >> 4); t < to; t += 2) *reinterpret_cast<uint4*>(v + t * 128) = make_uint4(0, 0, 0, 0);
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                }
                if (any_valid) {
                    uint32_t u[4][16];
#pragma unroll
                    for (int i = 0; i < 4; ++i) tmem_ld16_nowait(s_at + i * 16, u[i]);
                    tmem_wait_ld();
                    float s[kPrefixStepTokens];
#pragma unroll
                    for (int i = 0; i < kPrefixStepTokens; ++i) s[i] = __uint_as_float(u[i >> 4][i & 15]);
                    if (__any_sync(0xffffffffu, tok0 + kPrefixStepTokens > seen)) {
                        const int n = seen - tok0;
#pragma unroll
                        for (int i = 0; i < kPrefixStepTokens; ++i) s[i] = i < n ? s[i] : -INFINITY;
                    }
                    float mx[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
                    for (int i = 4; i < kPrefixStepTokens; ++i) mx[i & 3] = fmaxf(mx[i & 3], s[i]);
                    const float m_step = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * sc;   // -inf: the row sees nothing here
                    const bool lift = m_step > m_ref + kLazyMax;       // always so for the first visible step
                    if (__any_sync(0xffffffffu, lift)) {
                        const float m_new = lift ? m_step : m_ref;
                        const float factor = m_new == -INFINITY ? 1.f : ex2(m_ref - m_new);
                        if (mine > 0) {                                // O follows, once the products issued so far are in it
                            const int pc = count - 1;
                            ok = wait(c->pv_done[stream * 2 + (pc & 1)], (uint32_t)(pc >> 1) & 1u);
                            ok = __all_sync(0xffffffffu, ok);
                            if (!ok) break;
                            tc_fence_after();
#pragma unroll 1
                            for (int i = 0; i < kHeadDim; i += 16) {
                                uint32_t o[16];
                                tmem_ld16(lanes + 128 + i, o);
#pragma unroll
                                for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * factor);
                                tmem_st16(lanes + 128 + i, o);
                            }
                            tmem_wait_st();
                        }
                        l *= factor;
                        m_ref = m_new;
                    }
                    const float mu = m_ref == -INFINITY ? 0.f : m_ref;
                    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint32_t w[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const float a = ex2(fmaf(s[h * 32 + 2 * e], sc, -mu)), b2 = ex2(fmaf(s[h * 32 + 2 * e + 1], sc, -mu));
                            sum[(2 * e) & 3] += a;
                            sum[(2 * e + 1) & 3] += b2;
                            w[e] = pack_bf16(a, b2);
                        }
                        tmem_st16(s_at + h * 16, w);
                    }
                    l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
                    tmem_wait_st();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&c->p_ready[b]));
                ++count; ++mine;
            }
            if (!ok) break;
            // ---- the segment's state: pair segments one for all rows, solo segments one per stream (the second may be empty)
            const bool writes = pair || stream == start || (d.flags & kSegTwoStates);
            if (mine > 0) {
                const int pc = count - 1;
                ok = wait(c->pv_done[stream * 2 + (pc & 1)], (uint32_t)(pc >> 1) & 1u);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc_fence_after();
            }
            if (writes && any_valid) {
                const long long row = (long long)d.state_row0 + (!pair && stream != start ? d.rows : 0) + R;
                if (mine > 0) {
#pragma unroll 1
                    for (int i = 0; i < kHeadDim; i += 16) {
                        uint32_t o[16];
                        tmem_ld16(lanes + 128 + i, o);
                        if (valid) {
                            uint4* dst = reinterpret_cast<uint4*>(p.part_o + row * kHeadDim + i);
#pragma unroll
                            for (int e = 0; e < 4; ++e) dst[e] = make_uint4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
                        }
                    }
                }
                if (valid) *reinterpret_cast<float2*>(p.part_ml + row * 2) = make_float2(m_ref, l);
            }
            tc_fence_before();                                         // O has been read: the next segment's products may replace it
            order.done(pair, d.n_steps);
            close_segment(k);
        }
    }
    if (lane == 0 && *late) atomicOr(p.status, 1 << KAP_ERR_TIMEOUT);
    tc_fence_before();
    __syncthreads();
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(512) : "memory");
}

// ---- joins the states of every (query row, head): one warp each, a lane holds four columns.  Bound by latency and by the
// states' bytes (520 each, mostly still in L2).
__global__ void __launch_bounds__(128)
kap_prefix_merge_kernel(const PfxParams p)
{
    const int lane = threadIdx.x & 31;
    const long long cell = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (cell >= (long long)p.total_rows * p.hq) { pdl_wait(); return; }
    const int row = (int)(cell / p.hq), head = (int)(cell % p.hq), g = head / p.G, h = head % p.G;
    const PrefixRow where = p.row_map[row];                            // the schedule's arrays: final before the kernel in front
    const PrefixSeq s = p.seqs[where.seq];
    int n[2] = {0, 0};
    long long at[2] = {0, 0};
    int stride[2] = {0, 0};
    if (s.prefix_unit0 >= 0) {
        const int R = (row - s.group_row0) * p.G + h;
        const PrefixUnit u = p.units[s.prefix_unit0 + g * s.n_pairs + R / kPrefixUnitRows];
        n[0] = u.n_states; stride[0] = u.rows; at[0] = u.state_row0 + R % kPrefixUnitRows;
    }
    if (s.own_unit0 >= 0) {
        const PrefixUnit u = p.units[s.own_unit0 + g];
        n[1] = u.n_states; stride[1] = u.rows; at[1] = u.state_row0 + (row - s.row0) * p.G + h;
    }
    pdl_wait();
    // not the scheduled rows, or a context that outgrew the schedule or its block table
    if (lane == 0) {
        const int most = min(s.list_pages, p.bt_indptr[where.seq + 1] - p.bt_indptr[where.seq]);
        if (p.q_indptr[where.seq] != s.row0 || p.ctx_len[where.seq] > (long long)most * kPageSize) atomicOr(p.status, 1 << KAP_ERR_DEVICE_INDEX);
    }
    Merged acc; acc.m = -INFINITY; acc.l = 0.f; acc.o = make_float4(0.f, 0.f, 0.f, 0.f);
    const int total = n[0] + n[1];
    constexpr int kBatch = 8;
    for (int i0 = 0; i0 < total; i0 += kBatch) {
        float2 ml[kBatch];
        float4 o[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const int i = min(i0 + j, total - 1), part = i < n[0] ? 0 : 1;
            const long long r = at[part] + (long long)(i - part * n[0]) * stride[part];
            ml[j] = __ldcg(reinterpret_cast<const float2*>(p.part_ml + r * 2));
            o[j] = __ldcg(reinterpret_cast<const float4*>(p.part_o + r * kHeadDim) + lane);
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
            if (i0 + j < total && ml[j].y > 0.f) merge_into(acc, ml[j].x, ml[j].y, o[j]);   // an empty state's O was never written
    }
    const float inv = acc.l > 0.f ? 1.f / acc.l : 0.f;
    uint2 v;
    v.x = pack_bf16(acc.o.x * inv, acc.o.y * inv);
    v.y = pack_bf16(acc.o.z * inv, acc.o.w * inv);
    *reinterpret_cast<uint2*>(p.out + cell * kHeadDim + lane * 4) = v;
    if (p.lse && lane == 0) p.lse[cell] = acc.l > 0.f ? (acc.m + log2f(acc.l)) * 0.6931471805599453f : -INFINITY;
}

}  // namespace kap
