// Attention of many query rows over a shared prefix on the tensor cores (tcgen05.mma, accumulators in tensor memory), and the
// pass that joins the partial states of kap_shared_prefix_attn.
//
// Mathematics: flash decoding.  For a tile of up to 128 query rows and steps of 80 tokens,
//     S = Q K^T (128 x 80),   p = 2^(S scale - m),   l += sum p,   O += P V (128 x 128),
// with a lazy reference m: it moves only when a step's maximum exceeds it by more than 8 (weights stay below 256),
// and then l and O are rescaled.  P is rounded to bf16 for the product (the tensor core's operand type; 2^-8 of each weight,
// averaged by the sum); l adds the unrounded weights in fp32, so lse keeps fp32 accuracy.  Segments leave (m, l, O)
// un-normalised in fp32, and states of the same row join as M = max m, l = sum 2^(m_i - M) l_i, O likewise.
//
// Why this split: a block has up to 256 query rows (64 sequences x 4 heads), 4 x 256 x 128 operations for each 512 bytes of K
// and V: 256 operations a byte, right at the B200's balance point, so every K / V byte must be used by both row tiles
// from one copy in shared memory, and the two tiles' softmax must overlap each other's products.  One CTA per SM:
//   warps 0-3, 4-7  softmax of stream 0 and stream 1: one query row per thread (TMEM lane), 80 scores at a time
//   warp 8          TMA: query tiles, then K and V tiles through a ring of eight 20 KiB slots (four steps)
//   warp 9          issues the MMAs, for the two streams in turn: S of a step, then O += P V of the step before
// A pair segment gives each stream its own row tile and both the same K and V; a solo segment (at most 128 rows) alternates its
// steps between the streams.  Tensor memory, 256 of the 512 columns per stream: S (80), P (40), O (128).  Steps of 80 tokens are
// the longest whose weights fit beside the scores: S of the next step overwrites S as soon as it has been read, not only when
// P V has drained (with P over S in steps of 128 the tensor core idled 390 cycles a step waiting for that, or, with an issuer per
// stream, both streams drifted into step and took turns: 3970 and 4430 cycles for 128 tokens of a pair).
//
// Bounds on a step of a pair: a product 128 x 80 x 16 reads 6.5 KiB of shared memory, 51 cycles, eight of them 408; P V 320: 1456
// cycles for both; 2 x 128 x 80 exponentials take 1280 cycles of the SM's 16 a cycle, 960 with a quarter on the FMA pipe.
//
// Every wait on an mbarrier is bounded; when one runs out the CTA sets KAP_ERR_TIMEOUT, later waits return at once, the roles run
// to their end inside this CTA's shared and tensor memory, copies and products in flight are waited for (bounded again),
// tensor memory is freed and the kernel returns.
#pragma once

#include "kap_prefix.h"
#include "kap_ptx.cuh"

namespace kap {

constexpr int kPfxThreads = 384;
constexpr int kPfxSlots = 8;                                           // step n: K in slot 2 n, V in slot 2 n + 1 (mod 8)
constexpr int kPfxPlaneBytes = kPrefixStepTokens * 128;                // 80 tokens x 64 columns: 10 KiB
constexpr int kPfxSlotBytes = 2 * kPfxPlaneBytes;                      // columns 0-63 | 64-127
constexpr int kPfxQHalfBytes = kPrefixTileRows * 128;                  // 128 rows x 64 columns: 16 KiB
constexpr int kPfxQBytes = 2 * kPfxQHalfBytes;
constexpr int kPfxTmemP = 80, kPfxTmemO = 128;                         // columns of a stream's 256; S from 0
static_assert(kPfxPlaneBytes % 1024 == 0 && kPrefixStepTokens % 16 == 0 && kPfxTmemP >= kPrefixStepTokens &&
              kPfxTmemP + kPrefixStepTokens / 2 <= kPfxTmemO && kPfxSlots % 2 == 0, "tile geometry");

struct PfxControl {
    unsigned long long full[kPfxSlots], free[kPfxSlots];
    unsigned long long q_full[2], q_free[2];
    unsigned long long s_ready[2], s_free[2], p_ready[2], pv_done[2];  // [stream]
    unsigned long long drained;
    uint32_t tmem_base;
    int32_t timed_out;
};
constexpr int kPfxCtlBytes = 1024;
static_assert(sizeof(PfxControl) <= kPfxCtlBytes, "control block too large");
constexpr int kPfxSmemBytes = 2 * kPfxQBytes + kPfxSlots * kPfxSlotBytes + kPfxCtlBytes;
static_assert(kPfxSmemBytes <= 232448, "more than 227 KiB of shared memory");

struct PfxParams {
    const PrefixSegment* segments;
    const int32_t* cta_begin;
    const PrefixSeq* seqs;
    const PrefixRow* row_map;
    const PrefixUnit* units;
    const int32_t *q_indptr, *bt_indptr, *bt_pages, *ctx_len;
    const int32_t* q_end;                                              // the caller's row count, q_indptr[batch]
    float *part_o, *part_ml;
    __nv_bfloat16* out;
    float* lse;
    int32_t* status;
    long long num_pool_pages;
    int32_t total_rows, hq, hkv, G;
    float scale_log2;
};

// n scores of one row; with `masked` those from token n_seen on become -inf
template <int n>
__device__ __forceinline__ void mask_scores(float (&s)[n], int n_seen) {
#pragma unroll
    for (int i = 0; i < n; ++i) s[i] = i < n_seen ? s[i] : -INFINITY;
}
__device__ __forceinline__ void load_scores(uint32_t at, float (&s)[kPrefixStepTokens]) {
    uint32_t u[kPrefixStepPages][16];
#pragma unroll
    for (int i = 0; i < kPrefixStepPages; ++i) tmem_ld16_nowait(at + i * 16, u[i]);
    tmem_wait_ld();
#pragma unroll
    for (int i = 0; i < kPrefixStepTokens; ++i) s[i] = __uint_as_float(u[i >> 4][i & 15]);
}
__device__ __forceinline__ float row_max(const float (&s)[kPrefixStepTokens]) {
    float mx[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
    for (int i = 4; i + 8 <= kPrefixStepTokens; i += 8)
#pragma unroll
        for (int e = 0; e < 4; ++e) mx[e] = max3(mx[e], s[i + e], s[i + 4 + e]);
#pragma unroll
    for (int e = 0; e < 4; ++e) mx[e] = fmaxf(mx[e], s[kPrefixStepTokens - 4 + e]);
    return fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
}
// The weights 2^(s scale - mu) as packed bf16; returns their fp32 sum.  The SM's 16 exponentials a cycle bound this part, so with
// kPoly one pair in kPolyEvery is computed on the FMA pipe instead (3 % on a long prefix of 256 rows).  That gives at least 2^-126
// where 2^-inf = 0 is wanted, so steps with masked scores do without it.
constexpr int kPolyEvery = 4;
template <bool kPoly>
__device__ __forceinline__ float weights(const float (&s)[kPrefixStepTokens], float scale, float mu, uint32_t (&w)[kPrefixStepTokens / 2]) {
    const uint64_t sc2 = pack_f32x2(scale, scale), mu2 = pack_f32x2(-mu, -mu);
    uint64_t sum[2] = {0ull, 0ull};
#pragma unroll
    for (int e = 0; e < kPrefixStepTokens / 2; ++e) {
        const uint64_t x = fma_f32x2(pack_f32x2(s[2 * e], s[2 * e + 1]), sc2, mu2);
        float a, b;
        if (kPoly && e % kPolyEvery == kPolyEvery - 1) {
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

template <bool kNhd>
__global__ void __launch_bounds__(kPfxThreads, 1)
kap_prefix_kernel(const __grid_constant__ CUtensorMap kv_map, const __grid_constant__ CUtensorMap q_map, const PfxParams p)
{
    extern __shared__ unsigned char smem_raw[];
    if (smem_u32(smem_raw) & 1023u) {                                  // the tiles need it; no static shared memory, so it holds
        if (threadIdx.x == 0) atomicOr(p.status, 1 << KAP_ERR_DEVICE_INDEX);
        pdl_wait();
        return;
    }
    unsigned char* const q_tiles = smem_raw;
    unsigned char* const slots = smem_raw + 2 * kPfxQBytes;
    PfxControl* const c = reinterpret_cast<PfxControl*>(slots + kPfxSlots * kPfxSlotBytes);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    if (tid == 0) {
        for (int i = 0; i < kPfxSlots; ++i) { mbar_init(smem_u32(&c->full[i]), 1); mbar_init(smem_u32(&c->free[i]), 1); }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&c->q_full[i]), 1);
            mbar_init(smem_u32(&c->q_free[i]), 1);
            mbar_init(smem_u32(&c->s_ready[i]), 1);
            mbar_init(smem_u32(&c->s_free[i]), 4);                     // the stream's four softmax warps
            mbar_init(smem_u32(&c->p_ready[i]), 4);
            mbar_init(smem_u32(&c->pv_done[i]), 1);
        }
        mbar_init(smem_u32(&c->drained), 1);
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
    // Nothing of the caller's is read above.  The split kernel's results are not needed before the merge pass, but what the kernels in
    // front of it wrote is visible to a grid that waits, and to no other (without this wait 32K x 64 sequences took 60.4 us, with it
    // 61.9; four ragged prefixes 114.2 and 116.9).
    pdl_wait();
    pdl_launch_dependents();
    const uint64_t deadline = global_ns() + kWaitBudgetNs;
    volatile int32_t* const late = &c->timed_out;
    const int seg0 = p.cta_begin[blockIdx.x], seg1 = p.cta_begin[blockIdx.x + 1];
    auto wait = [&](unsigned long long& bar, uint32_t parity) { return mbar_wait(smem_u32(&bar), parity, deadline, late); };

    if (warp == 8) {
        // ---- TMA: 20 copies a step (five pages, K and V, two halves of 64 columns), issued by one elected lane with warp-uniform
        // coordinates (lanes with a copy each took twice as long: they are issued one by one all the same)
        uint64_t keep;
        asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(keep));
        int slot = 0, loads = 0, q_use[2] = {0, 0}, q_slot = 0;
        uint32_t parity = 1;                                           // of the slots' free barriers: the first round does not wait
        bool ok = true;
        const int q_end = *p.q_end;
        for (int k = seg0; k < seg1 && ok; ++k) {
            const PrefixSegment s = p.segments[k];
            const int list_at = p.bt_indptr[s.seq], listed = p.bt_indptr[s.seq + 1] - list_at;
            const int n_steps = __shfl_sync(0xffffffffu, s.step_end - s.step_begin, 0), page0 = __shfl_sync(0xffffffffu, s.step_begin, 0) * kPrefixStepPages;
            const int n_pages = min(__shfl_sync(0xffffffffu, s.n_pages, 0) - page0, n_steps * kPrefixStepPages);
            const int kv_head = __shfl_sync(0xffffffffu, s.kv_head, 0), tok_row0 = __shfl_sync(0xffffffffu, s.tok_row0, 0);
            const bool pair = __shfl_sync(0xffffffffu, s.flags, 0) & kSegPair;
            // page ids, 30 at a time and one batch ahead; an entry behind the table's end is reported like a bad one
            auto fetch = [&](int i) { return i >= n_pages ? 0 : page0 + i < listed ? p.bt_pages[list_at + page0 + i] : -1; };
            constexpr int kBatch = 30 / kPrefixStepPages;              // steps
            int32_t ids = 0, next_ids = lane < 30 ? fetch(lane) : 0;
            for (int t = 0; t < (pair ? 2 : 1) && ok; ++t) {
                const int to = pair ? t : q_slot;
                ok = q_use[to] == 0 || wait(c->q_free[to], (uint32_t)(q_use[to] - 1) & 1u);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                if (elect_one()) {
                    const uint32_t bar = smem_u32(&c->q_full[to]), dst = smem_u32(q_tiles) + to * kPfxQBytes;
                    const int tok = tok_row0 + t * (kPrefixTileRows / p.G);
                    if (min(tok + kPrefixTileRows / p.G, p.total_rows) <= q_end) {
                        mbar_expect_tx(bar, kPfxQBytes);
                        tma_load_3d(dst, &q_map, 0, kv_head * p.G, tok, bar, keep);
                        tma_load_3d(dst + kPfxQHalfBytes, &q_map, 64, kv_head * p.G, tok, bar, keep);
                    } else {                                           // fewer rows than scheduled (reported by the merge pass): none are read
                        mbar_arrive(bar);
                    }
                }
                __syncwarp();
                ++q_use[to];
            }
            if (!pair) q_slot ^= 1;
            int in_batch = 0;
            for (int j = 0; j < n_steps && ok; ++j) {
                if (in_batch == 0) {
                    ids = next_ids;
                    next_ids = lane < 30 ? fetch((j + kBatch) * kPrefixStepPages + lane) : 0;
                    if (ids < 0 || ids >= p.num_pool_pages) { ids = 0; atomicOr(p.status, 1 << KAP_ERR_DEVICE_INDEX); }
                }
                const int n = min(kPrefixStepPages, n_pages - j * kPrefixStepPages);
                int32_t page[kPrefixStepPages];
#pragma unroll
                for (int i = 0; i < kPrefixStepPages; ++i) page[i] = __shfl_sync(0xffffffffu, ids, in_batch * kPrefixStepPages + i);
                if (++in_batch == kBatch) in_batch = 0;
#pragma unroll 1
                for (int v = 0; v < 2 && ok; ++v) {
                    ok = wait(c->free[slot], parity);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    if (elect_one()) {
                        const uint32_t bar = smem_u32(&c->full[slot]), dst = smem_u32(slots) + slot * kPfxSlotBytes;
                        mbar_expect_tx(bar, (uint32_t)n * kTileBytes);
#pragma unroll
                        for (int i = 0; i < kPrefixStepPages; ++i) {
                            if (i >= n) break;
                            if (kNhd) {
                                const int z = (page[i] * 2 + v) * kPageSize;
                                tma_load_3d(dst + i * kHalfTileBytes, &kv_map, 0, kv_head, z, bar, keep);
                                tma_load_3d(dst + kPfxPlaneBytes + i * kHalfTileBytes, &kv_map, 64, kv_head, z, bar, keep);
                            } else {
                                const int y = ((page[i] * 2 + v) * p.hkv + kv_head) * kPageSize;
                                tma_load_2d(dst + i * kHalfTileBytes, &kv_map, 0, y, bar, keep);
                                tma_load_2d(dst + kPfxPlaneBytes + i * kHalfTileBytes, &kv_map, 64, y, bar, keep);
                            }
                        }
                    }
                    __syncwarp();
                    ++loads;
                    if (++slot == kPfxSlots) { slot = 0; parity ^= 1u; }
                }
            }
        }
        if (*late) {                                                   // copies in flight must land before the CTA ends
            const uint64_t last = global_ns() + kWaitBudgetNs;
            int32_t more = 0;
            for (int s = max(0, loads - kPfxSlots); s < loads; ++s) mbar_wait(smem_u32(&c->full[s % kPfxSlots]), (uint32_t)(s / kPfxSlots) & 1u, last, &more);
            for (int s = 0; s < 2; ++s)
                if (q_use[s]) mbar_wait(smem_u32(&c->q_full[s]), (uint32_t)(q_use[s] - 1) & 1u, last, &more);
        }
    } else if (warp == 9) {
        // ---- tensor core.  The queue in front of it is short (a group of products keeps its issuer for about as long as it
        // takes), so one elected lane runs through a whole segment, waits included, and nothing comes between the groups; every
        // value it uses is the same in all lanes, as the uniform registers that the products take their operands from want it.
        constexpr uint32_t idesc_o = umma_idesc(kPrefixTileRows, kHeadDim, true);
        // descriptors of the first query tile and, for K and for V, of the first slot; other places add their distance / 16
        const uint64_t q_desc = umma_smem_desc(smem_u32(q_tiles), 16, 1024), k_desc = umma_smem_desc(smem_u32(slots), 16, 1024);
        // V: 16 tokens (K) x 128 columns (N), N contiguous; columns 64-127 one plane further, 8 tokens = 1 KiB
        const uint64_t v_desc = umma_smem_desc(smem_u32(slots), kPfxPlaneBytes, 1024);
        int step0 = 0, q_slot = 0, count0 = 0, count1 = 0;             // steps so far; works of each stream so far
        uint32_t q_parity = 0;                                         // bit i: of query slot i
        for (int k = seg0; k < seg1; ++k) {
            const PrefixSegment seg = p.segments[k];
            const int n_steps = __shfl_sync(0xffffffffu, seg.step_end - seg.step_begin, 0);
            const int n_pages = __shfl_sync(0xffffffffu, seg.n_pages - seg.step_begin * kPrefixStepPages, 0);
            const int pair = __shfl_sync(0xffffffffu, seg.flags & kSegPair, 0) ? 1 : 0;
            const int base0 = count0, base1 = count1, base = step0, q_at = q_slot;
            if (elect_one()) {
                // S of step j for stream t (its work n)
                auto issue_s = [&](int t, int n, int j, bool last_user) {
                    const int slot = (2 * (base + j)) % kPfxSlots;
                    wait(c->full[slot], (uint32_t)((base + j) / (kPfxSlots / 2)) & 1u);
                    if (n > 0) wait(c->s_free[t], (uint32_t)(n - 1) & 1u);     // the softmax warps have read the scores before
                    tc_fence_after();
                    const uint64_t q = q_desc + (uint32_t)(pair ? t : q_at) * (kPfxQBytes / 16), kd = k_desc + (uint32_t)slot * (kPfxSlotBytes / 16);
                    const int pages = min(kPrefixStepPages, n_pages - j * kPrefixStepPages);
                    const uint32_t idesc_s = umma_idesc(kPrefixTileRows, kPageSize, false) + ((uint32_t)(pages - 1) * (kPageSize >> 3) << 17);
#pragma unroll
                    for (int ks = 0; ks < 8; ++ks)
                        umma_ss(tmem + t * 256, q + ((ks >> 2) * kPfxQHalfBytes + (ks & 3) * 32) / 16,
                                kd + ((ks >> 2) * kPfxPlaneBytes + (ks & 3) * 32) / 16, idesc_s, ks > 0);
                    umma_commit(smem_u32(&c->s_ready[t]));
                    if (last_user) umma_commit(smem_u32(&c->free[slot]));
                };
                auto issue_pv = [&](int t, int n, int j, bool first, bool last_user) {
                    const int slot = (2 * (base + j)) % kPfxSlots + 1;
                    wait(c->full[slot], (uint32_t)((base + j) / (kPfxSlots / 2)) & 1u);
                    wait(c->p_ready[t], (uint32_t)n & 1u);
                    tc_fence_after();
                    const uint64_t v = v_desc + (uint32_t)slot * (kPfxSlotBytes / 16);
                    const uint32_t o = tmem + t * 256 + kPfxTmemO, w = tmem + t * 256 + kPfxTmemP;
                    const int pages = min(kPrefixStepPages, n_pages - j * kPrefixStepPages);
#pragma unroll
                    for (int pg = 0; pg < kPrefixStepPages; ++pg)
                        if (pg < pages) umma_ts(o, w + pg * 8, v + pg * (kHalfTileBytes / 16), idesc_o, !first || pg > 0);
                    umma_commit(smem_u32(&c->pv_done[t]));
                    if (last_user) umma_commit(smem_u32(&c->free[slot]));
                };
                wait(c->q_full[pair ? 0 : q_at], (q_parity >> (pair ? 0 : q_at)) & 1u);
                if (pair) {
                    wait(c->q_full[1], q_parity >> 1);
                    for (int j = 0; j < n_steps; ++j) {
                        issue_s(0, base0 + j, j, false);
                        if (j > 0) issue_pv(0, base0 + j - 1, j - 1, j == 1, false);
                        issue_s(1, base1 + j, j, true);
                        if (j > 0) issue_pv(1, base1 + j - 1, j - 1, j == 1, true);
                    }
                    issue_pv(0, base0 + n_steps - 1, n_steps - 1, n_steps == 1, false);
                    issue_pv(1, base1 + n_steps - 1, n_steps - 1, n_steps == 1, true);
                    umma_commit(smem_u32(&c->q_free[0]));              // (all products of the segment are among those waited for)
                    umma_commit(smem_u32(&c->q_free[1]));
                } else {                                               // step j: work j / 2 of stream j mod 2
                    for (int j = 0; j < n_steps; ++j) {
                        issue_s(j & 1, (j & 1 ? base1 : base0) + (j >> 1), j, true);
                        if (j > 1) issue_pv(j & 1, (j & 1 ? base1 : base0) + (j >> 1) - 1, j - 2, j < 4, true);
                    }
                    for (int j = max(0, n_steps - 2); j < n_steps; ++j)
                        issue_pv(j & 1, (j & 1 ? base1 : base0) + (j >> 1), j, j < 2, true);
                    umma_commit(smem_u32(&c->q_free[q_at]));
                }
            }
            __syncwarp();
            step0 += n_steps;
            count0 += pair ? n_steps : (n_steps + 1) >> 1;
            count1 += pair ? n_steps : n_steps >> 1;
            q_parity ^= pair ? 3u : 1u << q_slot;
            if (!pair) q_slot ^= 1;
        }
        if (elect_one()) umma_commit(smem_u32(&c->drained));           // everything issued, whatever happened
        int32_t more = 0;
        mbar_wait(smem_u32(&c->drained), 0, global_ns() + kWaitBudgetNs, &more);
        __syncwarp();
    } else if (warp < 8) {
        // ---- softmax: stream = warp group, one query row per thread
        const int stream = warp >> 2, r = (warp & 3) * 32 + lane;
        const uint32_t t_s = tmem + ((uint32_t)((warp & 3) * 32) << 16) + stream * 256, t_p = t_s + kPfxTmemP, t_o = t_s + kPfxTmemO;
        const float sc = p.scale_log2;
        int count = 0;                                                 // works of this stream
        for (int k = seg0; k < seg1; ++k) {
            const PrefixSegment seg = p.segments[k];
            const bool pair = seg.flags & kSegPair;
            const int n_steps = seg.step_end - seg.step_begin;
            const int tile = pair ? stream : 0, R = tile * kPrefixTileRows + r;
            const bool valid = R < seg.rows, any_valid = tile * kPrefixTileRows + (warp & 3) * 32 < seg.rows;
            int seen = 0;                                              // tokens of the prefix that this row sees
            if (valid) {
                const PrefixRow row = p.row_map[seg.tok_row0 + R / p.G];
                seen = min(p.ctx_len[row.seq] + row.back, seg.n_pages * kPageSize);
            }
            float m_ref = -INFINITY, l = 0.f;
            int mine = 0;                                              // works of this stream in the segment
            for (int j = pair ? 0 : stream; j < n_steps; j += pair ? 1 : 2) {
                const int n_seen = seen - (seg.step_begin + j) * kPrefixStepTokens;
                wait(c->s_ready[stream], (uint32_t)count & 1u);
                __syncwarp();
                tc_fence_after();
                if (any_valid) {
                    float s[kPrefixStepTokens];
                    load_scores(t_s, s);
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&c->s_free[stream]));
                    const bool masked = __any_sync(0xffffffffu, n_seen < kPrefixStepTokens);
                    if (masked) mask_scores(s, n_seen);
                    const float m_step = row_max(s) * sc;              // -inf: the row sees nothing here
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
                    uint32_t w[kPrefixStepTokens / 2];
                    l += masked ? weights<false>(s, sc, mu, w) : weights<true>(s, sc, mu, w);
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
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&c->p_ready[stream]));
                ++count; ++mine;
            }
            // ---- the segment's state: pair segments one for all rows, solo segments one per stream
            if (mine > 0) {
                wait(c->pv_done[stream], (uint32_t)(count - 1) & 1u);
                __syncwarp();
                tc_fence_after();
                if (any_valid) {
                    const long long row = (long long)seg.state_row0 + (!pair && stream ? seg.rows : 0) + R;
#pragma unroll 1
                    for (int i = 0; i < kHeadDim; i += 32) {
                        uint32_t o[2][16];
                        tmem_ld16_nowait(t_o + i, o[0]);
                        tmem_ld16_nowait(t_o + i + 16, o[1]);
                        tmem_wait_ld();
                        if (valid) {
                            // 32-byte stores: each lane has a row of its own, so an instruction touches 32 lines whatever its width
                            float* dst = p.part_o + row * kHeadDim + i;
#pragma unroll
                            for (int e = 0; e < 4; ++e) store_32b(dst + 8 * e, &o[e >> 1][8 * (e & 1)]);
                        }
                    }
                    if (valid) *reinterpret_cast<float2*>(p.part_ml + row * 2) = make_float2(m_ref, l);
                }
                tc_fence_before();                                     // O has been read: the next segment's products may replace it
                __syncwarp();
            }
        }
    }
    if (lane == 0 && *late) atomicOr(p.status, 1 << KAP_ERR_TIMEOUT);
    tc_fence_before();
    __syncthreads();
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(512) : "memory");
}

// ---- joins the states of every (query row, head).  A warp takes H heads of a KV head's group, whose states lie next to each other; a
// lane holds four columns of each.  Bound by latency (the chain row -> units -> states, then batches of loads) and by the
// states' bytes (520 each, mostly still in L2).  kWide: the four warps of a CTA share the states of one such set and join
// theirs through shared memory.
template <int H, bool kWide>
__global__ void __launch_bounds__(128)
kap_prefix_merge_kernel(const PfxParams p)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long set = kWide ? blockIdx.x : (long long)blockIdx.x * 4 + warp;
    const int per_row = p.hq / H;
    if (set >= (long long)p.total_rows * per_row) { pdl_wait(); return; }
    const int row = (int)(set / per_row), head = (int)(set % per_row) * H, g = head / p.G, h = head % p.G;
    const PrefixRow where = p.row_map[row];                            // the schedule's arrays: final before the kernel in front
    const PrefixSeq s = p.seqs[where.seq];
    int n[2] = {0, 0};
    long long at[2] = {0, 0};
    int stride[2] = {0, 0};
    if (s.prefix_unit0 >= 0) {
        const int R = (row - s.group_row0) * p.G + h;                  // (H heads never straddle a block: H divides G, G divides 256)
        const PrefixUnit u = p.units[s.prefix_unit0 + g * s.n_blocks + R / s.block_rows];
        n[0] = u.n_states; stride[0] = u.rows; at[0] = u.state_row0 + R % s.block_rows;
    }
    if (s.own_unit0 >= 0) {
        const PrefixUnit u = p.units[s.own_unit0 + g];
        n[1] = u.n_states; stride[1] = u.rows; at[1] = u.state_row0 + (row - s.row0) * p.G + h;
    }
    pdl_wait();
    const int q_end = *p.q_end;                                        // rows behind it are not the caller's
    // not the scheduled rows, or a context that outgrew the schedule or its block table
    if (lane == 0 && (!kWide || warp == 0)) {
        const int most = min(s.list_pages, p.bt_indptr[where.seq + 1] - p.bt_indptr[where.seq]);
        if (p.q_indptr[where.seq] != s.row0 || q_end != p.total_rows || p.ctx_len[where.seq] > (long long)most * kPageSize) atomicOr(p.status, 1 << KAP_ERR_DEVICE_INDEX);
    }
    Merged acc[H];
#pragma unroll
    for (int e = 0; e < H; ++e) { acc[e].m = -INFINITY; acc[e].l = 0.f; acc[e].o = make_float4(0.f, 0.f, 0.f, 0.f); }
    const int total = n[0] + n[1];
    constexpr int kBatch = 8 / H, kStep = kWide ? 4 : 1;
    for (int i0 = kWide ? warp : 0; i0 < total; i0 += kBatch * kStep) {
        float2 ml[kBatch][H];
        float4 o[kBatch][H];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const int i = min(i0 + j * kStep, total - 1), part = i < n[0] ? 0 : 1;
            const long long r = at[part] + (long long)(i - part * n[0]) * stride[part];
#pragma unroll
            for (int e = 0; e < H; ++e) {
                ml[j][e] = __ldcg(reinterpret_cast<const float2*>(p.part_ml + (r + e) * 2));
                o[j][e] = __ldcg(reinterpret_cast<const float4*>(p.part_o + (r + e) * kHeadDim) + lane);
            }
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
#pragma unroll
            for (int e = 0; e < H; ++e)                                // (an empty state's O was never written)
                if (i0 + j * kStep < total && ml[j][e].y > 0.f) merge_into(acc[e], ml[j][e].x, ml[j][e].y, o[j][e]);
    }
    if constexpr (kWide) {
        __shared__ float4 other_o[3][H][32];
        __shared__ float2 other_ml[3][H];
        if (warp > 0) {
#pragma unroll
            for (int e = 0; e < H; ++e) {
                other_o[warp - 1][e][lane] = acc[e].o;
                if (lane == 0) other_ml[warp - 1][e] = make_float2(acc[e].m, acc[e].l);
            }
        }
        __syncthreads();
        if (warp > 0) return;
#pragma unroll
        for (int w = 0; w < 3; ++w)                                    // in a fixed order: results do not depend on timing
#pragma unroll
            for (int e = 0; e < H; ++e)
                if (other_ml[w][e].y > 0.f) merge_into(acc[e], other_ml[w][e].x, other_ml[w][e].y, other_o[w][e][lane]);
    }
    if (row >= q_end) return;
#pragma unroll
    for (int e = 0; e < H; ++e) {
        const long long cell = (long long)row * p.hq + head + e;
        const float inv = acc[e].l > 0.f ? 1.f / acc[e].l : 0.f;
        uint2 v;
        v.x = pack_bf16(acc[e].o.x * inv, acc[e].o.y * inv);
        v.y = pack_bf16(acc[e].o.z * inv, acc[e].o.w * inv);
        *reinterpret_cast<uint2*>(p.out + cell * kHeadDim + lane * 4) = v;
        if (p.lse && lane == 0) p.lse[cell] = acc[e].l > 0.f ? (acc[e].m + log2f(acc[e].l)) * 0.6931471805599453f : -INFINITY;
    }
}

}  // namespace kap
