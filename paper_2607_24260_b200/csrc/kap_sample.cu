// kap_sample_tokens: draw one token per logits row from the truncated softmax with a given uniform number.
//
// Mathematics, for a row x with temperature T > 0:  w_i = exp((x_i - max x) / T);  top-k keeps the k largest
// logits, top-p of those the shortest prefix by descending value whose weight reaches p of theirs, min-p those
// with w_i >= min_p;  the token is the first index, in vocabulary order, whose running sum of kept weights
// exceeds u times their total.  Equal logits rank by index.
//
// A sort is not needed: each filter is a threshold on the logit plus the number of logits equal to it that still
// count.  With I(x) an order-preserving integer image of the logit, a threshold is found on the distance
// I(max) - I(x) by a search of 1024 intervals at a time (a histogram of counts in shared memory; integer counts, so the
// order of the atomics does not matter): two or three levels instead of 32 bisections.  For top-p the counts give bounds of
// the weight in every interval; the weight above the remaining range is summed exactly.
//
// All sums are held in 64 bits and added in an order that the shape of the call alone fixes: the token is decided by comparing long
// sums, and 32-bit ones over 128 256 weights would move a border in every few hundred rows.  exp is a
// 64-bit polynomial after reduction to a power of two (exp2_f64 below).
//
// Layout of the filtered rows: one cluster of up to 16 CTAs per row, 512 threads each; the row is read once, into the shared memory of
// the cluster, as images.  A thread owns an odd number of consecutive logits (conflict-free, and in index order).  CTAs exchange
// partial results by writing to all peers' shared memory, one cluster barrier per exchange.  When at most 512 logits can still be
// drawn, the first CTA gets them and finishes alone (one row 32 -> 15 us, 64 mixed rows 85 -> 65).  A thread carries its weight of what
// the top-p search has passed, all of it kept, into the draw (64 mixed rows 65 -> 62, 100 flat rows 95 -> 87).
// Bound: the phases between the barriers, one after the other (of the 15 us of a single row the read takes 2), and with many rows
// shared-memory atomics and 64-bit sums: 64 rows of 128256 with mixed filters 61 us; 100 rows of 50257 in bf16, top-p 89 us.
#include <cmath>

#include "kap_ptx.cuh"

namespace kap {
void count_launch();

namespace {

constexpr int kSampleThreads = 512;
constexpr int kSampleWarps = kSampleThreads / 32;
constexpr int kBins = 1024;
constexpr int kFew = kSampleThreads;               // logits that one CTA finishes alone: one a thread
constexpr int kSms = 148;                          // of a B200; only the choices of a launch's shape use it
constexpr uint32_t kImageMinusInf = 0x007fffffu;   // image of -inf; nothing at or below it has weight
constexpr uint32_t kImagePlusInf = 0xff800000u;
constexpr int kMaxRounds = 48;                     // of a search, more than either can take
constexpr int kMaxStrip = 99;                      // logits a thread owns at most: 512 x 99 x 4 bytes of shared memory

__device__ __forceinline__ uint32_t logit_image(float v) {          // NaN like -inf, -0 = +0
    const uint32_t u = __float_as_uint(v + 0.0f);
    return v != v ? kImageMinusInf : u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float image_logit(uint32_t u) {
    return __uint_as_float(u ^ ((u >> 31) ? 0x80000000u : 0xffffffffu));
}
// The logit of an image as a double, by moving bits (the conversion instruction runs at a quarter of the rate of these).  Subnormal
// logits and zero come out within 2^-126 of themselves and +inf as 2^128; the order is kept.
__device__ __forceinline__ double wide_logit(uint32_t u) {
    const uint32_t flip = ~(uint32_t)((int)u >> 31);                    // all ones for a negative logit
    const uint32_t mag = (u ^ flip) & 0x7fffffffu;
    return __hiloint2double((int)(((mag >> 3) + 0x38000000u) | (flip & 0x80000000u)), (int)(mag << 29));
}
// 2^t for t <= 0 in 64 bits, to be discarded below the smallest normal number (`vanishes`).  t = n + f with |f| <= 1/2 (a sum with
// 1.5 2^52 holds n in its low word), 2^f by the polynomial of degree 9 of least largest relative error there among those that are 1
// at 0 (1.5e-14; Lawson's iteration), so that logits equal to the largest have the weight 1 and sums of them are exact.  Its
// coefficients are in constant memory, from where the products take them without a register.
__constant__ double kExp2[10] = {1.0148340385735375e-07, 1.3258335410465268e-06, 1.5252990017215676e-05, 0.0001540344088444558, 0.0013333557625466606,
                                 0.009618129181163905, 0.05550410866841578, 0.2402265069572282, 0.6931471805598851, 1.0};
__device__ __forceinline__ bool vanishes(double t) { return (uint32_t)__double2hiint(t) > 0xc08ff000u; }       // t < -1022
__device__ __forceinline__ double exp2_f64(double d, double scale) {           // 2^(d scale)
    const double s = fma(d, scale, 6755399441055744.0), f = fma(d, scale, 6755399441055744.0 - s);
    double y = kExp2[0];
#pragma unroll
    for (int i = 1; i < 10; ++i) y = fma(y, f, kExp2[i]);
    return __hiloint2double(__double2hiint(y) + (__double2loint(s) << 20), __double2loint(y));
}
__device__ __forceinline__ double exp2_f64(double t) { return exp2_f64(t, 1.0); }

struct SampleParams {
    const void* logits;
    long long row_stride;
    int32_t vocab, slice, strip, cluster;          // logits of a row, of a CTA, of a thread; CTAs of a row
    const float *temperature, *top_p, *min_p, *uniform;
    const int32_t* top_k;
    int32_t* token;
    float* logprob;
};

struct SampleShared {
    uint32_t hist[2][kBins];
    // filled by all CTAs of the cluster, one entry each
    int32_t best[kMaxCluster], finite[kMaxCluster];
    double level_sum[2][kMaxCluster], kept_sum[kMaxCluster];
    int32_t ties[kMaxCluster];
    // this CTA
    double warp_d[kSampleWarps][2];
    uint32_t warp_u[kSampleWarps];
    int32_t warp_i[kSampleWarps];
    int32_t bin[2];
    int32_t before[2];
    // first CTA: the logits that can still be drawn, when they are few
    int32_t few;
    uint32_t few_image[kFew];
    int32_t few_index[kFew];
    double few_weight[kFew];
    uint32_t bin_count;
    double edge;
};

__device__ __forceinline__ void put_remote(uint32_t addr, unsigned long long v) {
    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(addr), "l"(v) : "memory");
}
__device__ __forceinline__ void put_remote(uint32_t addr, int32_t v) {
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
__device__ __forceinline__ void put_remote(uint32_t addr, double v) { put_remote(addr, (unsigned long long)__double_as_longlong(v)); }
__device__ __forceinline__ uint2 get_remote(uint32_t addr) {
    uint2 v;
    asm volatile("ld.shared::cluster.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr));
    return v;
}

__device__ __forceinline__ float as_float(float v) { return v; }
__device__ __forceinline__ float as_float(__nv_bfloat16 v) { return __bfloat162float(v); }

template <typename T>
__global__ void __launch_bounds__(kSampleThreads, 2)
kap_sample_rows_kernel(const SampleParams p)
{
    extern __shared__ __align__(16) unsigned char smem[];
    SampleShared& sh = *reinterpret_cast<SampleShared*>(smem);
    uint32_t* const space = reinterpret_cast<uint32_t*>(smem + (sizeof(SampleShared) + 15) / 16 * 16);
    const int C = p.cluster, r = blockIdx.x / C, rank = blockIdx.x % C, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int first = min(p.vocab, rank * p.slice), n = min(p.vocab, first + p.slice) - first;      // this CTA's logits
    const T* x = reinterpret_cast<const T*>(p.logits) + (long long)r * p.row_stride + first;
    const int room = p.strip * kSampleThreads;
    if (C > 1) cluster_arrive();                                   // (its wait: every peer runs before anybody writes to it)

    auto to_all = [&](auto* slot, auto v) {                        // slot[rank] of every CTA's shared memory; threads 0 .. C - 1 call
        put_remote(map_to_cta(smem_u32(slot + rank), tid), v);
    };
    auto meet = [&] { if (C > 1) cluster_sync(); else __syncthreads(); };

    // ---- read the slice once; the row's largest logit, and with top-k how many logits have weight at all
    const int k = p.top_k ? p.top_k[r] : 0;
    const bool counted = k > 0 && k < p.vocab;
    constexpr int kVec = 16 / (int)sizeof(T);
    const int head = min(n, (int)(((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / sizeof(T)));
    const int n_vec = (n - head) / kVec;
    uint32_t* const img = space + ((4 - head) & 3);                    // image `head` on a 16-byte boundary
    uint32_t best = 0u;
    int finite = 0;
    auto image_of = [&](float v) {
        const uint32_t u = logit_image(v);
        best = max(best, u);
        if (counted) finite += u > kImageMinusInf;
        return u;
    };
    for (int i = tid; i < head; i += kSampleThreads) img[i] = image_of(as_float(x[i]));
    constexpr int kInFlight = 4;
    for (int j0 = tid; j0 < n_vec; j0 += kInFlight * kSampleThreads) {
        uint4 v[kInFlight];
#pragma unroll
        for (int u = 0; u < kInFlight; ++u)
            if (j0 + u * kSampleThreads < n_vec) v[u] = __ldcs(reinterpret_cast<const uint4*>(x + head) + j0 + u * kSampleThreads);
#pragma unroll
        for (int u = 0; u < kInFlight; ++u)
            if (j0 + u * kSampleThreads < n_vec) {
                const T* e = reinterpret_cast<const T*>(&v[u]);
                uint4* to = reinterpret_cast<uint4*>(img + head + (j0 + u * kSampleThreads) * kVec);
#pragma unroll
                for (int q = 0; q < kVec / 4; ++q)
                    to[q] = make_uint4(image_of(as_float(e[4 * q])), image_of(as_float(e[4 * q + 1])), image_of(as_float(e[4 * q + 2])), image_of(as_float(e[4 * q + 3])));
            }
    }
    for (int i = head + n_vec * kVec + tid; i < n; i += kSampleThreads) img[i] = image_of(as_float(x[i]));
    for (int i = n + tid; i < room; i += kSampleThreads) img[i] = 0u;
    for (int i = tid; i < 2 * kBins; i += kSampleThreads) (&sh.hist[0][0])[i] = 0u;
    if (tid == 0) sh.few = 0;
    best = __reduce_max_sync(0xffffffffu, best);
    finite = __reduce_add_sync(0xffffffffu, finite);
    if (lane == 0) { sh.warp_u[warp] = best; sh.warp_i[warp] = finite; }
    __syncthreads();
    if (C > 1) cluster_wait();
    if (tid < C) {
        best = 0u; finite = 0;
        for (int w = 0; w < kSampleWarps; ++w) { best = max(best, sh.warp_u[w]); finite += sh.warp_i[w]; }
        to_all(sh.best, (int32_t)best);
        to_all(sh.finite, finite);
    }
    meet();
    uint32_t top = 0u;
    finite = 0;
    for (int c = 0; c < C; ++c) { top = max(top, (uint32_t)sh.best[c]); finite += sh.finite[c]; }
    const uint32_t* const mine = img + tid * p.strip;
    const float t = p.temperature ? p.temperature[r] : 1.f;
    if (top <= kImageMinusInf) {                                       // no token at all
        if (rank == 0 && tid == 0) {
            p.token[r] = -1;
            if (p.logprob) p.logprob[r] = -INFINITY;
        }
        return;
    }
    if (!(t > 0.f)) {                                                  // greedy: the first CTA with a largest logit, the first place in it
        int c = 0;
        while ((uint32_t)sh.best[c] != top) ++c;
        if (c != rank) return;
        int at = 0x7fffffff;
        for (int i = p.strip - 1; i >= 0; --i)
            if (mine[i] == top) at = tid * p.strip + i;
        at = __reduce_min_sync(0xffffffffu, at);
        __syncthreads();
        if (lane == 0) sh.warp_i[warp] = at;
        __syncthreads();
        if (tid == 0) {
            for (int w = 1; w < kSampleWarps; ++w) at = min(at, sh.warp_i[w]);
            p.token[r] = first + at;
            if (p.logprob) p.logprob[r] = 0.f;
        }
        return;
    }
    // the weight 2^((x - max) / T / ln 2); +inf stands for the largest finite number (the conversion runs beside the sums, on its own pipe)
    auto widen = [](uint32_t u) { return (double)fminf(image_logit(u), 3.402823466e38f); };
    const double x_max = widen(top), per_bit = 1.4426950408889634 / (double)t;
    const uint32_t far_off = (uint32_t)__double2hiint(-1021.0 / per_bit);      // (-inf for an endless T)
    auto behind = [&](uint32_t u) { return widen(u) - x_max; };
    auto gone = [&](double d) { return (uint32_t)__double2hiint(d) >= far_off; };
    auto weight = [&](uint32_t u) {
        const double d = behind(u);
        return gone(d) ? 0.0 : exp2_f64(d, per_bit);
    };
    // Weights of the distances below `span` (and, of those equal to it, of the ones whose rank among the equal ones, from `tie_rank` on, is
    // below `quota`) in this thread's strip: which ones, 32 at a time, then three chains of products side by side for as long as a
    // lane of the warp has one left.
    auto strip_weight = [&](uint32_t from, uint32_t span, int tie_rank, int quota) {
        const uint32_t high = top - from;
        double s = 0.0;
        for (int i0 = 0; i0 < p.strip; i0 += 32) {
            const int n_here = min(32, p.strip - i0);
            uint32_t wanted = 0u;
#pragma unroll 4
            for (int i = 0; i < n_here; ++i) {
                const uint32_t d = high - mine[i0 + i];
                bool in = d < span;
                if (quota > 0 && d == span) in = tie_rank++ < quota;
                wanted |= (uint32_t)in << i;
            }
            while (__any_sync(0xffffffffu, wanted != 0u)) {
                double e[3], w[3];
                bool have[3];
#pragma unroll
                for (int j = 0; j < 3; ++j) {
                    have[j] = wanted != 0u;
                    e[j] = behind(mine[i0 + (have[j] ? __ffs(wanted) - 1 : 0)]);
                    wanted &= wanted - 1u;
                }
#pragma unroll
                for (int j = 0; j < 3; ++j) w[j] = exp2_f64(e[j], per_bit);
#pragma unroll
                for (int j = 0; j < 3; ++j)
                    if (have[j] && !gone(e[j])) s += w[j];
            }
        }
        return s;
    };
    // the same for everything that has weight, without the search
    auto strip_weight_all = [&](uint32_t span) {
        double s = 0.0;
        for (int i = 0; i < p.strip; i += 3) {
            uint32_t u[3];
            double e[3], w[3];
#pragma unroll
            for (int j = 0; j < 3; ++j) u[j] = i + j < p.strip ? mine[i + j] : 0u;
#pragma unroll
            for (int j = 0; j < 3; ++j) { e[j] = behind(u[j]); w[j] = exp2_f64(e[j], per_bit); }
#pragma unroll
            for (int j = 0; j < 3; ++j)
                if (top - u[j] < span && !gone(e[j])) s += w[j];
        }
        return s;
    };

    const uint32_t furthest = top == kImagePlusInf ? 0u : top - kImageMinusInf - 1u;
    // sum over the block in a fixed order, in every thread
    auto block_sum = [&](double v) {
#pragma unroll
        for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
        __syncthreads();
        if (lane == 0) sh.warp_d[warp][0] = v;
        __syncthreads();
        v = 0.0;
        for (int w = 0; w < kSampleWarps; ++w) v += sh.warp_d[w][0];
        return v;
    };
    double kept_near = 0.0;                                        // this thread's weight of distances below kept_from, all of them kept
    uint32_t kept_from = 0u;
    int level = 0;                                                 // of all searches of the row: parity selects the buffers
    // One level: the CTAs' histograms (of the distances base + [b << shift, (b + 1) << shift), by count_level) summed over the row, two
    // bins a thread; `partial` is summed over the row along the way.
    auto gather_level = [&](double partial, uint32_t (&bins)[2]) {
        const int buf = level & 1;
        const double sum = block_sum(partial);
        if (tid < C) to_all(sh.level_sum[buf], sum);
        meet();
        double total = 0.0;
        for (int c = 0; c < C; ++c) total += sh.level_sum[buf][c];
        bins[0] = bins[1] = 0u;
        const uint32_t at = smem_u32(&sh.hist[buf][2 * tid]);
        for (int c0 = 0; c0 < C; c0 += 4) {                        // four peers' counts under way together
            uint2 v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = get_remote(map_to_cta(at, min(c0 + e, C - 1)));
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (c0 + e < C) { bins[0] += v[e].x; bins[1] += v[e].y; }
        }
        // the other buffer was last read before this barrier: clear it for the next level
        sh.hist[buf ^ 1][2 * tid] = 0u; sh.hist[buf ^ 1][2 * tid + 1] = 0u;
        ++level;
        return total;
    };

    auto count_level = [&](uint64_t base, int shift, double partial, uint32_t (&bins)[2]) {
        // (a search ends before its base passes the last distance that has weight)
        const uint32_t high = top - (uint32_t)base, span = (uint32_t)min((uint64_t)kBins << shift, (uint64_t)furthest + 1 - base);
#pragma unroll 3
        for (int i = 0; i < p.strip; ++i) {
            const uint32_t d = high - mine[i];
            if (d < span) atomicAdd(&sh.hist[level & 1][d >> shift], 1u);
        }
        return gather_level(partial, bins);
    };

    const float top_p = p.top_p ? p.top_p[r] : 1.f, min_p = p.min_p ? p.min_p[r] : 0.f;     // NaN: no filter
    uint32_t min_p_cut = 0xffffffffu;                              // min-p as a cut: logits from the least float with weight enough on
    if (min_p > 0.f) {
        const uint32_t least = logit_image(__double2float_ru(x_max + (double)t * log(fmin((double)min_p, 1.0))));
        min_p_cut = least < top ? top - least : 0u;
    }
    const double u01 = (double)p.uniform[r];
    auto draw_at = [&](double total) { return u01 >= 0.0 ? fmin(u01 * total, total * 0.99999999999999978) : 0.0; };

    // When the logits up to a distance are at most kFew and hold whatever can be drawn, the first CTA gets them all and finishes alone, one
    // logit a thread: ranks by counting, then running sums by rank for top-p and by index for the draw.  Running sums of the block
    // are taken one after the other inside a warp, as in the draw below.
    auto block_run = [&](double v, double& before) {               // returns the total
        double run = 0.0;
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            const double s = __shfl_sync(0xffffffffu, v, j);
            if (lane > j) run += s;
        }
        __syncthreads();
        if (lane == 31) sh.warp_d[warp][0] = run + v;
        __syncthreads();
        double all = 0.0, offset = 0.0;
        for (int w = 0; w < kSampleWarps; ++w) { if (w == warp) offset = all; all += sh.warp_d[w][0]; }
        before = offset + run;
        return all;
    };
    auto finish_few = [&](uint32_t up_to, int most, double whole) {    // the first `most` ranks; weight that top-p refers to, or -1: theirs
        const uint32_t few_at = map_to_cta(smem_u32(&sh.few), 0), image_at = map_to_cta(smem_u32(sh.few_image), 0), index_at = map_to_cta(smem_u32(sh.few_index), 0);
        for (int i = 0; i < p.strip; ++i) {
            if (top - mine[i] > up_to) continue;
            int32_t slot;
            asm volatile("atom.shared::cluster.add.u32 %0, [%1], 1;" : "=r"(slot) : "r"(few_at) : "memory");
            if (slot >= kFew) continue;                            // (cannot be: they were counted)
            put_remote(image_at + 4 * slot, (int32_t)mine[i]);
            put_remote(index_at + 4 * slot, first + tid * p.strip + i);
        }
        meet();
        if (rank != 0) return;
        const int m = min(sh.few, kFew);
        const bool mine_too = tid < m;
        const uint32_t u = mine_too ? sh.few_image[tid] : 0u;
        const int index = mine_too ? sh.few_index[tid] : 0x7fffffff;
        int by_value = 0, by_index = 0;
        for (int j = 0; j < m; ++j) {
            const uint32_t uj = sh.few_image[j];
            const int ij = sh.few_index[j];
            by_value += uj > u || (uj == u && ij < index);
            by_index += ij < index;
        }
        double w = mine_too && by_value < most ? weight(u) : 0.0;
        bool keep = mine_too && by_value < most && top - u <= min_p_cut;
        if (top_p < 1.f) {
            sh.few_weight[tid] = 0.0;
            __syncthreads();
            if (mine_too) sh.few_weight[by_value] = w;
            __syncthreads();
            double before;
            const double all = block_run(sh.few_weight[tid], before);
            const bool stays = tid == 0 || before < (double)top_p * (whole < 0.0 ? all : whole);
            __syncthreads();
            sh.few_weight[tid] = stays ? 1.0 : 0.0;
            __syncthreads();
            keep = keep && sh.few_weight[by_value] > 0.0;
            __syncthreads();
        }
        if (!keep) w = 0.0;
        sh.few_weight[tid] = 0.0;
        __syncthreads();
        if (mine_too) sh.few_weight[by_index] = w;
        __syncthreads();
        double before;
        const double v = sh.few_weight[tid], total = block_run(v, before), target = draw_at(total);
        // (the place in index order whose weight holds the target; block_run's sums end where the next begins only up to a rounding,
        // so the last place that begins at or before the target is taken)
        if (tid == 0) sh.bin[0] = -1;
        __syncthreads();
        if (v > 0.0 && before <= target) atomicMax(&sh.bin[0], tid);
        __syncthreads();
        if (mine_too && by_index == sh.bin[0]) {
            p.token[r] = index;
            if (p.logprob) p.logprob[r] = (float)((per_bit * behind(u) - log2(total)) * 0.69314718055994531);
        }
    };

    // The cut: distances below it are kept, and `quota` of those equal to it (lowest index first).  At first all that have weight:
    // behind +inf nothing has.
    uint32_t cut = furthest;
    int quota = 0x7fffffff, ties_at_cut = 0;
    if (counted && k < finite) {
        uint64_t base = 0;
        int shift = 14, above = 0;                                 // two octaves below the largest logit at first
        for (int rounds = 0; rounds < kMaxRounds; ++rounds) {      // (at most four windows, then widths of 2^22, 2^12, 2^2 and 1)
            uint32_t bins[2];
            count_level(base, shift, 0.0, bins);
            // inclusive running count; the bin in which the k-th falls
            const int both = (int)(bins[0] + bins[1]);
            int run = both;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) { const int o = __shfl_up_sync(0xffffffffu, run, d); if (lane >= d) run += o; }
            if (lane == 31) sh.warp_i[warp] = run;
            if (tid == 0) sh.bin[0] = -1;
            __syncthreads();
            int total = 0;
            for (int w = 0; w < kSampleWarps; ++w) { if (w < warp) run += sh.warp_i[w]; total += sh.warp_i[w]; }
            const int start = above + run - both;                  // before this thread's first bin
            if (start < k && above + run >= k) {
                const bool second = start + (int)bins[0] < k;
                sh.bin[0] = 2 * tid + second;
                sh.before[0] = start + (second ? (int)bins[0] : 0);
                sh.bin_count = bins[second ? 1 : 0];
            }
            __syncthreads();
            const int b = sh.bin[0];
            if (b < 0) {                                           // further down: wider bins
                above += total;
                base += (uint64_t)kBins << shift;
                shift = min(shift + 3, 22);
                __syncthreads();
                if (base > furthest) break;                        // (fewer than k at +inf: they are all that has weight)
                continue;
            }
            above = sh.before[0];
            const int in_bin = (int)sh.bin_count;
            base += (uint64_t)b << shift;
            __syncthreads();
            if (above + in_bin <= kFew) {
                finish_few((uint32_t)min(base + ((uint64_t)1 << shift) - 1, (uint64_t)furthest), k, -1.0);
                return;
            }
            if (above + in_bin == k) { cut = (uint32_t)min(base + ((uint64_t)1 << shift) - 1, (uint64_t)furthest); break; }     // the whole bin
            if (shift == 0) { cut = (uint32_t)base; quota = k - above; ties_at_cut = in_bin; break; }
            shift = max(0, shift - 10);
        }
    }

    if (top_p < 1.f) {
        // the threshold lies where weights still matter: N exp(-R / T) < 1 - p leaves less than 1 - p of the whole behind R
        const double reach = (double)t * (log((double)p.vocab) - log(1.0 - fmax((double)top_p, 0.0))) * (1.0 + 1e-9) + 1e-30;
        const uint32_t far = logit_image(__double2float_rd(x_max - reach));
        const uint32_t last = min(far < top ? top - far : 0u, cut);
        auto shift_for = [&](uint64_t range) { int s = 0; while (((range - 1) >> s) >= kBins) ++s; return s; };
        double target = 0.0, above = 0.0;                          // p times the whole; weight of distances below base
        int b1, b2, in_bin;                                        // bins found; logits in the first one
        double edge;                                               // weight before that one
        // the first bin whose end may reach the target, by upper bounds of the bins' weights, and the first one whose end must
        auto find = [&](const uint32_t (&bins)[2], const double (&lo)[2], const double (&hi)[2], double slack) {
            double run_lo = lo[0] + lo[1], run_hi = hi[0] + hi[1];
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const double a = __shfl_up_sync(0xffffffffu, run_lo, d), b = __shfl_up_sync(0xffffffffu, run_hi, d);
                if (lane >= d) { run_lo += a; run_hi += b; }
            }
            __syncthreads();
            if (lane == 31) { sh.warp_d[warp][0] = run_lo; sh.warp_d[warp][1] = run_hi; }
            if (tid == 0) sh.bin[0] = sh.bin[1] = kBins;
            __syncthreads();
            double before_lo = above, before_hi = above;
            for (int w = 0; w < warp; ++w) { before_lo += sh.warp_d[w][0]; before_hi += sh.warp_d[w][1]; }
            run_lo += before_lo; run_hi += before_hi;
            const double mid_lo = run_lo - lo[1], mid_hi = run_hi - hi[1];
            if (bins[0] && mid_hi >= target - slack) atomicMin(&sh.bin[0], 2 * tid);
            else if (bins[1] && run_hi >= target - slack) atomicMin(&sh.bin[0], 2 * tid + 1);
            if (bins[0] && mid_lo >= target + slack) atomicMin(&sh.bin[1], 2 * tid);
            else if (bins[1] && run_lo >= target + slack) atomicMin(&sh.bin[1], 2 * tid + 1);
            __syncthreads();
            b1 = sh.bin[0]; b2 = sh.bin[1];
            if (b1 < kBins && (b1 >> 1) == tid) {
                const int e = b1 & 1;
                sh.edge = e ? mid_lo : mid_lo - lo[0];
                sh.bin_count = bins[e];
            }
            __syncthreads();
            in_bin = (int)sh.bin_count;
            edge = sh.edge;
        };
        double part = cut == furthest && quota == 0x7fffffff ? strip_weight_all(cut + 1u) : strip_weight(0u, quota == 0x7fffffff ? cut + 1u : cut, 0, 0);   // everything kept so far
        const double cut_part = quota == 0x7fffffff ? 0.0 : (double)quota * weight(top - cut);
        uint64_t base = 0, end = last;                             // distances between which the threshold lies
        const bool even = top != kImagePlusInf && last >= kBins;   // (few distances: their own intervals at once)
        if (even) {
            // First level by value, in equal intervals of what lies before R: intervals of the distance are narrow around zero and
            // wide away from it, so that a flat row would meet in a few of them.  The value of a bin's ends is known to a part in
            // 10^6 (three roundings to 32 bits); one part in 10^5 is allowed for.
            const double depth = fmin(reach, x_max - wide_logit(top - last)) * (1.0 + 1e-5) + 1e-30;
            const float high = image_logit(top), per_value = __double2float_rd((double)kBins / depth);
            const bool usable = per_value > 0.f && per_value < 1e37f;
#pragma unroll 3
            for (int i = 0; i < p.strip; ++i) {
                const uint32_t u = mine[i];
                const float b = (high - image_logit(u)) * per_value;
                if (usable && top - u <= cut && b < (float)kBins) atomicAdd(&sh.hist[level & 1][(int)b], 1u);
            }
            uint32_t bins[2];
            target = (double)top_p * (gather_level(part, bins) + cut_part);
            double lo[2], hi[2];
            const double bin_value = 1.0 / (double)per_value;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const double near = (double)(2 * tid + e) * bin_value * (1.0 - 1e-5), far_end = (double)(2 * tid + e + 1) * bin_value * (1.0 + 1e-5);
                const double a = -near * per_bit, b = -far_end * per_bit;
                hi[e] = bins[e] ? (vanishes(a) ? 0.0 : bins[e] * exp2_f64(a)) : 0.0;
                lo[e] = bins[e] ? (vanishes(b) ? 0.0 : bins[e] * exp2_f64(b)) : 0.0;
            }
            find(bins, lo, hi, 1e-12 * target);
            if (b2 < kBins && quota == 0x7fffffff) {               // few enough up to the end of the last bin in question?
                int upto = (2 * tid <= b2 ? (int)bins[0] : 0) + (2 * tid + 1 <= b2 ? (int)bins[1] : 0);
                upto = __reduce_add_sync(0xffffffffu, upto);
                if (lane == 0) sh.warp_i[warp] = upto;
                __syncthreads();
                upto = 0;
                for (int w = 0; w < kSampleWarps; ++w) upto += sh.warp_i[w];
                const uint32_t to = logit_image(__double2float_rd(x_max - (double)(b2 + 1) * bin_value * (1.0 + 1e-5)));
                // (the bins' ends are not exact: what lies up to `to` are these and perhaps some of the next bin, counted below)
                int exact = 0;
                if (upto <= kFew) {
                    for (int i = 0; i < p.strip; ++i) exact += top - mine[i] <= min(top - to, cut);
                }
                exact = __reduce_add_sync(0xffffffffu, exact);
                __syncthreads();
                if (lane == 0) sh.warp_i[warp] = exact;
                __syncthreads();
                if (upto <= kFew) {
                    exact = 0;
                    for (int w = 0; w < kSampleWarps; ++w) exact += sh.warp_i[w];
                    if (tid < C) to_all(sh.ties, exact);
                    meet();
                    exact = 0;
                    for (int c = 0; c < C; ++c) exact += sh.ties[c];
                    if (exact <= kFew) {
                        finish_few(min(top - to, cut), 0x7fffffff, target / (double)top_p);
                        return;
                    }
                    meet();                                        // sh.ties is used again
                }
            }
            if (b1 < kBins) {
                const uint32_t from = logit_image(__double2float_ru(x_max - (double)b1 * bin_value * (1.0 - 1e-5)));
                base = from < top ? top - from : 0u;
                if (b2 < kBins) {
                    const uint32_t to = logit_image(__double2float_rd(x_max - (double)(b2 + 1) * bin_value * (1.0 + 1e-5)));
                    end = min(end, (uint64_t)(top - to));
                }
                base = min(base, end);
                part = base > 0 ? strip_weight(0u, (uint32_t)base, 0, 0) : 0.0;
                kept_near = part;
                kept_from = (uint32_t)base;
            }
            if (b1 == kBins) part = 0.0;                           // (nothing learnt; `above` stays 0)
        }
        // A window of 1024 intervals over all distances in question.  What it leaves between the two bins found is at most half of them,
        // or (bounds too wide, as beside a gap in the values) their middle is tried: the weight in front of it, summed exactly, says on
        // which side of it the threshold lies.  So two rounds halve a range that begins below 2^32 and ends in single intervals
        // at 2^10: at most 45 rounds.  One to three are usual, ten the most seen (three values, p just past the weight of one of them).
        bool trial = false;                                        // `part` is the weight between base and `middle`
        uint64_t middle = 0;
        for (int rounds = 0; rounds < kMaxRounds; ++rounds) {
            const int shift = shift_for(end - base + 1);
            uint32_t bins[2];
            const double sum = count_level(base, shift, part, bins);
            if (trial) {
                trial = false;
                if (above + sum < target) {
                    above += sum;
                    kept_near += part;
                    base = middle;
                    kept_from = (uint32_t)base;
                } else {
                    end = middle - 1;
                }
                part = 0.0;
                __syncthreads();                                   // the histogram that the next level counts into has been cleared
                continue;
            }
            if (rounds == 0 && !even) target = (double)top_p * (sum + cut_part); else above += sum;
            double lo[2], hi[2];                                   // bounds of the weight in this thread's two bins
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const uint64_t from = base + ((uint64_t)(2 * tid + e) << shift), to = from + ((uint64_t)1 << shift) - 1;
                int c = (int)bins[e];
                if (from > cut) c = 0;
                else if (quota != 0x7fffffff && cut <= to) c -= ties_at_cut - quota;   // of the equal ones only some are left
                // (a bin that holds the cut may hold distances behind it as well: its bounds are too high then, but the
                // threshold does not lie behind it, whatever they say)
                bins[e] = (uint32_t)max(c, 0);
                lo[e] = c > 0 ? c * weight(top - (uint32_t)min(to, (uint64_t)furthest)) : 0.0;
                hi[e] = c > 0 ? (shift == 0 ? lo[e] : c * weight(top - (uint32_t)from)) : 0.0;
            }
            find(bins, lo, hi, shift == 0 ? 0.0 : 1e-12 * target); // at single distances the sums are exact
            if (b1 == kBins) {                                     // (a rounding short of the end: all that there is)
                if (end < cut) { cut = (uint32_t)end; quota = 0x7fffffff; }
                break;
            }
            const uint64_t next = base + ((uint64_t)b1 << shift), bin_end = next + ((uint64_t)1 << shift) - 1;
            if (shift == 0) {
                const uint32_t d = (uint32_t)next;
                const double w = weight(top - d), m = w > 0.0 ? ceil((target - edge) / w) : 1.0;
                const int keep = m < 1.0 ? 1 : m < (double)in_bin ? (int)m : in_bin;
                const bool all = keep == in_bin && !(d == cut && quota != 0x7fffffff);
                if (d != cut || quota == 0x7fffffff) ties_at_cut = in_bin;
                quota = all ? 0x7fffffff : keep;
                cut = d;
                break;
            }
            if (b1 == b2 && in_bin == 1 && bin_end < cut) {        // the one logit in it belongs to the prefix
                cut = (uint32_t)bin_end;
                quota = 0x7fffffff;
                break;
            }
            const uint64_t half = (end - base + 1) / 2;
            if (b2 == kBins) {                                     // the last bin that has any must
                int filled = bins[1] ? 2 * tid + 1 : bins[0] ? 2 * tid : 0;
                filled = __reduce_max_sync(0xffffffffu, filled);
                if (lane == 0) sh.warp_i[warp] = filled;
                __syncthreads();
                b2 = b1;
                for (int w = 0; w < kSampleWarps; ++w) b2 = max(b2, sh.warp_i[w]);
            }
            end = min(end, base + ((uint64_t)(b2 + 1) << shift) - 1);
            end = max(end, next);                                  // (a rounding past the end)
            trial = end - next >= half;
            middle = trial ? base + half : next;
            // what lies between the old base and the new one is above the range from now on
            part = strip_weight((uint32_t)base, (uint32_t)(middle - base), 0, 0);
            if (!trial) {
                base = next;
                kept_near += part;
                kept_from = (uint32_t)base;
            }
        }
    }

    // ---- the draw: running sums in index order over threads, CTAs, and then inside one thread's strip
    if (min_p_cut < cut) { cut = min_p_cut; quota = 0x7fffffff; }
    int tie_rank = 0;                                              // equal ones before this thread's strip
    if (quota != 0x7fffffff) {
        int ties = 0;
        for (int i = 0; i < p.strip; ++i) ties += mine[i] == top - cut;
        int run = ties;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) { const int o = __shfl_up_sync(0xffffffffu, run, d); if (lane >= d) run += o; }
        __syncthreads();
        if (lane == 31) sh.warp_i[warp] = run;
        __syncthreads();
        int total = 0;
        for (int w = 0; w < kSampleWarps; ++w) { if (w < warp) run += sh.warp_i[w]; total += sh.warp_i[w]; }
        if (tid < C) to_all(sh.ties, total);
        meet();
        tie_rank = run - ties;
        for (int c = 0; c < rank; ++c) tie_rank += sh.ties[c];
    }
    // (images below top - cut, the padding's 0 among them, are cut)
    if (kept_from > cut) { kept_near = 0.0; kept_from = 0u; }      // (min-p cuts deeper)
    const double sum = quota != 0x7fffffff ? kept_near + strip_weight(kept_from, cut - kept_from, tie_rank, quota)
                       : cut == furthest   ? strip_weight_all(cut + 1u)
                                           : kept_near + strip_weight(kept_from, cut - kept_from + 1u, 0, 0);
    // Running sums one after the other, so that a thread without weight ends exactly where the one before it does, and the end of a
    // warp or a CTA is the same number as the start of the next: one thread, with weight, holds the target.
    double run = 0.0;
#pragma unroll
    for (int j = 0; j < 32; ++j) {
        const double s = __shfl_sync(0xffffffffu, sum, j);
        if (lane >= j) run += s;
    }
    __syncthreads();
    if (lane == 31) sh.warp_d[warp][0] = run;
    __syncthreads();
    double block = 0.0, offset = 0.0;
    for (int w = 0; w < kSampleWarps; ++w) { if (w == warp) offset = block; block += sh.warp_d[w][0]; }
    if (tid < C) to_all(sh.kept_sum, block);
    meet();
    double total = 0.0, before = 0.0, cta_end = 0.0;
    for (int c = 0; c < C; ++c) { if (c == rank) before = total; total += sh.kept_sum[c]; if (c == rank) cta_end = total; }
    const double target = draw_at(total);
    if (!(before <= target && target < cta_end)) return;           // another CTA's (no remote access from here on)
    const double inner = offset + run, prev = __shfl_up_sync(0xffffffffu, inner, 1);
    const double start = before + (lane == 0 ? offset : prev), end = before + inner;
    const uint32_t holder = __ballot_sync(0xffffffffu, start <= target && target < end);
    if (!holder) return;
    // the warp walks through the strip of the thread that holds the target, 32 logits at a time
    const int who = __ffs(holder) - 1;
    const uint32_t* const strip = img + (warp * 32 + who) * p.strip;
    double at = __shfl_sync(0xffffffffu, start, who);
    int ties_before = __shfl_sync(0xffffffffu, tie_rank, who), found = -1;
    for (int i0 = 0; i0 < p.strip; i0 += 32) {
        const int i = i0 + lane;
        const uint32_t u = i < p.strip ? strip[i] : 0u, d = top - u;
        const uint32_t tied = __ballot_sync(0xffffffffu, i < p.strip && d == cut);
        const int my_rank = ties_before + __popc(tied & ((1u << lane) - 1u));
        ties_before += __popc(tied);
        const double w = i < p.strip && (d < cut || (d == cut && my_rank < quota)) ? weight(u) : 0.0;
        double upto = at;
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            const double o = __shfl_sync(0xffffffffu, w, j);
            if (lane >= j) upto += o;
        }
        const uint32_t weighed = __ballot_sync(0xffffffffu, w > 0.0), past = __ballot_sync(0xffffffffu, w > 0.0 && upto > target);
        if (past) { found = i0 + __ffs(past) - 1; break; }
        if (weighed) found = i0 + 31 - __clz(weighed);             // (the same sum in another order may fall a rounding short: the last one then)
        at = __shfl_sync(0xffffffffu, upto, 31);
    }
    if (lane == 0) {
        p.token[r] = first + (warp * 32 + who) * p.strip + found;
        if (p.logprob) p.logprob[r] = (float)((per_bit * behind(strip[found]) - log2(total)) * 0.69314718055994531);
    }
}

// ------------------------------------------------------------------ rows without a filter
// The draw alone: one pass over a row.  A warp reads 512 consecutive logits at a time into registers, 16 a lane, the next block's on the
// way meanwhile, and keeps their largest and the sum of their weights relative to it (64 bits).  The cluster agrees on the row's largest
// logit, puts the sums on it and adds them up in index order; the warp whose sums hold the target reads that block once more and
// walks through it.
// Bound: the 64-bit pipe and the issue slots (fourteen 64-bit instructions of about thirty a logit); 1000 rows of 128256: 184 us,
// 2.8 TB/s, the pipe half busy.  (Two blocks a pass, without the copy from the block on the way, spilled: 223 us.)  32-bit weights
// were slower with the bound of their error that was tried: as large as a flat row's weights, so that most rows had to be summed
// again in 64 bits (512 rows: 165 us, this kernel 97).
constexpr int kDrawThreads = 256, kDrawWarps = kDrawThreads / 32;
constexpr int kDrawBlock = 512, kDrawPer = kDrawBlock / 32;
constexpr int kDrawBlocks = kMaxCluster * kSampleThreads * kMaxStrip / kDrawBlock + 1;      // of a row at most; one more for an unaligned start

struct DrawShared {
    double sum[kDrawBlocks];
    float top[kDrawBlocks];
    uint32_t best[kMaxCluster];                    // filled by all CTAs of the cluster, one entry each
    double total[kMaxCluster];
    double warp_sum[kDrawWarps];
    uint32_t warp_top[kDrawWarps];
    int32_t first_block;
};

template <typename T>
__global__ void __launch_bounds__(kDrawThreads, 4)
kap_sample_draw_kernel(const SampleParams p)
{
    __shared__ __align__(16) DrawShared sh;
    constexpr int kVec = 16 / (int)sizeof(T), kLoads = kDrawPer / kVec;
    const int C = p.cluster, r = blockIdx.x / C, rank = blockIdx.x % C, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (C > 1) cluster_arrive();                                   // (its wait: every peer runs before anybody writes to it)
    const T* row = reinterpret_cast<const T*>(p.logits) + (long long)r * p.row_stride;
    // places are counted from the 16-byte boundary at or before the row's first logit; `skip` of them are not the row's
    const int skip = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T)), end = skip + p.vocab;
    const int all_blocks = (end + kDrawBlock - 1) / kDrawBlock, per_cta = (all_blocks + C - 1) / C;
    const int block0 = min(all_blocks, rank * per_cta), n_blocks = min(all_blocks, block0 + per_cta) - block0;
    const float t = p.temperature ? p.temperature[r] : 1.f;
    const double u01 = (double)p.uniform[r], per_bit = 1.4426950408889634 / (double)t;
    // logit e of load l of this lane has the place place_of(b, l) + e
    auto place_of = [&](int b, int l) { return (block0 + b) * kDrawBlock + l * (32 * kVec) + lane * kVec; };
    auto load = [&](int b, uint4 (&raw)[kLoads]) {                 // places that are not the row's: all bits set, which is NaN
        const int from = (block0 + b) * kDrawBlock;
        const T* const at = row + (place_of(b, 0) - skip);
        if (from >= skip && from + kDrawBlock <= end) {
#pragma unroll
            for (int l = 0; l < kLoads; ++l) raw[l] = __ldcs(reinterpret_cast<const uint4*>(at) + 32 * l);
        } else {                                                   // an end of the row
#pragma unroll
            for (int l = 0; l < kLoads; ++l) {
                raw[l] = make_uint4(0xffffffffu, 0xffffffffu, 0xffffffffu, 0xffffffffu);
                T* e = reinterpret_cast<T*>(&raw[l]);
#pragma unroll
                for (int j = 0; j < kVec; ++j) {
                    const int i = place_of(b, l) + j;
                    if (i >= skip && i < end) e[j] = row[i - skip];
                }
            }
        }
    };
    auto logit = [](const uint4 (&raw)[kLoads], int q) { return as_float(reinterpret_cast<const T*>(&raw[q / kVec])[q % kVec]); };
    // s += 2^((v - from) / T / ln 2), `from` the largest logit, for logits above `bar`: none for -inf and NaN, nor more than 2^-1021 below the
    // largest one, which is counted whatever T; beside +inf, which stands for the largest finite number, only +inf.  (The
    // conversion runs beside the sums, on its own pipe.)
    constexpr float kLargest = 3.402823466e38f;
    auto widen = [](float v) { return (double)fminf(v, kLargest); };
    const double reach = 1021.0 / per_bit;                         // (+inf for an endless T)
    auto bar_of = [&](uint32_t image) {
        const float before = image_logit(image - 1u);              // of +inf: the largest finite number
        const double bar = widen(image_logit(image)) - reach;
        return image == kImagePlusInf ? before : bar < -(double)kLargest ? -INFINITY : fminf(__double2float_ru(bar), before);
    };
    auto add_weight = [&](double& s, float v, double from, float bar) {
        const double w = exp2_f64(widen(v) - from, per_bit);
        if (v > bar) s += w;
    };

    uint32_t best = 0u;
    uint4 raw[kLoads];
    if (warp < n_blocks) load(warp, raw);
    for (int b = warp; b < n_blocks; b += kDrawWarps) {
        float top = -INFINITY;                                     // (fmaxf passes over NaN)
        uint4 now[kLoads];
#pragma unroll
        for (int l = 0; l < kLoads; ++l) now[l] = raw[l];
        if (b + kDrawWarps < n_blocks) load(b + kDrawWarps, raw);
#pragma unroll
        for (int q = 0; q < kDrawPer; ++q) top = fmaxf(top, logit(now, q));
        const uint32_t image = __reduce_max_sync(0xffffffffu, logit_image(top));
        best = max(best, image);
        const float block_top = image_logit(image), bar = bar_of(image);
        const double from = widen(block_top);
        double s0 = 0.0, s1 = 0.0;
#pragma unroll
        for (int q = 0; q < kDrawPer; q += 2) {
            add_weight(s0, logit(now, q), from, bar);
            add_weight(s1, logit(now, q + 1), from, bar);
        }
        s0 += s1;
#pragma unroll
        for (int d = 16; d; d >>= 1) s0 += __shfl_xor_sync(0xffffffffu, s0, d);
        if (lane == 0) { sh.top[b] = block_top; sh.sum[b] = s0; }
    }
    if (lane == 0) sh.warp_top[warp] = best;
    if (tid == 0) sh.first_block = n_blocks;
    __syncthreads();
    if (C > 1) cluster_wait();
    auto to_all = [&](auto* slot, auto v) { put_remote(map_to_cta(smem_u32(slot + rank), tid), v); };
    auto meet = [&] { if (C > 1) cluster_sync(); else __syncthreads(); };
    if (tid < C) {
        best = 0u;
        for (int w = 0; w < kDrawWarps; ++w) best = max(best, sh.warp_top[w]);
        to_all(reinterpret_cast<int32_t*>(sh.best), (int32_t)best);
    }
    meet();
    uint32_t top = 0u;
    for (int c = 0; c < C; ++c) top = max(top, sh.best[c]);
    if (top <= kImageMinusInf) {                                   // no token at all
        if (rank == 0 && tid == 0) {
            p.token[r] = -1;
            if (p.logprob) p.logprob[r] = -INFINITY;
        }
        return;
    }
    const float top_logit = image_logit(top);
    if (!(t > 0.f)) {                                              // greedy: the first CTA that has the largest logit
        int c = 0;
        while (sh.best[c] != top) ++c;
        if (c != rank) return;
        for (int b = tid; b < n_blocks; b += kDrawThreads)
            if (sh.top[b] == top_logit) atomicMin(&sh.first_block, b);
        __syncthreads();
        if (warp == 0) {
            load(sh.first_block, raw);
            int at = 0x7fffffff;
#pragma unroll
            for (int q = kDrawPer - 1; q >= 0; --q)
                if (logit(raw, q) == top_logit) at = place_of(sh.first_block, q / kVec) + q % kVec;
            at = __reduce_min_sync(0xffffffffu, at);
            if (lane == 0) {
                p.token[r] = at - skip;
                if (p.logprob) p.logprob[r] = 0.f;
            }
        }
        return;
    }
    const double x_max = widen(top_logit);
    const float bar = bar_of(top);
    // Running sums one after the other: consecutive blocks to a thread, then threads, warps and CTAs, so that a thread without weight
    // ends exactly where the one before it does, and the end of a warp or a CTA is the same number as the start of the next.
    const int per_thread = (n_blocks + kDrawThreads - 1) / kDrawThreads, own0 = min(n_blocks, tid * per_thread), own1 = min(n_blocks, own0 + per_thread);
    double mine = 0.0;
    for (int b = own0; b < own1; ++b) {
        double s = 0.0;
        add_weight(s, sh.top[b], x_max, bar);
        s *= sh.sum[b];
        sh.sum[b] = s;                                             // (this thread's alone, until the walk below)
        mine += s;
    }
    double run = 0.0;
#pragma unroll
    for (int j = 0; j < 32; ++j) {
        const double s = __shfl_sync(0xffffffffu, mine, j);
        if (lane >= j) run += s;
    }
    if (lane == 31) sh.warp_sum[warp] = run;
    __syncthreads();
    double cta = 0.0, offset = 0.0;
    for (int w = 0; w < kDrawWarps; ++w) { if (w == warp) offset = cta; cta += sh.warp_sum[w]; }
    if (tid < C) to_all(sh.total, cta);
    meet();                                                        // (no remote access from here on)
    double total = 0.0, before = 0.0, cta_end = 0.0;
    for (int c = 0; c < C; ++c) {
        if (c == rank) before = total;
        total += sh.total[c];
        if (c == rank) cta_end = total;
    }
    const double target = u01 >= 0.0 ? fmin(u01 * total, total * 0.99999999999999978) : 0.0;
    if (!(before <= target && target < cta_end)) return;
    const double inner = offset + run, prev = __shfl_up_sync(0xffffffffu, inner, 1);
    const double start = before + (lane == 0 ? offset : prev);
    const uint32_t holder = __ballot_sync(0xffffffffu, start <= target && target < before + inner);
    if (!holder) return;
    const int who = __ffs(holder) - 1;
    double at = __shfl_sync(0xffffffffu, start, who), upto = at;
    const int b0 = __shfl_sync(0xffffffffu, own0, who), b1 = __shfl_sync(0xffffffffu, own1, who);
    int block = -1;                                                // the last one with weight when a rounding falls short
    for (int b = b0; b < b1; ++b) {
        const double s = sh.sum[b];
        if (!(s > 0.0)) continue;
        if (block >= 0 && upto > target) break;
        block = b;
        at = upto;
        upto += s;
    }
    load(block, raw);
    int found = -1;                                                // likewise
    float chosen = 0.f;
    for (int l = 0; l < kLoads; ++l) {
        // this load's logits in index order: a lane's one after the other, lane by lane
        uint4 part = raw[0];
#pragma unroll
        for (int j = 1; j < kLoads; ++j) if (l == j) part = raw[j];
        float v[kVec];
        double w[kVec], lane_sum = 0.0;
#pragma unroll
        for (int j = 0; j < kVec; ++j) {
            v[j] = as_float(reinterpret_cast<const T*>(&part)[j]);
            w[j] = 0.0;
            add_weight(w[j], v[j], x_max, bar);
            lane_sum += w[j];
        }
        double to = at;
        for (int j = 0; j < 32; ++j) {
            const double s = __shfl_sync(0xffffffffu, lane_sum, j);
            if (lane > j) to += s;
        }
        int place = -1;
        float v_place = 0.f;
        bool past = false;
#pragma unroll
        for (int j = 0; j < kVec; ++j)
            if (w[j] > 0.0 && !past) {
                to += w[j];
                place = place_of(block, l) + j;
                v_place = v[j];
                past = to > target;
            }
        const uint32_t over = __ballot_sync(0xffffffffu, past), weighed = __ballot_sync(0xffffffffu, place >= 0);
        if (weighed) {
            const int pick = over ? __ffs(over) - 1 : 31 - __clz(weighed);
            found = __shfl_sync(0xffffffffu, place, pick);
            chosen = __shfl_sync(0xffffffffu, v_place, pick);
        }
        if (over) break;
        at = __shfl_sync(0xffffffffu, to, 31);
    }
    if (lane == 0) {
        p.token[r] = found - skip;
        if (p.logprob) p.logprob[r] = (float)(((widen(chosen) - x_max) * per_bit - log2(total)) * 0.69314718055994531);
    }
}

}  // namespace
}  // namespace kap

extern "C" kap_status kap_sample_tokens(
    const void* logits, int32_t logits_type, int64_t row_stride, int32_t rows, int32_t vocab, const float* temperature,
    const int32_t* top_k, const float* top_p, const float* min_p, const float* uniform, int32_t* token, float* logprob,
    void* cuda_stream)
{
    using namespace kap;
    if (logits_type != KAP_LOGITS_F32 && logits_type != KAP_LOGITS_BF16)
        return fail(KAP_ERR_UNSUPPORTED, "logits_type %d (KAP_LOGITS_F32 = 0, KAP_LOGITS_BF16 = 1)", logits_type);
    if (rows < 0 || vocab < 1 || row_stride < vocab)
        return fail(KAP_ERR_INVALID_ARG, "rows %d, vocab %d, row_stride %lld", rows, vocab, (long long)row_stride);
    constexpr int kMost = kMaxCluster * kSampleThreads * kMaxStrip;
    if (vocab > kMost) return fail(KAP_ERR_UNSUPPORTED, "vocab %d (at most %d: a row stays in a cluster's shared memory)", vocab, kMost);
    if (rows == 0) return KAP_OK;
    if (!logits || !uniform || !token) return fail(KAP_ERR_INVALID_ARG, "NULL pointer");
    if (reinterpret_cast<uintptr_t>(logits) & (logits_type == KAP_LOGITS_F32 ? 3 : 1))
        return fail(KAP_ERR_INVALID_ARG, "logits are not aligned to their type");
    if ((reinterpret_cast<uintptr_t>(temperature) | reinterpret_cast<uintptr_t>(top_k) | reinterpret_cast<uintptr_t>(top_p) |
         reinterpret_cast<uintptr_t>(min_p) | reinterpret_cast<uintptr_t>(uniform) | reinterpret_cast<uintptr_t>(token) |
         reinterpret_cast<uintptr_t>(logprob)) & 3)
        return fail(KAP_ERR_INVALID_ARG, "a parameter or result array is not 4-byte aligned");
    SampleParams p{logits, row_stride, vocab, 0, 0, 1, temperature, top_p, min_p, uniform, top_k, token, logprob};
    int& C = p.cluster;                                            // CTAs of a row
    const bool f32 = logits_type == KAP_LOGITS_F32;
    void (*kernel)(SampleParams);
    cudaLaunchConfig_t cfg{};
    const int draw_blocks = (vocab + kDrawBlock - 1) / kDrawBlock;
    cudaError_t e = cudaSuccess;
    if (!top_k && !top_p && !min_p && (draw_blocks > 32 || rows > kSms)) {
        // Without filters, unless the rows are short and few (this kernel / the other one: 8192 logits, 148 rows 9.2 / 8.4 us, 256 rows
        // 9.7 / 11.8; 32000 logits, 8 rows 9.6 / 8.2, 100 rows 13.3 / 16.9; 128256 logits, 512 rows 97 / 248).  CTAs of a row: three on an
        // SM and a block for each of their warps, and two for long rows, whose tail one CTA would stretch (128256 logits, 1 / 2 / 4 / 8
        // CTAs a row: 8 rows 49 / 28 / 18 / 12 us, 100 rows 49 / 34 / 28 / 30, 512 rows 111 / 97 / 106 / 123; 1000 rows of 32000
        // 55 / 62 / 81 / 118).
        kernel = f32 ? kap_sample_draw_kernel<float> : kap_sample_draw_kernel<__nv_bfloat16>;
        while (C < 8 && C * 2 * kDrawWarps <= draw_blocks && (int64_t)rows * C * 2 <= 3 * kSms) C *= 2;
        if (C == 1 && draw_blocks >= 128) C = 2;
        cfg.blockDim = dim3(kDrawThreads);
    } else {
        // As many CTAs as keep two of them on an SM, 33 logits a thread (64 rows of 128256 with mixed filters: 61 us; 17 logits 102, 65
        // logits 64).  With few rows more, while that leaves a thread a strip worth its barriers and the large clusters half of the SMs,
        // since they do not fit everywhere (top-k to 80 and top-p: 1 row of 32000 11.4 with 8 CTAs, 12.9 with 16, 14.0 with 2; 16 rows
        // 13.0 with 4, 16.1 with 8; 16 rows of 50257 14.0 with 4, 17.0 with 8, 26 with 16).
        kernel = f32 ? kap_sample_rows_kernel<float> : kap_sample_rows_kernel<__nv_bfloat16>;
        auto strip_of = [&](int c) { const int s = ((vocab + c - 1) / c + kSampleThreads - 1) / kSampleThreads; return s | 1; };
        while (C < kMaxCluster && strip_of(C) > 33) C *= 2;
        while (C < kMaxCluster && strip_of(C) > (C < 8 ? 5 : 13) && (int64_t)rows * C * 2 <= (C < 4 ? kSms : kSms / 2)) C *= 2;
        p.strip = strip_of(C);
        p.slice = p.strip * kSampleThreads;
        auto smem_for = [](int slice) { return (sizeof(SampleShared) + 15) / 16 * 16 + ((size_t)slice + 4) * sizeof(uint32_t); };
        static_assert((sizeof(SampleShared) + 15) / 16 * 16 + ((size_t)kSampleThreads * kMaxStrip + 4) * 4 <= 232448, "more than 227 KiB of shared memory");
        cfg.blockDim = dim3(kSampleThreads);
        cfg.dynamicSmemBytes = smem_for(p.slice);
        // (attributes belong to the current device; setting them again costs less than a microsecond)
        e = cudaFuncSetAttribute((const void*)kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_for(kSampleThreads * kMaxStrip));
        if (e == cudaSuccess && C > 8) e = cudaFuncSetAttribute((const void*)kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    }
    if (rows > 0x7fffffff / C) return fail(KAP_ERR_UNSUPPORTED, "%d rows", rows);
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)C; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cfg.gridDim = dim3((unsigned)rows * (unsigned)C);
    cfg.stream = (cudaStream_t)cuda_stream;
    cfg.attrs = attr;
    cfg.numAttrs = C > 1 ? 1 : 0;
    if (e == cudaSuccess) e = cudaLaunchKernelEx(&cfg, kernel, p);
    if (e != cudaSuccess) return fail(KAP_ERR_CUDA, "kap_sample_tokens launch failed: %s", cudaGetErrorString(e));
    count_launch();
    return KAP_OK;
}
