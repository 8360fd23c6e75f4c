// kap_sample_tokens: draw one token per logits row from the truncated softmax with a given uniform number.
//
// Mathematics, for a row x with temperature T > 0:  w_i = exp((x_i - max x) / T);  top-k keeps the k largest
// logits, top-p of those the shortest prefix by descending value whose weight reaches p of theirs, min-p those
// with w_i >= min_p;  the token is the first index, in vocabulary order, whose running sum of kept weights
// exceeds u times their total.  Equal logits rank by index.  A sort is not needed: each filter is a threshold
// on the logit (found by bisection on an order-preserving integer image, counting or summing what lies above)
// plus the number of logits equal to it that still count.  Sums are held in 64 bits: the token is decided by
// comparing long sums, and 32-bit ones over 128 256 weights would move a border in every few hundred rows.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "kap_internal.h"

namespace kap {
void count_launch();

namespace {

constexpr int kSampleThreads = 1024;
constexpr uint32_t kImageMinusInf = 0x007fffffu;   // image of -inf; nothing at or below it has weight

__device__ __forceinline__ uint32_t logit_image(float v) {          // NaN lowest, -0 = +0
    const uint32_t u = __float_as_uint(v + 0.0f);
    return v != v ? 0u : u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float image_logit(uint32_t u) {
    return __uint_as_float(u ^ ((u >> 31) ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ float load_logit(const float* x, int i) { return x[i]; }
__device__ __forceinline__ float load_logit(const __nv_bfloat16* x, int i) { return __bfloat162float(x[i]); }

// the sum (in a fixed order) over the block, in every thread
template <typename V>
__device__ V block_sum(V v, V* scratch) {
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    v = scratch[threadIdx.x & 31];
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}

struct SampleParams {
    const void* logits;
    long long row_stride;
    int32_t vocab;
    const float *temperature, *top_p, *min_p, *uniform;
    const int32_t* top_k;
    int32_t* token;
    float* logprob;
};

template <typename T>
__global__ void __launch_bounds__(kSampleThreads)
kap_sample_rows_kernel(const SampleParams p)
{
    __shared__ double scratch[33];
    __shared__ double scan[kSampleThreads + 1];
    __shared__ int tie_scan[kSampleThreads + 1];
    __shared__ unsigned long long best;
    const int r = blockIdx.x, tid = threadIdx.x, V = p.vocab;
    const T* x = reinterpret_cast<const T*>(p.logits) + (long long)r * p.row_stride;
    if (tid == 0) best = 0ull;
    __syncthreads();
    unsigned long long mine = 0ull;
    for (int i = tid; i < V; i += kSampleThreads) {
        const unsigned long long k = ((unsigned long long)logit_image(load_logit(x, i)) << 32) | (uint32_t)~i;
        mine = k > mine ? k : mine;
    }
    atomicMax(&best, mine);
    __syncthreads();
    const uint32_t top = (uint32_t)(best >> 32);
    const int top_index = (int)~(uint32_t)best;
    const float t = p.temperature ? p.temperature[r] : 1.f;
    if (top <= kImageMinusInf || !(t > 0.f)) {                    // no token at all / greedy
        if (tid == 0) {
            const bool none = top <= kImageMinusInf;
            p.token[r] = none ? -1 : top_index;
            if (p.logprob) p.logprob[r] = none ? -INFINITY : 0.f;
        }
        return;
    }
    const double x_max = (double)image_logit(top), td = (double)t;
    auto scaled = [&](uint32_t img) { return img == top ? 0.0 : ((double)image_logit(img) - x_max) / td; };
    auto weight = [&](uint32_t img) { return img <= kImageMinusInf ? 0.0 : exp(scaled(img)); };

    // the threshold (image, how many equal to it count) of top-k
    uint32_t cut = 0;                                             // everything above it counts ...
    int quota = V;                                                // ... and so many equal to it, lowest index first
    const int k = p.top_k ? p.top_k[r] : 0;
    if (k > 0 && k < V) {
        for (int bit = 31; bit >= 0; --bit) {                     // the largest image with at least k at or above it
            const uint32_t c = cut | (1u << bit);
            int n = 0;
            for (int i = tid; i < V; i += kSampleThreads) n += logit_image(load_logit(x, i)) >= c;
            if (block_sum<int>(n, (int*)scratch) >= k) cut = c;
        }
        int above = 0;
        for (int i = tid; i < V; i += kSampleThreads) above += logit_image(load_logit(x, i)) > cut;
        quota = k - block_sum<int>(above, (int*)scratch);
    }
    auto sum_above = [&](uint32_t c) {                            // weight strictly above the image c
        double s = 0.0;
        for (int i = tid; i < V; i += kSampleThreads) {
            const uint32_t u = logit_image(load_logit(x, i));
            if (u > c) s += weight(u);
        }
        return block_sum<double>(s, scratch);
    };
    const float top_p = p.top_p ? p.top_p[r] : 1.f;
    if (top_p < 1.f) {
        int ties = 0;
        for (int i = tid; i < V; i += kSampleThreads) ties += logit_image(load_logit(x, i)) == cut;
        ties = min(block_sum<int>(ties, (int*)scratch), quota);
        const double target = (double)top_p * (sum_above(cut) + ties * weight(cut));
        // the smallest image, not below the present cut, such that less than the target lies above it
        uint32_t lo = cut, hi = top;                              // sum_above(top) = 0 < target, or top alone stays
        while (lo < hi) {
            const uint32_t mid = lo + (hi - lo) / 2;
            if (sum_above(mid) < target) hi = mid; else lo = mid + 1;
        }
        const double w = weight(lo), left = target - sum_above(lo);
        const int most = lo == cut ? quota : V;
        const double n = w > 0.0 ? ceil(left / w) : (double)most;
        quota = n < 1.0 ? 1 : n < (double)most ? (int)n : most;
        cut = lo;
    }
    const float min_p = p.min_p ? p.min_p[r] : 0.f;
    const double floor_z = min_p > 0.f ? log((double)min_p) : -INFINITY;

    // running sums in vocabulary order: thread t owns a contiguous strip
    const int per = (V + kSampleThreads - 1) / kSampleThreads;
    const int i0 = min(V, tid * per), i1 = min(V, i0 + per);
    int ties = 0;
    for (int i = i0; i < i1; ++i) ties += logit_image(load_logit(x, i)) == cut;
    tie_scan[tid + 1] = ties;
    __syncthreads();
    if (tid == 0) {
        tie_scan[0] = 0;
        for (int j = 1; j <= kSampleThreads; ++j) tie_scan[j] += tie_scan[j - 1];
    }
    __syncthreads();
    // sum of the strip's kept weights; *found: the first index past the target, or (the same sum in another
    // order may fall a rounding short of it) the last one with weight
    auto walk = [&](double from, double target, int* found) {
        int rank = tie_scan[tid];
        for (int i = i0; i < i1; ++i) {
            const uint32_t u = logit_image(load_logit(x, i));
            const bool in = u > cut || (u == cut && rank++ < quota);
            if (!in || u <= kImageMinusInf || !(scaled(u) >= floor_z)) continue;
            const double w = weight(u);
            from += w;
            if (found && w > 0.0) {
                *found = i;
                if (from > target) return from;
            }
        }
        return from;
    };
    scan[tid + 1] = walk(0.0, 0.0, nullptr);
    __syncthreads();
    if (tid == 0) {
        scan[0] = 0.0;
        for (int j = 1; j <= kSampleThreads; ++j) scan[j] += scan[j - 1];
    }
    __syncthreads();
    const double total = scan[kSampleThreads];
    const double u01 = (double)p.uniform[r];
    const double target = u01 >= 0.0 ? fmin(u01 * total, total * 0.99999999999999978) : 0.0;
    if (scan[tid] <= target && scan[tid + 1] > target) {
        int found = -1;
        walk(scan[tid], target, &found);
        p.token[r] = found;
        if (p.logprob) p.logprob[r] = (float)(scaled(logit_image(load_logit(x, found))) - log(total));
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
    if (rows == 0) return KAP_OK;
    if (!logits || !uniform || !token) return fail(KAP_ERR_INVALID_ARG, "NULL pointer");
    if (reinterpret_cast<uintptr_t>(logits) & (logits_type == KAP_LOGITS_F32 ? 3 : 1))
        return fail(KAP_ERR_INVALID_ARG, "logits are not aligned to their type");
    SampleParams p{logits, row_stride, vocab, temperature, top_p, min_p, uniform, top_k, token, logprob};
    if (logits_type == KAP_LOGITS_F32)
        kap_sample_rows_kernel<float><<<(unsigned)rows, kSampleThreads, 0, (cudaStream_t)cuda_stream>>>(p);
    else
        kap_sample_rows_kernel<__nv_bfloat16><<<(unsigned)rows, kSampleThreads, 0, (cudaStream_t)cuda_stream>>>(p);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return fail(KAP_ERR_CUDA, "kap_sample_tokens launch failed: %s", cudaGetErrorString(e));
    count_launch();
    return KAP_OK;
}
