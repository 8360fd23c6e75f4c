// kap_adjust_logits: penalties for repeated tokens, biases and grammar masks on logits rows, in front of kap_sample_tokens (the paper fixes no
// sampling rule).
//
// Mathematics, for token t of a row with logit x: c = times t occurs in the answer so far, s = t occurs in the prompt or the answer,
//     x1 = s ? (x > 0 ? x / r : x r) : x,   x2 = x1 - f c - p [c > 0],   x3 = x2 + bias_t,   out = allowed_t ? x3 : -inf,
// in fp32, rounded to the logits' type once.
// Layout: a cluster of CTAs per row; CTA i owns the i-th slice of the vocabulary, copies it under the mask, and keeps a 32-bit word for each
// of its tokens in shared memory (times in the answer; whether in the prompt).  The history is dealt out over the cluster: each
// CTA clears, then counts its share's tokens in their owners' words through distributed shared memory, so no word is touched that no
// token names, and the history is read from memory once (its second and third pass hit L1 / L2).  Whoever then takes a token's word out
// (an atomic exchange) corrects that token's logit; which thread it is does not change the value.  Tokens with a bias are left to the
// owner of the bias.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "kap_internal.h"

namespace kap {
void count_launch();

namespace {

constexpr int kLogitThreads = 512;
constexpr uint32_t kInPrompt = 1u << 30, kHasBias = 1u << 31, kCountMask = kInPrompt - 1;

struct LogitParams {
    const void* logits;
    void* out;
    const int32_t* history;
    const long long* history_at;                              // [rows][3]: first token, first of the answer, end
    const float *repetition, *presence, *frequency;
    const int32_t *bias_indptr, *bias_token;
    const float* bias_value;
    const uint32_t* allowed;
    const int32_t* allowed_row;
    int32_t* status;
    long long row_stride, out_stride, history_len, bias_len, allowed_stride;
    int32_t rows, vocab, num_masks, slice;                    // slice: tokens of a CTA, a multiple of 32
};

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ uint32_t peer_addr(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void cluster_arrive_release() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait_acquire() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

template <typename T> __device__ __forceinline__ float to_float(T x);
template <> __device__ __forceinline__ float to_float(float x) { return x; }
template <> __device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float(float x) { return __float2bfloat16_rn(x); }
template <typename T> __device__ __forceinline__ uint4 minus_inf_vector();
template <> __device__ __forceinline__ uint4 minus_inf_vector<float>() { return make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u); }
template <> __device__ __forceinline__ uint4 minus_inf_vector<__nv_bfloat16>() { return make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u); }

struct Rules { float repetition, presence, frequency; };
__device__ __forceinline__ float penalised(float x, uint32_t word, const Rules& r) {
    const uint32_t c = word & kCountMask;
    if (word & (kInPrompt | kCountMask)) x = x > 0.f ? __fdiv_rn(x, r.repetition) : x * r.repetition;
    if (c) x = x - r.frequency * (float)c - r.presence;
    return x;
}

template <typename T>
__global__ void __launch_bounds__(kLogitThreads)
kap_adjust_logits_kernel(const LogitParams p)
{
    extern __shared__ uint32_t words[];                       // [slice], used when the row has a history or biases
    cluster_arrive_release();                                 // (peers' words may be written once they run: waited for below)
    const int tid = threadIdx.x, n_cta = gridDim.x, rank = blockIdx.x, row = blockIdx.y;     // (the cluster spans x)
    const T* const in = reinterpret_cast<const T*>(p.logits) + row * p.row_stride;
    T* const out = reinterpret_cast<T*>(p.out) + row * p.out_stride;
    const bool in_place = p.logits == p.out;
    Rules r{1.f, 0.f, 0.f};
    if (p.repetition) { const float v = p.repetition[row]; if (v > 0.f) r.repetition = v; }
    if (p.presence) { const float v = p.presence[row]; if (v == v) r.presence = v; }
    if (p.frequency) { const float v = p.frequency[row]; if (v == v) r.frequency = v; }
    long long h0 = 0, h1 = 0, h2 = 0;
    if (p.history && (r.repetition != 1.f || r.presence != 0.f || r.frequency != 0.f)) {
        h0 = p.history_at[row * 3ll]; h1 = p.history_at[row * 3ll + 1]; h2 = p.history_at[row * 3ll + 2];
        if (h0 < 0 || h1 < h0 || h2 < h1 || h2 > p.history_len || h2 - h0 > (long long)kCountMask) {
            if (tid == 0 && rank == 0 && p.status) atomicOr(p.status, 1 << KAP_ERR_DEVICE_INDEX);
            h0 = h1 = h2 = 0;
        }
    }
    const bool counted = h2 > h0;                             // the same for the whole cluster
    int b0 = 0, b1 = 0;
    if (p.bias_token) {
        b0 = p.bias_indptr[row]; b1 = p.bias_indptr[row + 1];
        if (b0 < 0 || b1 < b0 || b1 > p.bias_len) {
            if (tid == 0 && rank == 0 && p.status) atomicOr(p.status, 1 << KAP_ERR_DEVICE_INDEX);
            b0 = b1 = 0;
        }
    }
    const uint32_t* mask = nullptr;
    if (p.allowed) {
        const int m = p.allowed_row ? p.allowed_row[row] : row;
        if (m >= 0 && m < p.num_masks) mask = p.allowed + m * p.allowed_stride;
        else if (m != -1 && tid == 0 && rank == 0 && p.status) atomicOr(p.status, 1 << KAP_ERR_DEVICE_INDEX);
    }
    const int v0 = min(rank * p.slice, p.vocab), v1 = min(v0 + p.slice, p.vocab);
    const uint32_t base = smem_addr(words);
    // this CTA's share of the history
    const long long share = (h2 - h0 + n_cta - 1) / n_cta, s0 = min(h0 + rank * share, h2), s1 = min(s0 + share, h2);
    auto word_of = [&](int t) { return peer_addr(base + (uint32_t)(t % p.slice) * 4u, (uint32_t)(t / p.slice)); };

    cluster_wait_acquire();
    if (counted) {
        for (long long i = s0 + tid; i < s1; i += kLogitThreads) {
            const int t = p.history[i];
            if (t >= 0 && t < p.vocab) asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(word_of(t)), "r"(0u) : "memory");
        }
        for (int i = b0 + tid; i < b1; i += kLogitThreads) {
            const int t = p.bias_token[i];
            if (t >= v0 && t < v1) words[t - v0] = 0u;
        }
        cluster_arrive_release();
    }
    // ---- the slice, under the mask
    if (!in_place || mask) {
        constexpr int kVec = 16 / sizeof(T);
        const uintptr_t from = reinterpret_cast<uintptr_t>(in + v0), to = reinterpret_cast<uintptr_t>(out + v0);
        if (((from ^ to) & 15) == 0) {
            const int head = min((int)((16 - (to & 15)) & 15) / (int)sizeof(T), v1 - v0), n_vec = (v1 - v0 - head) / kVec;
            auto single = [&](int t) {
                const bool open = !mask || (__ldg(mask + (t >> 5)) >> (t & 31) & 1u);
                if (!open) out[t] = from_float<T>(-INFINITY);
                else if (!in_place) out[t] = in[t];
            };
            for (int i = tid; i < head; i += kLogitThreads) single(v0 + i);
            for (int i = v0 + head + n_vec * kVec + tid; i < v1; i += kLogitThreads) single(i);
            const uint4* src = reinterpret_cast<const uint4*>(in + v0 + head);
            uint4* dst = reinterpret_cast<uint4*>(out + v0 + head);
#pragma unroll 4
            for (int i = tid; i < n_vec; i += kLogitThreads) {
                uint32_t open = (1u << kVec) - 1u;
                if (mask) {
                    const int t = v0 + head + i * kVec, w = t >> 5, k = t & 31;
                    open = __ldg(mask + w) >> k;
                    if (k + kVec > 32) open |= __ldg(mask + w + 1) << (32 - k);
                    open &= (1u << kVec) - 1u;
                }
                if (open == 0u) { dst[i] = minus_inf_vector<T>(); continue; }
                if (open == (1u << kVec) - 1u) {
                    if (!in_place) dst[i] = __ldcs(src + i);
                    continue;
                }
                uint4 x = src[i];
                T* e = reinterpret_cast<T*>(&x);
#pragma unroll
                for (int j = 0; j < kVec; ++j)
                    if (!(open >> j & 1u)) e[j] = from_float<T>(-INFINITY);
                dst[i] = x;
            }
        } else {
#pragma unroll 4
            for (int t = v0 + tid; t < v1; t += kLogitThreads) {
                const bool open = !mask || (__ldg(mask + (t >> 5)) >> (t & 31) & 1u);
                out[t] = open ? in[t] : from_float<T>(-INFINITY);
            }
        }
    }
    if (counted) {
        cluster_wait_acquire();
        for (long long i = s0 + tid; i < s1; i += kLogitThreads) {
            const int t = p.history[i];
            if (t < 0 || t >= p.vocab) continue;
            if (i < h1) asm volatile("red.shared::cluster.or.b32 [%0], %1;" ::"r"(word_of(t)), "r"(kInPrompt) : "memory");
            else asm volatile("red.shared::cluster.add.u32 [%0], %1;" ::"r"(word_of(t)), "r"(1u) : "memory");
        }
        for (int i = b0 + tid; i < b1; i += kLogitThreads) {
            const int t = p.bias_token[i];
            if (t >= v0 && t < v1) atomicOr(&words[t - v0], kHasBias);
        }
        cluster_arrive_release();
        cluster_wait_acquire();
    } else {
        __syncthreads();
    }
    auto closed = [&](int t) { return mask && !(__ldg(mask + (t >> 5)) >> (t & 31) & 1u); };
    // ---- biases, ascending by token, by the owner of the slice; of equal tokens the first entry adds up all
    for (int i = b0 + tid; i < b1; i += kLogitThreads) {
        const int t = p.bias_token[i];
        const int prior = i > b0 ? p.bias_token[i - 1] : INT32_MIN;
        if (prior > t && rank == 0 && p.status) atomicOr(p.status, 1 << KAP_ERR_DEVICE_INDEX);
        if (prior == t || t < v0 || t >= v1 || closed(t)) continue;
        float add = p.bias_value[i];
        for (int j = i + 1; j < b1 && p.bias_token[j] == t; ++j) add += p.bias_value[j];
        float x = to_float(in[t]);
        if (counted) x = penalised(x, words[t - v0], r);
        out[t] = from_float<T>(x + add);
    }
    if (counted) {
        for (long long i = s0 + tid; i < s1; i += kLogitThreads) {
            const int t = p.history[i];
            if (t < 0 || t >= p.vocab) continue;
            const uint32_t at = word_of(t);
            uint32_t word;
            asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(word) : "r"(at) : "memory");
            if (word == 0u || (word & kHasBias)) continue;
            asm volatile("atom.shared::cluster.exch.b32 %0, [%1], %2;" : "=r"(word) : "r"(at), "r"(0u) : "memory");
            if (word == 0u || closed(t)) continue;
            out[t] = from_float<T>(penalised(to_float(in[t]), word, r));
        }
        cluster_arrive_release();                             // nobody leaves while a peer may still read its words
        cluster_wait_acquire();
    }
}

template <typename T>
kap_status launch_logits(const LogitParams& p, int cluster, size_t smem, cudaStream_t stream) {
    auto* kernel = kap_adjust_logits_kernel<T>;
    cudaError_t e = cudaSuccess;
    if (smem > 48 * 1024) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e == cudaSuccess && cluster > 8) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return fail(KAP_ERR_CUDA, "cudaFuncSetAttribute failed: %s", cudaGetErrorString(e));
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)cluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)cluster, (unsigned)p.rows);
    cfg.blockDim = dim3(kLogitThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, kernel, p);
    if (e != cudaSuccess) return fail(KAP_ERR_CUDA, "kap_adjust_logits launch failed: %s", cudaGetErrorString(e));
    count_launch();
    return KAP_OK;
}

}  // namespace
}  // namespace kap

using namespace kap;

extern "C" kap_status kap_adjust_logits(
    const void* logits, int32_t logits_type, int64_t row_stride, int32_t rows, int32_t vocab, void* out, int64_t out_stride,
    const int32_t* history, int64_t history_len, const int64_t* history_at, const float* repetition, const float* presence,
    const float* frequency, const int32_t* bias_indptr, const int32_t* bias_token, const float* bias_value, int64_t bias_len,
    const uint32_t* allowed, int32_t num_masks, int64_t allowed_stride, const int32_t* allowed_row, int32_t* device_status, void* cuda_stream)
{
    if (logits_type != KAP_LOGITS_F32 && logits_type != KAP_LOGITS_BF16)
        return fail(KAP_ERR_UNSUPPORTED, "logits_type %d (KAP_LOGITS_F32 = 0, KAP_LOGITS_BF16 = 1)", logits_type);
    if (rows < 0 || vocab < 1 || row_stride < vocab || out_stride < vocab)
        return fail(KAP_ERR_INVALID_ARG, "%d rows of %d logits, row strides %lld and %lld", rows, vocab, (long long)row_stride, (long long)out_stride);
    constexpr int32_t kMostVocab = 811008;
    if (vocab > kMostVocab || rows > 65535) return fail(KAP_ERR_UNSUPPORTED, "%d rows of %d logits (at most 65535 of %d)", rows, vocab, kMostVocab);
    if (rows == 0) return KAP_OK;
    if (!logits || !out) return fail(KAP_ERR_INVALID_ARG, "NULL logits or out");
    if (logits == out && row_stride != out_stride) return fail(KAP_ERR_INVALID_ARG, "in place, but with two row strides");
    if (history_len < 0 || (history && !history_at)) return fail(KAP_ERR_INVALID_ARG, "history needs history_at and a length");
    if (!history && (repetition || presence || frequency)) return fail(KAP_ERR_INVALID_ARG, "penalties need the history");
    if ((bias_token != nullptr) != (bias_indptr != nullptr) || (bias_token != nullptr) != (bias_value != nullptr))
        return fail(KAP_ERR_INVALID_ARG, "biases need bias_indptr, bias_token and bias_value");
    if (bias_len < 0) return fail(KAP_ERR_INVALID_ARG, "bias_len %lld", (long long)bias_len);
    if (allowed ? num_masks < 1 || allowed_stride < (vocab + 31) / 32 : allowed_row != nullptr)
        return fail(KAP_ERR_INVALID_ARG, "%d masks of %lld words for %d logits", num_masks, (long long)allowed_stride, vocab);
    if (allowed && !allowed_row && num_masks < rows) return fail(KAP_ERR_INVALID_ARG, "%d masks for %d rows: allowed_row is needed", num_masks, rows);
    const uintptr_t size_bits = logits_type == KAP_LOGITS_F32 ? 3 : 1;
    if ((reinterpret_cast<uintptr_t>(logits) | reinterpret_cast<uintptr_t>(out)) & size_bits)
        return fail(KAP_ERR_INVALID_ARG, "logits or out are not aligned to their type");
    for (const void* a : {(const void*)history, (const void*)repetition, (const void*)presence, (const void*)frequency, (const void*)bias_indptr,
                          (const void*)bias_token, (const void*)bias_value, (const void*)allowed, (const void*)allowed_row, (const void*)device_status})
        if (reinterpret_cast<uintptr_t>(a) & 3) return fail(KAP_ERR_INVALID_ARG, "an array of 32-bit values is not 4-byte aligned");
    if (reinterpret_cast<uintptr_t>(history_at) & 7) return fail(KAP_ERR_INVALID_ARG, "history_at is not 8-byte aligned");
    LogitParams p{};
    p.logits = logits; p.out = out; p.history = history; p.history_at = reinterpret_cast<const long long*>(history_at);
    p.repetition = repetition; p.presence = presence; p.frequency = frequency;
    p.bias_indptr = bias_indptr; p.bias_token = bias_token; p.bias_value = bias_value;
    p.allowed = allowed; p.allowed_row = allowed_row; p.status = device_status;
    p.row_stride = row_stride; p.out_stride = out_stride; p.history_len = history_len; p.bias_len = bias_len; p.allowed_stride = allowed_stride;
    p.rows = rows; p.vocab = vocab; p.num_masks = num_masks;
    const bool needs_words = history && (repetition || presence || frequency);
    if (!needs_words) p.history = nullptr;
    int cluster = 8;
    while (cluster < 16 && (int64_t)(vocab + cluster - 1) / cluster * 4 > 200 * 1024) cluster *= 2;
    p.slice = ((vocab + cluster - 1) / cluster + 31) / 32 * 32;
    const size_t smem = needs_words ? (size_t)p.slice * 4 : 0;
    return logits_type == KAP_LOGITS_F32 ? launch_logits<float>(p, cluster, smem, (cudaStream_t)cuda_stream)
                                         : launch_logits<__nv_bfloat16>(p, cluster, smem, (cudaStream_t)cuda_stream);
}
