// kap_adjust_logits: penalties for repeated tokens, biases and grammar masks on logits rows, in front of kap_sample_tokens (the paper fixes no
// sampling rule).
//
// Mathematics, for token t of a row with logit x: c = times t occurs in the answer so far, s = t occurs in the prompt or the answer,
//     x1 = s ? (x > 0 ? x / r : x r) : x,   x2 = x1 - f c - p [c > 0],   x3 = x2 + bias_t,   out = allowed_t ? x3 : -inf,
// in fp32, rounded to the logits' type once.
// Layout: a row is cut into slices of the vocabulary, a CTA each.  The CTA keeps a 32-bit word for each of its tokens in shared memory (times in the
// answer; whether in the prompt; whether it has a bias), reads the row's whole history and counts the tokens that are its own, and then passes over its slice
// once, logits, words and mask together; its first logits are loaded before the history is counted.  Tokens with a bias are left to the biases' pass.
// Bound: memory without a history (512 rows of 128256: 80 us, a plain copy's rate).  A history of 2000 to 4000 tokens a row makes it 118 us: 57 of the 82
// million warp instructions are its words' (cleared, counted, found and corrected).  Words in a cluster's shared memory, the history dealt out: 210 us, since
// frequent tokens meet at one address; a list of touched words corrected after the copy: 158, since their logits are then waited for once more.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "kap_internal.h"

namespace kap {
void count_launch();

namespace {

constexpr int kLogitThreads = 512;
constexpr int kMostSlice = 16384, kMostWords = kMostSlice + 8;            // tokens of a CTA's slice, and words for it
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
    if (word & ~kHasBias) x = x > 0.f ? __fdiv_rn(x, r.repetition) : x * r.repetition;
    if (c) x = x - r.frequency * (float)c - r.presence;
    return x;
}

// The values of a row that decide what has to be done, the same in all of its CTAs.
struct LogitRow {
    Rules r;
    long long h0, h1, h2;
    int b0, b1;
    const uint32_t* mask;
    bool counted;
};
__device__ __forceinline__ LogitRow load_row(const LogitParams& p, int row, bool reports) {
    LogitRow v;
    const float rep = p.repetition ? p.repetition[row] : 1.f, pres = p.presence ? p.presence[row] : 0.f, freq = p.frequency ? p.frequency[row] : 0.f;
    v.h0 = v.h1 = v.h2 = 0;
    if (p.history_at) { v.h0 = p.history_at[row * 3ll]; v.h1 = p.history_at[row * 3ll + 1]; v.h2 = p.history_at[row * 3ll + 2]; }
    v.b0 = p.bias_indptr ? p.bias_indptr[row] : 0;
    v.b1 = p.bias_indptr ? p.bias_indptr[row + 1] : 0;
    const int m = !p.allowed ? -1 : p.allowed_row ? p.allowed_row[row] : row;
    bool bad = false;
    v.r.repetition = rep > 0.f ? rep : 1.f;
    v.r.presence = pres == pres ? pres : 0.f;
    v.r.frequency = freq == freq ? freq : 0.f;
    if (v.h0 < 0 || v.h1 < v.h0 || v.h2 < v.h1 || v.h2 > p.history_len || v.h2 - v.h0 > (long long)kCountMask) { bad = true; v.h0 = v.h1 = v.h2 = 0; }
    if (v.r.repetition == 1.f && v.r.presence == 0.f && v.r.frequency == 0.f) v.h0 = v.h1 = v.h2 = 0;      // (checked all the same)
    if (v.b0 < 0 || v.b1 < v.b0 || v.b1 > p.bias_len) { bad = true; v.b0 = v.b1 = 0; }
    v.mask = m >= 0 && m < p.num_masks ? p.allowed + m * p.allowed_stride : nullptr;
    if (m < -1 || m >= p.num_masks) bad = bad || p.allowed;
    if (bad && reports && p.status) atomicOr(p.status, 1 << KAP_ERR_DEVICE_INDEX);
    v.counted = v.h2 > v.h0;
    return v;
}

template <typename T>
__global__ void __launch_bounds__(kLogitThreads, 3)
kap_adjust_logits_kernel(const LogitParams p)
{
    extern __shared__ uint4 word_space[];                     // [slice] words, used when the row has a history
    constexpr int kVec = 16 / sizeof(T), kAhead = 2;
    const int tid = threadIdx.x, rank = blockIdx.x, row = blockIdx.y;
    const T* const in = reinterpret_cast<const T*>(p.logits) + row * p.row_stride;
    T* const out = reinterpret_cast<T*>(p.out) + row * p.out_stride;
    const bool in_place = p.logits == p.out;
    const int v0 = min(rank * p.slice, p.vocab), v1 = min(v0 + p.slice, p.vocab);
    // the slice in 16-byte vectors of logits and results, where both lie alike; head and rest singly
    const uintptr_t from = reinterpret_cast<uintptr_t>(in + v0), to = reinterpret_cast<uintptr_t>(out + v0);
    const bool alike = ((from ^ to) & 15) == 0;
    const int row_head = alike ? (int)((16 - (reinterpret_cast<uintptr_t>(out) & 15)) & 15) / (int)sizeof(T) : 0;      // (slices begin at multiples of 32 tokens)
    const int head = alike ? min(row_head, v1 - v0) : v1 - v0, n_vec = (v1 - v0 - head) / kVec;
    const uint4* const src = reinterpret_cast<const uint4*>(in + v0 + head);
    uint4* const dst = reinterpret_cast<uint4*>(out + v0 + head);
    // the word of token v0 + i is words[i], placed so that a vector's words are aligned
    uint32_t* const words = reinterpret_cast<uint32_t*>(word_space) + (kVec - row_head) % kVec;
    uint4 ahead[kAhead];                                      // (loaded before it is known whether the row has a mask, whose pass reads for itself)
    if (!in_place) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (tid + k * kLogitThreads < n_vec) ahead[k] = __ldcs(src + tid + k * kLogitThreads);
    }
    const LogitRow q = load_row(p, row, tid == 0 && rank == 0);
    const bool counted = q.counted;

    // ---- the words: every CTA of the row reads the whole history and counts the tokens of its slice
    if (counted) {
        for (int i = tid; i < (p.slice + kVec) / 4; i += kLogitThreads) word_space[i] = make_uint4(0u, 0u, 0u, 0u);
        __syncthreads();
        const int n_prompt = (int)(q.h1 - q.h0), n_all = (int)(q.h2 - q.h0);              // (below 2^30)
        const int32_t* const h = p.history + q.h0;
        auto count = [&](int i, int t) {
            const uint32_t at = (uint32_t)(t - v0);
            if (at >= (uint32_t)(v1 - v0)) return;
            if (i < n_prompt) atomicOr(&words[at], kInPrompt);
            else atomicAdd(&words[at], 1u);
        };
        // in fours, from the first 16-byte boundary on
        const int before = min((int)((16 - (reinterpret_cast<uintptr_t>(h) & 15)) & 15) / 4, n_all), n4 = (n_all - before) / 4;
        const int4* const fours = reinterpret_cast<const int4*>(h + before);
        if (tid < before) count(tid, h[tid]);
        if (tid < n_all - before - 4 * n4) count(before + 4 * n4 + tid, h[before + 4 * n4 + tid]);
#pragma unroll 4
        for (int k = tid; k < n4; k += kLogitThreads) {
            const int4 t = __ldg(fours + k);
            const int i = before + 4 * k;
            count(i, t.x); count(i + 1, t.y); count(i + 2, t.z); count(i + 3, t.w);
        }
        for (int i = q.b0 + tid; i < q.b1; i += kLogitThreads) {
            const int t = p.bias_token[i];
            if (t >= v0 && t < v1) atomicOr(&words[t - v0], kHasBias);
        }
        __syncthreads();
    }
    // ---- the slice: logits, words and mask
    auto closed = [&](int t) { return q.mask && !(__ldg(q.mask + (t >> 5)) >> (t & 31) & 1u); };
    if (!in_place || q.mask || counted) {
        auto single = [&](int t) {
            const uint32_t w = counted ? words[t - v0] : 0u;
            if (closed(t)) out[t] = from_float<T>(-INFINITY);
            else if (w & kHasBias) return;
            else if (w) out[t] = from_float<T>(penalised(to_float(in[t]), w, q.r));
            else if (!in_place) out[t] = in[t];
        };
#pragma unroll 4
        for (int i = tid; i < head; i += kLogitThreads) single(v0 + i);
        for (int i = v0 + head + n_vec * kVec + tid; i < v1; i += kLogitThreads) single(i);
        // The words of a vector, as a bit for each that is not 0; what has a bias is left alone.
        auto find = [&](int i, uint32_t (&w)[kVec], uint32_t& left) {
            uint32_t hits = 0u;
            left = 0u;
#pragma unroll
            for (int j = 0; j < kVec; j += 4) {
                const uint4 z = *reinterpret_cast<const uint4*>(words + head + i * kVec + j);
                w[j] = z.x; w[j + 1] = z.y; w[j + 2] = z.z; w[j + 3] = z.w;
            }
#pragma unroll
            for (int j = 0; j < kVec; ++j) hits |= w[j];
            if (hits == 0u) return 0u;
            hits = 0u;
#pragma unroll
            for (int j = 0; j < kVec; ++j) {
                hits |= (w[j] & ~kHasBias ? 1u : 0u) << j;
                left |= (w[j] >> 31) << j;
            }
            return hits & ~left;
        };
        auto correct = [&](uint4& x, const uint32_t (&w)[kVec], uint32_t hits) {
            // most lanes have one, but not the same one: a turn of the loop for each, not a case for each place
            T* e = reinterpret_cast<T*>(&x);
            while (hits) {
                const int at = __ffs(hits) - 1;
                hits &= hits - 1u;
                float v = 0.f;
                uint32_t word = 0u;
#pragma unroll
                for (int j = 0; j < kVec; ++j)
                    if (j == at) { v = to_float(e[j]); word = w[j]; }
                const T y = from_float<T>(penalised(v, word, q.r));
#pragma unroll
                for (int j = 0; j < kVec; ++j)
                    if (j == at) e[j] = y;
            }
        };
        auto store = [&](int i, const uint4& x, uint32_t left) {
            if (left == 0u) { __stcs(dst + i, x); return; }
            const T* e = reinterpret_cast<const T*>(&x);
            const int t = v0 + head + i * kVec;
#pragma unroll
            for (int j = 0; j < kVec; ++j)
                if (!(left >> j & 1u)) out[t + j] = e[j];
        };
        if (!q.mask) {
            auto vector = [&](int i, uint4 x) {
                uint32_t left = 0u;
                if (counted) {
                    uint32_t w[kVec];
                    const uint32_t hits = find(i, w, left);
                    if (in_place) {
                        if (hits == 0u) return;
                        x = src[i];
                    }
                    correct(x, w, hits);
                }
                store(i, x, left);
            };
            if (in_place) {
                for (int i = tid; i < n_vec; i += kLogitThreads) vector(i, make_uint4(0u, 0u, 0u, 0u));
            } else {
#pragma unroll
                for (int k = 0; k < kAhead; ++k)
                    if (tid + k * kLogitThreads < n_vec) vector(tid + k * kLogitThreads, ahead[k]);
                int i = tid + kAhead * kLogitThreads;
                for (; i + (kAhead - 1) * kLogitThreads < n_vec; i += kAhead * kLogitThreads) {
                    uint4 x[kAhead];
#pragma unroll
                    for (int k = 0; k < kAhead; ++k) x[k] = __ldcs(src + i + k * kLogitThreads);
#pragma unroll
                    for (int k = 0; k < kAhead; ++k) vector(i + k * kLogitThreads, x[k]);
                }
                for (; i < n_vec; i += kLogitThreads) vector(i, __ldcs(src + i));
            }
        } else {
            constexpr uint32_t kAllOpen = (1u << kVec) - 1u;
            for (int i = tid; i < n_vec; i += kLogitThreads) {
                const int t = v0 + head + i * kVec, word = t >> 5, k = t & 31;
                uint32_t open = __ldg(q.mask + word) >> k;
                if (k + kVec > 32) open |= __ldg(q.mask + word + 1) << (32 - k);
                open &= kAllOpen;
                if (open == 0u) { __stcs(dst + i, minus_inf_vector<T>()); continue; }       // (needs no logits)
                uint32_t w[kVec], left = 0u, hits = counted ? find(i, w, left) & open : 0u;
                left &= open;
                if (open == kAllOpen && hits == 0u && in_place) continue;
                uint4 x = src[i];
                T* e = reinterpret_cast<T*>(&x);
                correct(x, w, hits);
#pragma unroll
                for (int j = 0; j < kVec; ++j)
                    if (!(open >> j & 1u)) e[j] = from_float<T>(-INFINITY);
                store(i, x, left);
            }
        }
    }
    if (q.b1 > q.b0) {
        // biases, ascending by token, by the owner of the slice; of equal tokens the first entry adds up all
        if (!counted) __syncthreads();                        // their logits have been copied above
        for (int i = q.b0 + tid; i < q.b1; i += kLogitThreads) {
            const int t = p.bias_token[i];
            const int prior = i > q.b0 ? p.bias_token[i - 1] : INT32_MIN;
            if (prior > t && rank == 0 && p.status) atomicOr(p.status, 1 << KAP_ERR_DEVICE_INDEX);
            if (prior == t || t < v0 || t >= v1 || closed(t)) continue;
            float add = p.bias_value[i];
            for (int j = i + 1; j < q.b1 && p.bias_token[j] == t; ++j) add += p.bias_value[j];
            float x = to_float(in[t]);
            if (counted) x = penalised(x, words[t - v0], q.r);
            out[t] = from_float<T>(x + add);
        }
    }
}

template <typename T>
kap_status launch_logits(const LogitParams& p, int slices, size_t smem, cudaStream_t stream) {
    auto* kernel = kap_adjust_logits_kernel<T>;
    cudaError_t e = cudaSuccess;
    // (always to the most that a call may need: another thread's call must not find less than it asked for)
    if (smem > 48 * 1024) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostWords * 4);
    if (e != cudaSuccess) return fail(KAP_ERR_CUDA, "cudaFuncSetAttribute failed: %s", cudaGetErrorString(e));
    kernel<<<dim3((unsigned)slices, (unsigned)p.rows), kLogitThreads, smem, stream>>>(p);
    e = cudaGetLastError();
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
    if (history_len < 0 || (history && !history_at) || (history_at && !history && history_len > 0)) return fail(KAP_ERR_INVALID_ARG, "history needs history_at and a length");
    if (!history_at && (repetition || presence || frequency)) return fail(KAP_ERR_INVALID_ARG, "penalties need the history");
    if (bias_len < 0) return fail(KAP_ERR_INVALID_ARG, "bias_len %lld", (long long)bias_len);
    // (a list without entries needs no address)
    if (bias_indptr ? bias_len > 0 && (!bias_token || !bias_value) : bias_len > 0 || bias_token || bias_value)
        return fail(KAP_ERR_INVALID_ARG, "biases need bias_indptr, bias_token and bias_value");
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
    const bool needs_words = history_at && (repetition || presence || frequency);
    // Slices of at most 16384 tokens (64 KiB of words: three CTAs on an SM), and of fewer where there are rows too few to fill the device: every CTA of a
    // row reads its whole history, so no more than that (512 rows of 128256, histories of 2000 to 4000: 8 slices 118 us, 10 120, 12
    // 123; one row with 20000: 8 slices 14 us, 64 8).
    constexpr int kOneWave = 148 * 3, kMostSlices = 64;       // 148 SMs of a B200; only this choice uses it
    const int least = (vocab + kMostSlice - 1) / kMostSlice;
    int slices = least < kMostSlices ? (kOneWave / rows < least ? least : kOneWave / rows > kMostSlices ? kMostSlices : kOneWave / rows) : least;
    p.slice = ((vocab + slices - 1) / slices + 31) / 32 * 32;
    slices = (vocab + p.slice - 1) / p.slice;
    const size_t smem = needs_words ? ((size_t)p.slice + 8) * 4 : 0;
    return logits_type == KAP_LOGITS_F32 ? launch_logits<float>(p, slices, smem, (cudaStream_t)cuda_stream)
                                         : launch_logits<__nv_bfloat16>(p, slices, smem, (cudaStream_t)cuda_stream);
}
