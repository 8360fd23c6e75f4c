// kap_append_kv_rope: kap_append_kv with the position rotation applied on the way.  The pool holds keys
// encoded at their logical position and the attention calls expect queries encoded at theirs (the
// logical-position preservation of the KAP paper, Section 2.1); this call takes q and k as the projection
// leaves them, rotates both and places k and v into their slots (Section 3.1 / 3.2, as kap_append_kv).
//
// Mathematics: pair i of a head turns by the angle pos[axis(i)] * inv_freq[i]:
//     (a, b) -> (a cos - b sin, b cos + a sin).
// The angle is formed and reduced in 64 bits as a number of turns, the remainder's sine and cosine in 32 bits.  (In 32 bits a product
// of about 131 071 rad is rounded by up to 2^-8 rad, a whole bf16 step of a cosine between 1/2 and 1.  Here the product and the
// turns are off by less than 1e-10 rad, and rounding the remainder, at most half a turn, to fp32 adds up to pi 2^-25, 1e-7 rad.)
// Every value is rounded to bf16 once, when it is stored.
//
// Bound: memory; a token row moves 2 (Hq + 2 Hkv) 256 bytes and its angles are shared by all heads.  2 x 8192 rows of 32 / 8 heads
// take 66 us, 6.1 TB/s (93 % of a plain copy's rate); a batch's single step is a launch, 3.3 us for 4 rows, 3.5 for 64.
// Layout: one CTA per token row, 128 threads; a thread task is two 16-byte pieces of one head that hold
// both partners of eight pairs, so a rotation never crosses threads and q may be rotated in place.  What hides the look-ups is other
// CTAs on the SM: reading a thread's values before them costs registers and was slower (2 x 8192 rows: 72 us with the 10 CTAs that then fit on an SM, 68 with 12, 66 with 16).
//
// kap_append_kv_norm_rope is the same kernel with the heads of q and k normalised first: y = x / sqrt(mean(x^2) + eps) w, then the rotation, all in fp32.
// A head's eight threads are neighbours and exchange their sums of squares (three shuffles).  Bound: 2 x 8192 rows of 32 / 8 heads take 77 us, 5.2 TB/s,
// at 64 % of the issue slots; without norms 66.  Arithmetic on pairs of values (55.7 million warp instructions, 69.9 without), values loaded a task
// ahead, the first ones before the look-ups, 8 CTAs on an SM (the first ones behind the look-ups 79 us, only those ahead 84; 7 CTAs 76, but 83 instead of 79 with
// half of a head rotated; 9 and 10 CTAs without loads ahead 79 and 84).  64 single rows: 4.5 us.
#include "kap_ptx.cuh"

namespace kap {
void count_launch();
void kv_written_in_bulk(void* cuda_stream);

namespace {

constexpr int kRopeThreads = 128;
constexpr int kPieces = kHeadDim / 8;              // 16-byte pieces of a head
constexpr int kTasks = kPieces / 2;                // thread tasks of a head: two pieces each

struct RopeParams {
    const __nv_bfloat16 *q, *k, *v;
    __nv_bfloat16 *q_out, *pool;
    long long q_stride, k_stride, v_stride, q_out_stride;      // elements between token rows
    const int32_t *new_indptr, *bt_indptr, *bt_pages, *ctx_len, *positions, *pos_offset;
    const float* inv_freq;
    int32_t *ctx_out, *status;
    long long positions_stride, num_pool_pages;
    int32_t batch, hq, hkv, half, interleaved, nhd;            // half = rotated pairs of a head
    uint8_t axis[kHeadDim / 2];
};
struct NormParams {                                // of kap_append_kv_norm_rope
    const void *q_weight, *k_weight;               // [128], or [heads][128] with a head stride of 128; NULL: ones
    int32_t q_head_stride, k_head_stride, f32, unit_offset;
    float eps;
};

__device__ __forceinline__ void rotate(uint32_t& a, uint32_t& b, const float2 t0, const float2 t1) {
    // a holds the first partners of two pairs, b the second ones
    const float a0 = __uint_as_float(a << 16), a1 = __uint_as_float(a & 0xffff0000u);
    const float b0 = __uint_as_float(b << 16), b1 = __uint_as_float(b & 0xffff0000u);
    const __nv_bfloat162 x = __floats2bfloat162_rn(a0 * t0.x - b0 * t0.y, a1 * t1.x - b1 * t1.y);
    const __nv_bfloat162 y = __floats2bfloat162_rn(b0 * t0.x + a0 * t0.y, b1 * t1.x + a1 * t1.y);
    a = *reinterpret_cast<const uint32_t*>(&x);
    b = *reinterpret_cast<const uint32_t*>(&y);
}
__device__ __forceinline__ uint32_t rotate_neighbours(uint32_t v, const float2 t) {
    const float a = __uint_as_float(v << 16), b = __uint_as_float(v & 0xffff0000u);
    const __nv_bfloat162 x = __floats2bfloat162_rn(a * t.x - b * t.y, b * t.x + a * t.y);
    return *reinterpret_cast<const uint32_t*>(&x);
}

// Two times eight values in pairs, from the two pieces of a task: the first and the second partners where neighbours rotate (the words'
// lower and upper halves), else the pieces one after the other; and back, rounded.
struct Halves { uint64_t a[4], b[4]; };
template <bool neighbours>
__device__ __forceinline__ Halves widen(const uint4& x, const uint4& y) {
    const uint32_t u[4] = {x.x, x.y, x.z, x.w}, v[4] = {y.x, y.y, y.z, y.w};
    Halves h;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t p = neighbours ? (e < 2 ? u[2 * e] : v[2 * e - 4]) : u[e], q = neighbours ? (e < 2 ? u[2 * e + 1] : v[2 * e - 3]) : v[e];
        h.a[e] = neighbours ? pack_f32x2(bf16_lo(p), bf16_lo(q)) : pack_f32x2(bf16_lo(p), bf16_hi(p));
        h.b[e] = neighbours ? pack_f32x2(bf16_hi(p), bf16_hi(q)) : pack_f32x2(bf16_lo(q), bf16_hi(q));
    }
    return h;
}
template <bool neighbours>
__device__ __forceinline__ void narrow(const Halves& h, uint4& x, uint4& y) {
    uint32_t u[4], v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float a0, a1, b0, b1;
        unpack_f32x2(h.a[e], a0, a1);
        unpack_f32x2(h.b[e], b0, b1);
        u[e] = neighbours ? pack_bf16(a0, b0) : pack_bf16(a0, a1);
        v[e] = neighbours ? pack_bf16(a1, b1) : pack_bf16(b0, b1);
    }
    x = neighbours ? make_uint4(u[0], v[0], u[1], v[1]) : make_uint4(u[0], u[1], u[2], u[3]);
    y = neighbours ? make_uint4(u[2], v[2], u[3], v[3]) : make_uint4(v[0], v[1], v[2], v[3]);
}
// The weights of a task's columns, arranged like its values.
template <bool neighbours>
__device__ __forceinline__ Halves load_weights(const NormParams& n, const void* of, int first, int second) {
    Halves h;
    if (!of) {
#pragma unroll
        for (int e = 0; e < 4; ++e) h.a[e] = h.b[e] = pack_f32x2(1.f, 1.f);
        return h;
    }
    if (n.f32) {
        const float4 *f = reinterpret_cast<const float4*>((const float*)of + first), *g = reinterpret_cast<const float4*>((const float*)of + second);
        const float4 q[4] = {__ldg(f), __ldg(f + 1), __ldg(g), __ldg(g + 1)};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float4 u = neighbours ? q[e] : q[e >> 1], v = neighbours ? q[e] : q[2 + (e >> 1)];
            h.a[e] = neighbours ? pack_f32x2(u.x, u.z) : e & 1 ? pack_f32x2(u.z, u.w) : pack_f32x2(u.x, u.y);
            h.b[e] = neighbours ? pack_f32x2(v.y, v.w) : e & 1 ? pack_f32x2(v.z, v.w) : pack_f32x2(v.x, v.y);
        }
    } else {
        h = widen<neighbours>(__ldg(reinterpret_cast<const uint4*>((const __nv_bfloat16*)of + first)), __ldg(reinterpret_cast<const uint4*>((const __nv_bfloat16*)of + second)));
    }
    if (n.unit_offset) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            h.a[e] = add_f32x2(h.a[e], pack_f32x2(1.f, 1.f));
            h.b[e] = add_f32x2(h.b[e], pack_f32x2(1.f, 1.f));
        }
    }
    return h;
}
__device__ __forceinline__ void load_pairs(const float* at, uint64_t (&v)[4]) {          // eight values, 16-byte aligned
    const ulonglong2 p = *reinterpret_cast<const ulonglong2*>(at), q = *(reinterpret_cast<const ulonglong2*>(at) + 1);
    v[0] = p.x; v[1] = p.y; v[2] = q.x; v[3] = q.y;
}

template <bool kNorm, bool kNeighbours>                        // the second: of calls with norms, where neighbouring columns rotate
__global__ void __launch_bounds__(kRopeThreads, kNorm ? 8 : 16)
kap_append_kv_rope_kernel(const RopeParams p, const NormParams n)
{
    __shared__ float2 turn[kNorm ? 1 : kHeadDim / 2];           // (cos, sin) of this row's pairs
    // with norms: cos, sin and -sin apart, for arithmetic on pairs
    __shared__ alignas(16) float cosine[kNorm ? kHeadDim / 2 : 1], sine[kNorm ? kHeadDim / 2 : 1], minus_sine[kNorm ? kHeadDim / 2 : 1];
    const int row = blockIdx.x, tid = threadIdx.x;
    // the sequence that owns the row, the last one that begins at or before it: 32 probes at a time (a bisection waits for one
    // probe after the other; 2928 rows of 24 sequences 17.6 us with it, 17.1 so)
    int b = row, place = 0;
    if (p.new_indptr) {
        const int first = p.new_indptr[0], end = p.new_indptr[p.batch];
        int lo = 0, hi = p.batch;                   // new_indptr[lo] <= row < new_indptr[hi], if the row has an owner
        while (hi - lo > 1) {
            const int step = (hi - lo + 31) / 32, probe = lo + (tid & 31) * step;
            const uint32_t below = __ballot_sync(0xffffffffu, probe < hi && p.new_indptr[probe] <= row);
            lo += max(__popc(below) - 1, 0) * step;
            hi = min(hi, lo + step);
        }
        if (row < first || row >= end) return;      // nobody's row: left as it is
        b = lo;
        place = row - p.new_indptr[lo];
    }
    const int q_tasks = p.q ? p.hq * kTasks : 0, k_tasks = p.hkv * kTasks, n_tasks = q_tasks + 2 * k_tasks;
    const int rotated = p.half / 8;                 // tasks of a head that rotate
    struct Task { bool is_q, is_v, apart; int head, t, c0, c1; };      // c0, c1: the two pieces, partners half a rotation apart, or neighbours
    auto task = [&](int i) {
        Task k;
        k.is_q = i < q_tasks; k.is_v = i >= q_tasks + k_tasks;
        const int j = k.is_q ? i : k.is_v ? i - q_tasks - k_tasks : i - q_tasks;
        k.head = j / kTasks; k.t = j % kTasks;
        k.apart = !(kNorm ? kNeighbours : p.interleaved) && k.t < rotated && !k.is_v;
        k.c0 = k.apart ? k.t : 2 * k.t; k.c1 = k.apart ? k.t + rotated : 2 * k.t + 1;
        return k;
    };
    auto fetch = [&](int i, uint4& x, uint4& y) {
        const Task k = task(i);
        const __nv_bfloat16* src = k.is_q ? p.q + row * p.q_stride : k.is_v ? p.v + row * p.v_stride : p.k + row * p.k_stride;
        const uint4* s4 = reinterpret_cast<const uint4*>(src + k.head * kHeadDim);
        x = s4[k.c0]; y = s4[k.c1];
    };
    // With norms a thread's values are loaded a task ahead, the first ones before the look-ups.
    uint4 next_x = make_uint4(0u, 0u, 0u, 0u), next_y = next_x;
    if (kNorm && tid < n_tasks) fetch(tid, next_x, next_y);
    const int L = p.ctx_len[b];
    const long long at = (long long)L + place;      // logical index of the token
    const int list0 = p.bt_indptr[b], n_bt = p.bt_indptr[b + 1] - list0;
    int32_t page = -1;
    if (L >= 0 && place >= 0 && at / kPageSize < n_bt) page =            // (place < 0: offsets that fall)
        p.bt_pages[list0 + at / kPageSize];
    const bool stored = page >= 0 && page < p.num_pool_pages;
    if (!stored && tid == 0 && p.status) atomicOr(p.status, 1 << KAP_ERR_DEVICE_INDEX);
    if (tid < p.half) {
        const double pos = p.positions ? (double)p.positions[p.axis[tid] * p.positions_stride + row]
                                       : (double)at + (p.pos_offset ? (double)p.pos_offset[b] : 0.0);
        double t = pos * (double)p.inv_freq[tid] * 0.15915494309189533577;    // 1 / (2 pi): turns
        t -= rint(t);
        float s, c;
        sincospif((float)(2.0 * t), &s, &c);
        if (kNorm) { cosine[tid] = c; sine[tid] = s; minus_sine[tid] = -s; }
        else turn[tid] = make_float2(c, s);
    }
    __syncthreads();
    if (p.ctx_out && tid == 0) p.ctx_out[b] = L + 1;   // one row a sequence: no other CTA reads ctx_len[b]

    for (int i = tid; i < n_tasks; i += kRopeThreads) {
        const Task k = task(i);
        const bool is_q = k.is_q, is_v = k.is_v, apart = k.apart;
        const int head = k.head, t = k.t, c0 = k.c0, c1 = k.c1;
        uint4 x = next_x, y = next_y;
        if (kNorm && i + kRopeThreads < n_tasks) fetch(i + kRopeThreads, next_x, next_y);
        if (!is_q && !stored) continue;
        if (!kNorm) fetch(i, x, y);
        if (kNorm && !is_v) {
            // a head's eight threads are neighbours: its sum of squares takes three exchanges
            Halves h = widen<kNeighbours>(x, y);
            uint64_t sum2 = mul_f32x2(h.a[0], h.a[0]);
            sum2 = fma_f32x2(h.b[0], h.b[0], sum2);
#pragma unroll
            for (int e = 1; e < 4; ++e) sum2 = fma_f32x2(h.b[e], h.b[e], fma_f32x2(h.a[e], h.a[e], sum2));
            float lo, hi;
            unpack_f32x2(sum2, lo, hi);
            float sum = lo + hi;
            const uint32_t group = 0xffu << (tid & 24);
#pragma unroll
            for (int d = 1; d < kTasks; d *= 2) sum += __shfl_xor_sync(group, sum, d);
            const float r = rsqrtf(sum * (1.f / kHeadDim) + n.eps);
            const uint64_t r2 = pack_f32x2(r, r);
            const int at = head * (is_q ? n.q_head_stride : n.k_head_stride);
            const Halves w = load_weights<kNeighbours>(n, is_q ? n.q_weight : n.k_weight, at + c0 * 8, at + c1 * 8);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                h.a[e] = mul_f32x2(h.a[e], mul_f32x2(r2, w.a[e]));
                h.b[e] = mul_f32x2(h.b[e], mul_f32x2(r2, w.b[e]));
            }
            if (t < rotated) {
                uint64_t c[4], v[4], m[4];
                load_pairs(&cosine[t * 8], c);
                load_pairs(&sine[t * 8], v);
                load_pairs(&minus_sine[t * 8], m);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint64_t a = h.a[e], b = h.b[e];
                    h.a[e] = fma_f32x2(a, c[e], mul_f32x2(b, m[e]));
                    h.b[e] = fma_f32x2(b, c[e], mul_f32x2(a, v[e]));
                }
            }
            narrow<kNeighbours>(h, x, y);
        } else if (apart) {
            const float2* f = turn + t * 8;
            rotate(x.x, y.x, f[0], f[1]); rotate(x.y, y.y, f[2], f[3]);
            rotate(x.z, y.z, f[4], f[5]); rotate(x.w, y.w, f[6], f[7]);
        } else if (!is_v && t < rotated) {
            const float2* f = turn + t * 8;
            x.x = rotate_neighbours(x.x, f[0]); x.y = rotate_neighbours(x.y, f[1]);
            x.z = rotate_neighbours(x.z, f[2]); x.w = rotate_neighbours(x.w, f[3]);
            y.x = rotate_neighbours(y.x, f[4]); y.y = rotate_neighbours(y.y, f[5]);
            y.z = rotate_neighbours(y.z, f[6]); y.w = rotate_neighbours(y.w, f[7]);
        }
        __nv_bfloat16* dst;
        if (is_q) {
            dst = p.q_out + row * p.q_out_stride + head * kHeadDim;
        } else {
            const int slot = (int)(at % kPageSize), kv = is_v ? 1 : 0;
            const long long r = p.nhd ? ((long long)kv * kPageSize + slot) * p.hkv + head
                                      : ((long long)kv * p.hkv + head) * kPageSize + slot;
            dst = p.pool + ((long long)page * 2 * p.hkv * kPageSize + r) * kHeadDim;
        }
        reinterpret_cast<uint4*>(dst)[c0] = x;
        reinterpret_cast<uint4*>(dst)[c1] = y;
    }
}

__global__ void kap_advance_ctx_kernel(const int32_t* __restrict__ new_indptr, int32_t* ctx_len, int batch) {
    const int b = blockIdx.x * blockDim.x + threadIdx.x;
    if (b < batch) ctx_len[b] += new_indptr[b + 1] - new_indptr[b];
}

}  // namespace
}  // namespace kap

namespace kap {
namespace {

kap_status append_rope(
    const NormParams* norm, const void* q, int64_t q_stride, const void* k_new, int64_t k_stride, const void* v_new, int64_t v_stride,
    void* q_out, int64_t q_out_stride, const int32_t* new_indptr, int32_t total_rows, const float* inv_freq,
    int32_t rotary_dim, int32_t interleaved, const int32_t* positions, int64_t positions_stride, int32_t num_axes,
    const uint8_t* freq_axis, const int32_t* position_offset, void* kv_pool, int64_t num_pool_pages,
    const int32_t* bt_indptr, const int32_t* bt_pages, int32_t* ctx_len, int32_t advance, int32_t batch,
    int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim, int32_t page_size, int32_t kv_layout,
    int32_t* device_status, void* cuda_stream)
{
    if (head_dim != kHeadDim || page_size != kPageSize)
        return fail(KAP_ERR_UNSUPPORTED, "head_dim %d / page_size %d (supported: 128 / 16)", head_dim, page_size);
    if (rotary_dim < 16 || rotary_dim > kHeadDim || rotary_dim % 16)
        return fail(KAP_ERR_UNSUPPORTED, "rotary_dim %d (supported: multiples of 16 from 16 to 128)", rotary_dim);
    if (batch < 0 || total_rows < 0 || num_kv_heads <= 0 || num_q_heads < 0 || (q && num_q_heads == 0))
        return fail(KAP_ERR_INVALID_ARG, "batch %d / rows %d / heads %d / %d", batch, total_rows, num_q_heads, num_kv_heads);
    if (kv_layout != KAP_KV_HND && kv_layout != KAP_KV_NHD)
        return fail(KAP_ERR_INVALID_ARG, "kv_layout %d (KAP_KV_HND = 0, KAP_KV_NHD = 1)", kv_layout);
    if (!new_indptr && total_rows != batch)
        return fail(KAP_ERR_INVALID_ARG, "%d rows for %d sequences: new_indptr is needed", total_rows, batch);
    if (positions ? num_axes < 1 || num_axes > kHeadDim / 2 || (num_axes > 1 && (!freq_axis || positions_stride < total_rows))
                  : num_axes > 1 || freq_axis)
        return fail(KAP_ERR_INVALID_ARG, "%d position axes: several need positions[num_axes][rows] and freq_axis", num_axes);
    if (positions && position_offset) return fail(KAP_ERR_INVALID_ARG, "position_offset goes with the default positions only");
    if (freq_axis)
        for (int i = 0; i < rotary_dim / 2; ++i)
            if (freq_axis[i] >= num_axes)
                return fail(KAP_ERR_INVALID_ARG, "freq_axis[%d] = %d with %d axes", i, freq_axis[i], num_axes);
    if (batch == 0 || total_rows == 0) return KAP_OK;
    if (!k_new || !v_new || !kv_pool || !bt_indptr || !bt_pages || !ctx_len || !inv_freq || num_pool_pages <= 0 || (q && !q_out))
        return fail(KAP_ERR_INVALID_ARG, "NULL pointer or empty pool");
    const int64_t kv_row = (int64_t)num_kv_heads * kHeadDim, q_row = (int64_t)num_q_heads * kHeadDim;
    if (k_stride < kv_row || v_stride < kv_row || (q && (q_stride < q_row || q_out_stride < q_row)))
        return fail(KAP_ERR_INVALID_ARG, "a row stride is smaller than its row");
    uintptr_t bits = reinterpret_cast<uintptr_t>(k_new) | reinterpret_cast<uintptr_t>(v_new) | reinterpret_cast<uintptr_t>(kv_pool) |
                     (uintptr_t)(k_stride * 2) | (uintptr_t)(v_stride * 2);
    if (q) bits |= reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(q_out) | (uintptr_t)(q_stride * 2) | (uintptr_t)(q_out_stride * 2);
    if (bits & 15) return fail(KAP_ERR_INVALID_ARG, "q, k_new, v_new, q_out, kv_pool and their row strides must be 16-byte aligned");

    if ((reinterpret_cast<uintptr_t>(new_indptr) | reinterpret_cast<uintptr_t>(inv_freq) | reinterpret_cast<uintptr_t>(positions) |
         reinterpret_cast<uintptr_t>(position_offset) | reinterpret_cast<uintptr_t>(bt_indptr) | reinterpret_cast<uintptr_t>(bt_pages) |
         reinterpret_cast<uintptr_t>(ctx_len) | reinterpret_cast<uintptr_t>(device_status)) & 3)
        return fail(KAP_ERR_INVALID_ARG, "an index or frequency array is not 4-byte aligned");

    RopeParams p{};
    p.q = (const __nv_bfloat16*)q; p.k = (const __nv_bfloat16*)k_new; p.v = (const __nv_bfloat16*)v_new;
    p.q_out = (__nv_bfloat16*)q_out; p.pool = (__nv_bfloat16*)kv_pool;
    p.q_stride = q_stride; p.k_stride = k_stride; p.v_stride = v_stride; p.q_out_stride = q_out_stride;
    p.new_indptr = new_indptr; p.bt_indptr = bt_indptr; p.bt_pages = bt_pages; p.ctx_len = ctx_len;
    p.positions = positions; p.pos_offset = position_offset; p.inv_freq = inv_freq;
    p.ctx_out = advance && !new_indptr ? ctx_len : nullptr; p.status = device_status;
    p.positions_stride = positions_stride; p.num_pool_pages = num_pool_pages;
    p.batch = batch; p.hq = num_q_heads; p.hkv = num_kv_heads; p.half = rotary_dim / 2;
    p.interleaved = interleaved != 0; p.nhd = kv_layout == KAP_KV_NHD;
    if (freq_axis)
        for (int i = 0; i < p.half; ++i) p.axis[i] = freq_axis[i];
    auto* kernel = !norm ? kap_append_kv_rope_kernel<false, false> : interleaved ? kap_append_kv_rope_kernel<true, true> : kap_append_kv_rope_kernel<true, false>;
    kernel<<<(unsigned)total_rows, kRopeThreads, 0, (cudaStream_t)cuda_stream>>>(p, norm ? *norm : NormParams{});
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return fail(KAP_ERR_CUDA, "launch failed: %s", cudaGetErrorString(e));
    count_launch();
    if (new_indptr) {
        if (advance) {                              // several CTAs read a ctx_len[b]: it moves when they are done
            kap_advance_ctx_kernel<<<(unsigned)((batch + 127) / 128), 128, 0, (cudaStream_t)cuda_stream>>>(new_indptr, ctx_len, batch);
            e = cudaGetLastError();
            if (e != cudaSuccess) return fail(KAP_ERR_CUDA, "launch failed: %s", cudaGetErrorString(e));
            count_launch();
        }
        kv_written_in_bulk(cuda_stream);            // see kap_append_kv
    }
    return KAP_OK;
}

}  // namespace
}  // namespace kap

extern "C" kap_status kap_append_kv_rope(
    const void* q, int64_t q_stride, const void* k_new, int64_t k_stride, const void* v_new, int64_t v_stride,
    void* q_out, int64_t q_out_stride, const int32_t* new_indptr, int32_t total_rows, const float* inv_freq,
    int32_t rotary_dim, int32_t interleaved, const int32_t* positions, int64_t positions_stride, int32_t num_axes,
    const uint8_t* freq_axis, const int32_t* position_offset, void* kv_pool, int64_t num_pool_pages,
    const int32_t* bt_indptr, const int32_t* bt_pages, int32_t* ctx_len, int32_t advance, int32_t batch,
    int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim, int32_t page_size, int32_t kv_layout,
    int32_t* device_status, void* cuda_stream)
{
    return kap::append_rope(nullptr, q, q_stride, k_new, k_stride, v_new, v_stride, q_out, q_out_stride, new_indptr, total_rows, inv_freq,
                            rotary_dim, interleaved, positions, positions_stride, num_axes, freq_axis, position_offset, kv_pool,
                            num_pool_pages, bt_indptr, bt_pages, ctx_len, advance, batch, num_q_heads, num_kv_heads, head_dim, page_size,
                            kv_layout, device_status, cuda_stream);
}

extern "C" kap_status kap_append_kv_norm_rope(
    const void* q, int64_t q_stride, const void* k_new, int64_t k_stride, const void* v_new, int64_t v_stride,
    void* q_out, int64_t q_out_stride, const int32_t* new_indptr, int32_t total_rows,
    const void* q_weight, const void* k_weight, int32_t weight_type, int32_t weight_per_head, int32_t unit_offset, float eps,
    const float* inv_freq, int32_t rotary_dim, int32_t interleaved, const int32_t* positions, int64_t positions_stride, int32_t num_axes,
    const uint8_t* freq_axis, const int32_t* position_offset, void* kv_pool, int64_t num_pool_pages,
    const int32_t* bt_indptr, const int32_t* bt_pages, int32_t* ctx_len, int32_t advance, int32_t batch,
    int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim, int32_t page_size, int32_t kv_layout,
    int32_t* device_status, void* cuda_stream)
{
    using namespace kap;
    if (weight_type != KAP_NORM_F32 && weight_type != KAP_NORM_BF16)
        return fail(KAP_ERR_UNSUPPORTED, "weight_type %d (KAP_NORM_F32 = 0, KAP_NORM_BF16 = 1)", weight_type);
    if (!(eps >= 0.f) || eps > 3e38f) return fail(KAP_ERR_INVALID_ARG, "eps %g", (double)eps);
    if ((reinterpret_cast<uintptr_t>(q_weight) | reinterpret_cast<uintptr_t>(k_weight)) & 15)
        return fail(KAP_ERR_INVALID_ARG, "q_weight and k_weight must be 16-byte aligned");
    NormParams n{};
    n.q_weight = q_weight; n.k_weight = k_weight;
    n.q_head_stride = n.k_head_stride = weight_per_head ? kHeadDim : 0;
    n.f32 = weight_type == KAP_NORM_F32; n.unit_offset = unit_offset != 0; n.eps = eps;
    return append_rope(&n, q, q_stride, k_new, k_stride, v_new, v_stride, q_out, q_out_stride, new_indptr, total_rows, inv_freq,
                       rotary_dim, interleaved, positions, positions_stride, num_axes, freq_axis, position_offset, kv_pool,
                       num_pool_pages, bt_indptr, bt_pages, ctx_len, advance, batch, num_q_heads, num_kv_heads, head_dim, page_size,
                       kv_layout, device_status, cuda_stream);
}
