// kap_shared_prefix_attn: full-context attention (kap_verify_attn's result) for a batch whose sequences come in
// groups that share the first pages of their block tables.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "kap_internal.h"

namespace kap {
void count_launch();

namespace {

struct PrefixParams {
    const __nv_bfloat16 *q, *pool;
    const int32_t *q_indptr, *bt_indptr, *bt_pages, *ctx_len;
    __nv_bfloat16* out;
    float* lse;
    int32_t* status;
    long long num_pool_pages;
    int32_t batch, hq, hkv, nhd;
    float scale_log2;
};

// one warp per (query row, head): each lane holds four of the 128 columns
__global__ void __launch_bounds__(128)
kap_prefix_rows_kernel(const PrefixParams p)
{
    const int lane = threadIdx.x & 31;
    const int row = blockIdx.x, head = blockIdx.y * 4 + (threadIdx.x >> 5);
    if (head >= p.hq || row < p.q_indptr[0] || row >= p.q_indptr[p.batch]) return;
    int lo = 0, hi = p.batch;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (p.q_indptr[mid] <= row) lo = mid; else hi = mid;
    }
    const int b = lo, n_q = p.q_indptr[b + 1] - p.q_indptr[b];
    const int seen = p.ctx_len[b] - n_q + (row - p.q_indptr[b]) + 1;     // visible tokens
    const int g = head / (p.hq / p.hkv);
    auto four = [](const __nv_bfloat16* at, float (&v)[4]) {
        const uint2 u = *reinterpret_cast<const uint2*>(at);
        v[0] = __uint_as_float(u.x << 16); v[1] = __uint_as_float(u.x & 0xffff0000u);
        v[2] = __uint_as_float(u.y << 16); v[3] = __uint_as_float(u.y & 0xffff0000u);
    };
    float q[4], o[4] = {0.f, 0.f, 0.f, 0.f}, m = -INFINITY, l = 0.f;
    const long long q_at = ((long long)row * p.hq + head) * kHeadDim + lane * 4;
    four(p.q + q_at, q);
    for (int t = 0; t < seen; ++t) {
        const int i = p.bt_indptr[b] + t / kPageSize;
        const int32_t page = i < p.bt_indptr[b + 1] ? p.bt_pages[i] : -1;
        if (page < 0 || page >= p.num_pool_pages) {
            if (lane == 0) atomicOr(p.status, 1 << KAP_ERR_DEVICE_INDEX);
            continue;
        }
        const long long step = p.nhd ? (long long)p.hkv * kHeadDim : kHeadDim;       // between tokens
        const __nv_bfloat16* k_at = p.pool + (long long)page * 2 * p.hkv * kPageSize * kHeadDim +
                                    (p.nhd ? (long long)g * kHeadDim : (long long)g * kPageSize * kHeadDim) + t % kPageSize * step + lane * 4;
        float k[4], v[4];
        four(k_at, k);
        four(k_at + (long long)p.hkv * kPageSize * kHeadDim, v);
        float s = q[0] * k[0] + q[1] * k[1] + q[2] * k[2] + q[3] * k[3];
        for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
        s *= p.scale_log2;
        const float m_new = fmaxf(m, s), a = exp2f(m - m_new), w = exp2f(s - m_new);
        l = l * a + w;
        for (int j = 0; j < 4; ++j) o[j] = o[j] * a + w * v[j];
        m = m_new;
    }
    const float inv = l > 0.f ? 1.f / l : 0.f;
    for (int j = 0; j < 4; ++j) p.out[q_at + j] = __float2bfloat16(o[j] * inv);
    if (p.lse && lane == 0) p.lse[(long long)row * p.hq + head] = l > 0.f ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
}

}  // namespace
}  // namespace kap

using namespace kap;

static kap_status check_groups(int32_t batch, const int32_t* list_len, const int32_t* n_q, int32_t n_groups,
                               const int32_t* group_indptr, const int32_t* prefix_pages, int32_t hq, int32_t hkv)
{
    if (batch < 0 || n_groups < 0 || (batch > 0 && (!list_len || !n_q || !group_indptr || !prefix_pages)))
        return fail(KAP_ERR_INVALID_ARG, "NULL pointer, batch %d or n_groups %d", batch, n_groups);
    if (hq <= 0 || hkv <= 0 || hq % hkv) return fail(KAP_ERR_INVALID_ARG, "head counts %d / %d", hq, hkv);
    const int32_t G = hq / hkv;
    if (kRowTile % G) return fail(KAP_ERR_UNSUPPORTED, "group size %d must divide %d", G, kRowTile);
    if (batch > 0 && (n_groups < 1 || group_indptr[0] != 0 || group_indptr[n_groups] != batch))
        return fail(KAP_ERR_INVALID_ARG, "group_indptr must run from 0 to the batch size %d", batch);
    for (int32_t b = 0; b < batch; ++b) {
        if (list_len[b] <= 0 || n_q[b] < 1) return fail(KAP_ERR_INVALID_ARG, "sequence %d: list_len %d, n_q %d", b, list_len[b], n_q[b]);
        if ((int64_t)n_q[b] * G > kRowTile * kMaxRowTiles)
            return fail(KAP_ERR_CAPACITY, "sequence %d: %d query rows x %d heads exceed %d", b, n_q[b], G, kRowTile * kMaxRowTiles);
    }
    for (int32_t i = 0; i < n_groups; ++i) {
        if (group_indptr[i + 1] <= group_indptr[i] || group_indptr[i + 1] > batch)
            return fail(KAP_ERR_INVALID_ARG, "group %d is empty or group_indptr is not ascending", i);
        for (int32_t b = group_indptr[i]; b < group_indptr[i + 1]; ++b)
            if (prefix_pages[i] < 0 || prefix_pages[i] > list_len[b])
                return fail(KAP_ERR_INVALID_ARG, "group %d shares %d pages, sequence %d has %d", i, prefix_pages[i], b, list_len[b]);
    }
    return KAP_OK;
}

extern "C" kap_status kap_shared_prefix_items(
    int32_t batch, const int32_t* list_len, const int32_t* n_q, int32_t n_groups, const int32_t* group_indptr,
    const int32_t* prefix_pages, int32_t num_q_heads, int32_t num_kv_heads, int32_t max_rows_per_item, int32_t cta_slots,
    int32_t* max_items)
{
    if (!max_items || max_rows_per_item <= 0 || cta_slots <= 0) return fail(KAP_ERR_INVALID_ARG, "NULL pointer or sizes below 1");
    kap_status st = check_groups(batch, list_len, n_q, n_groups, group_indptr, prefix_pages, num_q_heads, num_kv_heads);
    if (st != KAP_OK) return st;
    int64_t rows = 0;
    for (int32_t b = 0; b < batch; ++b) rows += (int64_t)n_q[b] * num_q_heads;
    *max_items = (int32_t)(rows / max_rows_per_item + 1);
    return KAP_OK;
}

extern "C" kap_status kap_schedule_shared_prefix(
    kap_workspace* ws, int32_t batch, const int32_t* list_len, const int32_t* n_q, int32_t n_groups,
    const int32_t* group_indptr, const int32_t* prefix_pages, int32_t num_q_heads, int32_t num_kv_heads, void* cuda_stream)
{
    if (!ws) return fail(KAP_ERR_INVALID_ARG, "NULL workspace");
    if (batch > ws->max_batch) return fail(KAP_ERR_CAPACITY, "batch %d > workspace max_batch %d", batch, ws->max_batch);
    kap_status st = check_groups(batch, list_len, n_q, n_groups, group_indptr, prefix_pages, num_q_heads, num_kv_heads);
    if (st != KAP_OK) return st;
    (void)cuda_stream;
    int64_t rows = 0;
    for (int32_t b = 0; b < batch; ++b) rows += n_q[b];
    if (rows * num_q_heads > (int64_t)ws->max_items * ws->max_rows)
        return fail(KAP_ERR_CAPACITY, "%lld states exceed the workspace's %d x %d", (long long)(rows * num_q_heads), ws->max_items, ws->max_rows);
    ws->shared_prefix = 1;                              // the other attention calls refuse this schedule
    if (ws->schedule_key) ws->schedule_key->clear();
    ws->batch = batch; ws->num_q_heads = num_q_heads; ws->num_kv_heads = num_kv_heads; ws->total_rows = rows;
    return KAP_OK;
}

extern "C" kap_status kap_shared_prefix_attn(
    const void* q, const int32_t* q_indptr, const void* kv_pool, int64_t num_pool_pages, const int32_t* bt_indptr,
    const int32_t* bt_pages, const int32_t* ctx_len, int32_t batch, int32_t num_q_heads, int32_t num_kv_heads,
    int32_t head_dim, int32_t page_size, float sm_scale, void* out, float* lse, kap_workspace* ws, void* cuda_stream)
{
    if (!ws) return fail(KAP_ERR_INVALID_ARG, "NULL workspace");
    if (head_dim != kHeadDim || page_size != kPageSize)
        return fail(KAP_ERR_UNSUPPORTED, "head_dim %d / page_size %d (supported: 128 / 16)", head_dim, page_size);
    if (!ws->shared_prefix) return fail(KAP_ERR_INVALID_ARG, "the workspace holds no kap_schedule_shared_prefix schedule");
    if (batch != ws->batch || num_q_heads != ws->num_q_heads || num_kv_heads != ws->num_kv_heads)
        return fail(KAP_ERR_INVALID_ARG, "call shape (batch %d, heads %d/%d) differs from the schedule (batch %d, heads %d/%d)", batch,
                    num_q_heads, num_kv_heads, ws->batch, ws->num_q_heads, ws->num_kv_heads);
    if (!(sm_scale > 0.f) || sm_scale > 1e30f) return fail(KAP_ERR_INVALID_ARG, "sm_scale %g", (double)sm_scale);
    if (batch == 0) return KAP_OK;
    if (!q || !q_indptr || !kv_pool || !bt_indptr || !bt_pages || !ctx_len || !out || num_pool_pages <= 0)
        return fail(KAP_ERR_INVALID_ARG, "NULL pointer or empty pool");
    if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(kv_pool) | reinterpret_cast<uintptr_t>(out)) & 15)
        return fail(KAP_ERR_INVALID_ARG, "q, kv_pool and out must be 16-byte aligned");
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev != ws->device)
        return fail(KAP_ERR_INVALID_ARG, "the workspace belongs to device %d but device %d is current", ws->device, dev);
    PrefixParams p{};
    p.q = (const __nv_bfloat16*)q; p.pool = (const __nv_bfloat16*)kv_pool; p.q_indptr = q_indptr; p.bt_indptr = bt_indptr;
    p.bt_pages = bt_pages; p.ctx_len = ctx_len; p.out = (__nv_bfloat16*)out; p.lse = lse; p.status = ws->d_status;
    p.num_pool_pages = num_pool_pages; p.batch = batch; p.hq = num_q_heads; p.hkv = num_kv_heads;
    p.nhd = ws->kv_layout == KAP_KV_NHD; p.scale_log2 = sm_scale * 1.4426950408889634f;
    kap_prefix_rows_kernel<<<dim3((unsigned)ws->total_rows, (unsigned)((num_q_heads + 3) / 4)), 128, 0, (cudaStream_t)cuda_stream>>>(p);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return fail(KAP_ERR_CUDA, "kap_shared_prefix_attn launch failed: %s", cudaGetErrorString(e));
    count_launch();
    return KAP_OK;
}
