// Host side of kap_shared_prefix_attn: full-context attention (kap_verify_attn's result, Section 3.2 of the KAP paper) for a
// batch whose sequences come in groups that share the first pages of their block tables.  The work list is built in
// kap_prefix_schedule.cpp, the kernels are in kap_prefix_kernel.cuh.
#include <algorithm>
#include <cstring>
#include <exception>

#include "kap_prefix_kernel.cuh"

namespace kap {
void count_launch();
kap_status workspace_kv_map(kap_workspace* ws, const void* pool, int64_t pages, int32_t hkv, const void** map);
kap_status encode_query_map(void* map, const void* q, int64_t rows, int32_t hq, int32_t G, int32_t tile_rows);
bool launch_programmatically();
kap_status launch_prefix_parts(kap_workspace* ws, const void* kv_map, const void* q, const int32_t* bt_indptr, const int32_t* bt_pages,
                               const int32_t* ctx_len, const WorkItem* items, int32_t n_items, const void* row_map,
                               const int32_t* q_end, int64_t num_pool_pages, int32_t batch, int32_t hq, int32_t hkv, float scale_log2, cudaStream_t stream);

namespace {

#define KAP_CUDA(call)                                                                         \
    do {                                                                                       \
        cudaError_t e_ = (call);                                                               \
        if (e_ != cudaSuccess)                                                                 \
            return fail(KAP_ERR_CUDA, "%s failed: %s", #call, cudaGetErrorString(e_));         \
    } while (0)

kap_status upload_schedule(kap_workspace* ws, const PrefixSchedule& s, int32_t batch, int32_t hq, int32_t hkv, cudaStream_t stream) {
    int dev = -1;
    KAP_CUDA(cudaGetDevice(&dev));
    if (dev != ws->device) KAP_CUDA(cudaSetDevice(ws->device));
    cudaError_t e = cudaEventSynchronize((cudaEvent_t)ws->upload_event);   // the pinned staging may still feed the previous upload
    const PrefixLayout at = prefix_layout(s);
    if (e == cudaSuccess && batch > 0) {
        unsigned char* first = reinterpret_cast<unsigned char*>(ws->h_items);
        unsigned char* third = reinterpret_cast<unsigned char*>(ws->h_merge);
        std::memcpy(first, s.items.data(), at.segments);
        std::memcpy(first + at.segments, s.segments.data(), at.first_bytes - at.segments);
        std::memcpy(ws->h_groups, s.units.data(), at.second_bytes);
        std::memcpy(third, s.seqs.data(), at.rows);
        std::memcpy(third + at.rows, s.rows.data(), at.ctas - at.rows);
        std::memcpy(third + at.ctas, s.cta_begin.data(), s.cta_begin.size() * sizeof(int32_t));
        e = cudaMemcpyAsync(ws->d_items, first, at.first_bytes, cudaMemcpyHostToDevice, stream);
        if (e == cudaSuccess) e = cudaMemcpyAsync(ws->d_groups, ws->h_groups, at.second_bytes, cudaMemcpyHostToDevice, stream);
        if (e == cudaSuccess) e = cudaMemcpyAsync(ws->d_merge, third, at.third_bytes, cudaMemcpyHostToDevice, stream);
    }
    if (e == cudaSuccess) e = cudaEventRecord((cudaEvent_t)ws->upload_event, stream);
    if (dev != ws->device) cudaSetDevice(dev);                             // the caller's current device is put back
    if (e != cudaSuccess) return fail(KAP_ERR_CUDA, "schedule upload failed: %s", cudaGetErrorString(e));
    ws->shared_prefix = 1;                                                 // the other attention calls refuse this schedule
    ws->prefix_ctas = s.n_cta;
    if (ws->schedule_key) ws->schedule_key->clear();
    ws->batch = batch; ws->num_q_heads = hq; ws->num_kv_heads = hkv; ws->total_rows = s.total_rows;
    ws->n_items = (int32_t)s.items.size(); ws->n_groups = (int32_t)s.units.size(); ws->prefix_segments = (int32_t)s.segments.size();
    ws->ring_slots = kPrefixRingSlots;
    ws->max_splits = 1;
    for (const PrefixUnit& u : s.units) ws->max_splits = std::max(ws->max_splits, u.n_states);
    return KAP_OK;
}

}  // namespace
}  // namespace kap

using namespace kap;

extern "C" kap_status kap_schedule_shared_prefix(
    kap_workspace* ws, int32_t batch, const int32_t* list_len, const int32_t* n_q, int32_t n_groups,
    const int32_t* group_indptr, const int32_t* prefix_pages, int32_t num_q_heads, int32_t num_kv_heads, void* cuda_stream)
{
    if (!ws) return fail(KAP_ERR_INVALID_ARG, "NULL workspace");
    if (batch > ws->max_batch) return fail(KAP_ERR_CAPACITY, "batch %d > workspace max_batch %d", batch, ws->max_batch);
    try {
        PrefixSchedule s;
        kap_status st = build_prefix_schedule(batch, list_len, n_q, n_groups, group_indptr, prefix_pages, num_q_heads, num_kv_heads,
                                              ws->sm_count, s);
        if (st != KAP_OK) return st;
        const int64_t need = prefix_items_needed(s, ws->max_rows);
        if (need > ws->max_items)
            return fail(KAP_ERR_CAPACITY, "the schedule needs a workspace of %lld items of %d rows, this one has %d", (long long)need,
                        ws->max_rows, ws->max_items);
        return upload_schedule(ws, s, batch, num_q_heads, num_kv_heads, (cudaStream_t)cuda_stream);
    } catch (const std::exception& e) {                                    // no exception leaves a C entry point
        return fail(KAP_ERR_CAPACITY, "the schedule does not fit the host's memory: %s", e.what());
    }
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
    if ((reinterpret_cast<uintptr_t>(q_indptr) | reinterpret_cast<uintptr_t>(bt_indptr) | reinterpret_cast<uintptr_t>(bt_pages) |
         reinterpret_cast<uintptr_t>(ctx_len) | reinterpret_cast<uintptr_t>(lse)) & 3)
        return fail(KAP_ERR_INVALID_ARG, "an index array or lse is not 4-byte aligned");
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev != ws->device)
        return fail(KAP_ERR_INVALID_ARG, "the workspace belongs to device %d but device %d is current", ws->device, dev);
    const void* kv_map = nullptr;
    alignas(64) CUtensorMap q_map;
    const int32_t G = num_q_heads / num_kv_heads;
    kap_status st = workspace_kv_map(ws, kv_pool, num_pool_pages, num_kv_heads, &kv_map);
    if (st == KAP_OK) st = encode_query_map(&q_map, q, ws->total_rows, num_q_heads, G, kPrefixTileRows);
    if (st != KAP_OK) return st;
    const bool nhd = ws->kv_layout == KAP_KV_NHD;
    if (!ws->prefix_attrs_set) {                                           // function attributes are per device
        KAP_CUDA(cudaFuncSetAttribute(kap_prefix_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kPfxSmemBytes));
        KAP_CUDA(cudaFuncSetAttribute(kap_prefix_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kPfxSmemBytes));
        ws->prefix_attrs_set = 1;
    }
    PfxParams p{};
    const PrefixLayout at((size_t)ws->n_items, (size_t)ws->prefix_segments, (size_t)ws->n_groups, (size_t)batch, (size_t)ws->total_rows, (size_t)ws->prefix_ctas);
    const unsigned char* first = reinterpret_cast<const unsigned char*>(ws->d_items);
    const unsigned char* third = reinterpret_cast<const unsigned char*>(ws->d_merge);
    p.segments = reinterpret_cast<const PrefixSegment*>(first + at.segments);
    p.units = reinterpret_cast<const PrefixUnit*>(ws->d_groups);
    p.seqs = reinterpret_cast<const PrefixSeq*>(third);
    p.row_map = reinterpret_cast<const PrefixRow*>(third + at.rows);
    p.cta_begin = reinterpret_cast<const int32_t*>(third + at.ctas);
    p.q_indptr = q_indptr; p.bt_indptr = bt_indptr; p.bt_pages = bt_pages; p.ctx_len = ctx_len;
    p.part_o = ws->d_part_o; p.part_ml = ws->d_part_ml; p.out = (__nv_bfloat16*)out; p.lse = lse; p.status = ws->d_status;
    p.num_pool_pages = num_pool_pages; p.total_rows = (int32_t)ws->total_rows; p.q_end = q_indptr + batch;
    p.hq = num_q_heads; p.hkv = num_kv_heads; p.G = G;
    p.scale_log2 = sm_scale * 1.4426950408889634f;
    // the sequences' own pages and small prefixes, then the large prefixes, then the join of their states
    if (ws->n_items > 0) {
        st = launch_prefix_parts(ws, kv_map, q, bt_indptr, bt_pages, ctx_len, ws->d_items, ws->n_items, p.row_map, p.q_end, num_pool_pages, batch,
                                 num_q_heads, num_kv_heads, p.scale_log2, (cudaStream_t)cuda_stream);
        if (st != KAP_OK) return st;
    }
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)ws->prefix_ctas);
    cfg.blockDim = dim3(kPfxThreads);
    cfg.dynamicSmemBytes = kPfxSmemBytes;
    cfg.stream = (cudaStream_t)cuda_stream;
    cfg.attrs = attr;
    cfg.numAttrs = launch_programmatically() ? 1 : 0;
    const CUtensorMap& kv = *reinterpret_cast<const CUtensorMap*>(kv_map);
    if (ws->prefix_ctas > 0) {
        if (nhd) KAP_CUDA(cudaLaunchKernelEx(&cfg, kap_prefix_kernel<true>, kv, q_map, p));
        else KAP_CUDA(cudaLaunchKernelEx(&cfg, kap_prefix_kernel<false>, kv, q_map, p));
        count_launch();
    }
    // Few cells: one a warp.  Many: four heads a warp, one metadata chain for all of them.  (64 sequences with 32K shared tokens: 61.7 us
    // for the call, one head a warp 64.7; 16 sequences of two rows with 64K 72.0 against 76.9.  4 sequences with 512 / 8K tokens: one head a
    // warp 8.4 / 16.6, four 9.9 / 21.1.)  More than four states: four warps a set, while the sets are one wave of CTAs (64 sequences with
    // 32K, 20 states: 61.5 against 71.8 with one warp; 4 sequences with 512, eight states 8.4 against 9.2; 256 sequences on two prefixes
    // of 8K, several waves: 81.7 with one warp, 85.4 with four).
    const int64_t cells = ws->total_rows * num_q_heads, one_wave = (int64_t)ws->sm_count * 6;
    const int H = cells <= one_wave ? 1 : G >= 4 ? 4 : G;
    const int64_t sets = cells / H;
    const bool wide = ws->max_splits > 4 && sets <= one_wave;
    cfg.gridDim = dim3((unsigned)(wide ? sets : (sets + 3) / 4));
    cfg.blockDim = dim3(128);
    cfg.dynamicSmemBytes = 0;
    if (H == 4) KAP_CUDA(cudaLaunchKernelEx(&cfg, wide ? kap_prefix_merge_kernel<4, true> : kap_prefix_merge_kernel<4, false>, p));
    else if (H == 2) KAP_CUDA(cudaLaunchKernelEx(&cfg, wide ? kap_prefix_merge_kernel<2, true> : kap_prefix_merge_kernel<2, false>, p));
    else KAP_CUDA(cudaLaunchKernelEx(&cfg, wide ? kap_prefix_merge_kernel<1, true> : kap_prefix_merge_kernel<1, false>, p));
    count_launch();
    return KAP_OK;
}
