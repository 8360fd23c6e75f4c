// Host side of kap_chunk_attn: attention of chunks of new tokens over the paged cache.  The kernels are in kap_chunk_kernel.cuh.
#include <algorithm>

#include "kap_chunk_kernel.cuh"

namespace kap {
void count_launch();
kap_status workspace_page_map(kap_workspace* ws, const void* pool, int64_t pages, int32_t hkv, const void** map);
kap_status encode_query_map(void* map, const void* q, int64_t rows, int32_t hq, int32_t G, int32_t tile_rows);
bool launch_programmatically();

namespace {

#define KAP_CUDA(call)                                                                         \
    do {                                                                                       \
        cudaError_t e_ = (call);                                                               \
        if (e_ != cudaSuccess)                                                                 \
            return fail(KAP_ERR_CUDA, "%s failed: %s", #call, cudaGetErrorString(e_));         \
    } while (0)

// rows x heads up to which states are joined by rows (see the two merge kernels).  By rows / by units, 32 heads, behind 4K: 16 rows 23.4 / 24.9 us, 50 28.0 / 33.4,
// 128 34.5 / 37.9, 256 43.8 / 43.0, 512 64.2 / 58.6, 1024 102 / 84; 64 to 512 single tokens at 2K and 8K within 1 % of each other.
constexpr int64_t kFewMergeCells = 16384;
// rows of the partial buffer: the CTAs' states, and behind them how the work was divided
int64_t cut_rows(int32_t n_cta) { return ((n_cta + 1) * (int64_t)sizeof(ChunkCut) + sizeof(ChunkInStep) + kHeadDim * 4 - 1) / (kHeadDim * 4); }
int64_t rows_needed(int32_t n_cta) { return (int64_t)kChunkStates * n_cta * kChunkUnitRows + cut_rows(n_cta); }

}  // namespace
}  // namespace kap

using namespace kap;

extern "C" kap_status kap_chunk_attn_items(int32_t max_rows_per_item, int32_t cta_slots, int32_t* max_items)
{
    if (!max_items) return fail(KAP_ERR_INVALID_ARG, "NULL max_items");
    if (max_rows_per_item < 1 || max_rows_per_item > kRowTile * kMaxRowTiles || cta_slots < 1 || cta_slots > 4096)
        return fail(KAP_ERR_INVALID_ARG, "max_rows_per_item %d (1 to 64), cta_slots %d (1 to 4096)", max_rows_per_item, cta_slots);
    *max_items = (int32_t)((rows_needed(cta_slots) + max_rows_per_item - 1) / max_rows_per_item);
    return KAP_OK;
}

extern "C" kap_status kap_chunk_attn(
    const void* q, const int32_t* q_indptr, int32_t total_rows, const void* kv_pool, int64_t num_pool_pages, const int32_t* bt_indptr,
    const int32_t* bt_pages, const int32_t* ctx_len, int32_t batch, int32_t num_q_heads, int32_t num_kv_heads,
    int32_t head_dim, int32_t page_size, float sm_scale, int32_t window, int32_t n_sink, void* out, float* lse, kap_workspace* ws,
    void* cuda_stream)
{
    if (!ws) return fail(KAP_ERR_INVALID_ARG, "NULL workspace");
    if (head_dim != kHeadDim || page_size != kPageSize)
        return fail(KAP_ERR_UNSUPPORTED, "head_dim %d / page_size %d (supported: 128 / 16)", head_dim, page_size);
    if (batch < 0 || total_rows < 0 || num_kv_heads <= 0 || num_q_heads <= 0 || num_q_heads % num_kv_heads)
        return fail(KAP_ERR_INVALID_ARG, "batch %d, rows %d, heads %d/%d", batch, total_rows, num_q_heads, num_kv_heads);
    const int32_t G = num_q_heads / num_kv_heads;
    if (G > 16 || (G & (G - 1))) return fail(KAP_ERR_UNSUPPORTED, "%d query heads per KV head (supported: 1, 2, 4, 8, 16)", G);
    if (num_kv_heads > 32767) return fail(KAP_ERR_UNSUPPORTED, "%d KV heads", num_kv_heads);
    if (batch > ws->max_batch) return fail(KAP_ERR_CAPACITY, "batch %d > workspace max_batch %d", batch, ws->max_batch);
    if (window < 0 || n_sink < 0) return fail(KAP_ERR_INVALID_ARG, "window %d, n_sink %d", window, n_sink);
    if (!(sm_scale > 0.f) || sm_scale > 1e30f) return fail(KAP_ERR_INVALID_ARG, "sm_scale %g", (double)sm_scale);
    const int32_t n_cta = ws->sm_count;
    if (rows_needed(n_cta) > (int64_t)ws->max_items * ws->max_rows)
        return fail(KAP_ERR_CAPACITY, "the call needs a workspace of %lld rows (items x rows of an item), this one has %lld",
                    (long long)rows_needed(n_cta), (long long)ws->max_items * ws->max_rows);
    if (batch == 0 || total_rows == 0) return KAP_OK;
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
    kap_status st = workspace_page_map(ws, kv_pool, num_pool_pages, num_kv_heads, &kv_map);
    if (st == KAP_OK) st = encode_query_map(&q_map, q, total_rows, num_q_heads, G, kChunkTileRows);
    if (st != KAP_OK) return st;
    const bool nhd = ws->kv_layout == KAP_KV_NHD;
    if (!ws->chunk_attrs_set) {                                            // function attributes are per device
        KAP_CUDA(cudaFuncSetAttribute(kap_chunk_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kChunkSmemBytes));
        KAP_CUDA(cudaFuncSetAttribute(kap_chunk_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kChunkSmemBytes));
        ws->chunk_attrs_set = 1;
    }
    ChunkParams p{};
    p.q_indptr = q_indptr; p.bt_indptr = bt_indptr; p.bt_pages = bt_pages; p.ctx_len = ctx_len;
    p.part_o = ws->d_part_o; p.part_ml = ws->d_part_ml;
    p.cuts = reinterpret_cast<ChunkCut*>(ws->d_part_o + (int64_t)kChunkStates * n_cta * kChunkUnitRows * kHeadDim);
    p.in_step = reinterpret_cast<ChunkInStep*>(p.cuts + n_cta + 1);
    p.out = (__nv_bfloat16*)out; p.lse = lse; p.status = ws->d_status;
    p.num_pool_pages = num_pool_pages; p.batch = batch; p.total_rows = total_rows;
    p.hq = num_q_heads; p.hkv = num_kv_heads; p.G = G; p.log2_g = __builtin_ctz((unsigned)G); p.window = window; p.n_sink = window ? n_sink : 0;
    p.wide_out = (reinterpret_cast<uintptr_t>(out) & 31) == 0;
    p.scale_log2 = sm_scale * 1.4426950408889634f;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)n_cta);
    cfg.blockDim = dim3(kChunkThreads);
    cfg.dynamicSmemBytes = kChunkSmemBytes;
    cfg.stream = (cudaStream_t)cuda_stream;
    cfg.attrs = attr;
    cfg.numAttrs = launch_programmatically() ? 1 : 0;
    const CUtensorMap& kv = *reinterpret_cast<const CUtensorMap*>(kv_map);
    if (nhd) KAP_CUDA(cudaLaunchKernelEx(&cfg, kap_chunk_kernel<true>, kv, q_map, p));
    else KAP_CUDA(cudaLaunchKernelEx(&cfg, kap_chunk_kernel<false>, kv, q_map, p));
    count_launch();
    if (n_cta > 1) {
        const int64_t cells = (int64_t)total_rows * num_q_heads, warps = kChunkMergeThreads / 32;
        const bool few = cells <= kFewMergeCells;
        cfg.gridDim = dim3(few ? (unsigned)((cells + warps - 1) / warps) : (unsigned)(n_cta - 1) * (kChunkUnitRows / kChunkMergeRows));
        cfg.blockDim = dim3(kChunkMergeThreads);
        cfg.dynamicSmemBytes = 0;
        KAP_CUDA(cudaLaunchKernelEx(&cfg, few ? kap_chunk_merge_rows_kernel : kap_chunk_merge_kernel, p, n_cta));
        count_launch();
    }
    return KAP_OK;
}
