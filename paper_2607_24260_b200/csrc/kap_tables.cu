// kap_build_block_tables / kap_release_pages: the step's block tables and slots from the requests' lengths, on the device (the KAP paper's
// block tables and slot mappings, Section 3.1, are taken as given by its host runtime).
//
// Mathematics: with L tokens cached, n new ones and held pages, sequence b lists ceil((L + n) / P) pages and takes those it does not hold from the
// top of a stack of free pages; where a sequence's list, new rows and taken pages begin are three prefix sums over the batch.  A negative entry of the
// page table is a page that its request has given back: a release passes it over, and a new row may not lie on it.
// Layout: one CTA does the sums, the checks and the state (page table, held pages, stack), all or nothing; a second kernel, started while
// the first runs, copies the lists and writes the slots, a CTA for each 2048 entries, whose owners it finds by bisection.
// Bound: latency.  A step and its release are three kernels, each a chain of look-ups: 10.4 us for 64 sequences at 16K, 18.3 us for 512 of up to 128K (the bytes
// alone 0.03 and 1.5 us); of the 18.3, 0.7 look at the pages that first rows lie on.  Each alone (cold): sums 5.7 and 7, lists and slots 9.5 and 13, release 5 and 7.
#include <cuda_runtime.h>

#include "kap_internal.h"

namespace kap {
void count_launch();
bool launch_programmatically();

namespace {

// Of the first kernel, for batches of up to 128 sequences the second number.  (A step and its release with 128 / 1024 threads: 32 single tokens 11.1 / 12.4 us, 128 11.9 /
// 13.5; 32 chunks of 64 13.2 / 15.1, 64 15.0 / 15.8, 128 17.0 / 15.8.)
constexpr int kTableThreads = 1024, kFewThreads = 128;
constexpr int kFillThreads = 256, kFillEntries = 2048;
constexpr long long kMostEntries = INT32_MAX - kFillEntries;  // of a step's block table, and rows: the second kernel counts past them in 32 bits
constexpr int32_t kMaxRequests = 1 << 20;                     // a bit each in the first kernel's shared memory

struct TableParams {
    const int32_t *request, *ctx_len, *n_new;                 // release: ctx_len = tokens to keep
    int32_t *page_table, *pages_held, *free_pages, *free_count, *bt_indptr, *bt_pages, *new_indptr, *position, *status;
    long long* slot;
    long long table_stride, bt_capacity, row_capacity;
    int32_t batch, page_size, num_requests, free_capacity;
};

struct Entry {
    int32_t request, held, pages, moved, n;                   // pages: listed (build) or kept (release); moved: taken, or entries given up
    bool bad, full, on_held;                                  // on_held: the first new row lies on a page held,
    int32_t first_page;                                       // this one
    __device__ __forceinline__ bool on_none() const { return on_held && first_page < 0; }      // it has been given back
};

template <bool kRelease>
__device__ __forceinline__ Entry load_entry(const TableParams& p, int b, uint32_t* seen) {
    Entry e{0, 0, 0, 0, 0, false, false, false, 0};
    if (b >= p.batch) return e;
    e.request = p.request ? p.request[b] : b;
    const int L = p.ctx_len ? p.ctx_len[b] : 0;
    e.n = kRelease ? 0 : p.n_new ? p.n_new[b] : 1;
    if (e.request < 0 || e.request >= p.num_requests || L < 0 || e.n < 0) { e.bad = true; e.n = 0; return e; }
    const int32_t* const row = p.page_table + e.request * p.table_stride;
    // the page of the first new row, which may be held already: loaded beside the number of those, not behind it, and looked at as late as can be
    const int first = L / p.page_size;
    if (!kRelease && seen && e.n > 0 && first < p.table_stride) e.first_page = row[first];
    e.held = p.pages_held[e.request];
    if (seen) e.bad = atomicOr(&seen[e.request >> 5], 1u << (e.request & 31)) >> (e.request & 31) & 1u;   // named twice
    if (e.held < 0 || e.held > p.table_stride) { e.bad = true; e.held = 0; }
    const long long pages = ((long long)L + e.n + p.page_size - 1) / p.page_size;
    if (kRelease) {
        e.pages = (int32_t)min(pages, (long long)e.held);
        e.moved = e.held - e.pages;
    } else {
        if (pages > p.table_stride || L > INT32_MAX - e.n) { e.full = true; return e; }      // (a position has 32 bits)
        e.pages = (int32_t)pages;
        e.moved = max(0, e.pages - e.held);
        if (seen && e.n > 0) {                                // new rows on pages held: not on entries that the caller has given back
            const int end = min(e.held, e.pages);
            e.on_held = first < end;
            // (64 chunks of 512 on pages held 9 us, of 8192 17, one of 131072 111: by whole warps 10, 54, 20)
            for (int i = first + 1; i < end; ++i) e.bad |= row[i] < 0;
        }
    }
    return e;
}

// Inclusive sums over the block, and the block's totals.  (All threads; the shared arrays may be used again after another barrier.)
struct Sums { long long pages, moved, rows; };
__device__ __forceinline__ Sums operator+(const Sums& a, const Sums& b) { return {a.pages + b.pages, a.moved + b.moved, a.rows + b.rows}; }
__device__ __forceinline__ Sums warp_scan(Sums v) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const Sums o{__shfl_up_sync(0xffffffffu, v.pages, d), __shfl_up_sync(0xffffffffu, v.moved, d), __shfl_up_sync(0xffffffffu, v.rows, d)};
        if (lane >= d) v = v + o;
    }
    return v;
}
template <int kWarps>
__device__ __forceinline__ Sums block_scan(Sums v, Sums& all, Sums* warp_sums) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    v = warp_scan(v);
    if (lane == 31) warp_sums[warp] = v;
    __syncthreads();
    const Sums w = warp_scan(lane < kWarps ? warp_sums[lane] : Sums{0, 0, 0});         // by every warp for itself
    const Sums none{0, 0, 0}, before{__shfl_sync(0xffffffffu, w.pages, warp ? warp - 1 : 0), __shfl_sync(0xffffffffu, w.moved, warp ? warp - 1 : 0),
                                     __shfl_sync(0xffffffffu, w.rows, warp ? warp - 1 : 0)};
    all = {__shfl_sync(0xffffffffu, w.pages, 31), __shfl_sync(0xffffffffu, w.moved, 31), __shfl_sync(0xffffffffu, w.rows, 31)};
    return v + (warp ? before : none);
}

// The sequence that owns the i-th entry moved of those of a block's threads: upto[t] counts the entries of the first t + 1.
template <int kThreads>
__device__ __forceinline__ int moved_by(const int32_t* upto, int i) {
    int lo = 0;                                               // sequences whose entries all come before i
#pragma unroll
    for (int d = kThreads / 2; d > 0; d /= 2)
        if (upto[lo + d - 1] <= i) lo += d;
    return lo;
}

template <bool kRelease, int kThreads>
__global__ void __launch_bounds__(kThreads)
kap_tables_kernel(const TableParams p)
{
    extern __shared__ uint32_t seen[];
    __shared__ Sums warp_sums[kThreads / 32];
    __shared__ int32_t upto[kThreads], first[kThreads], request[kThreads];
    const int tid = threadIdx.x;
    for (int i = tid; i < (p.num_requests + 31) / 32; i += kThreads) seen[i] = 0u;
    if (!kRelease) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");    // the second kernel, which waits
    const int count = *p.free_count;
    __syncthreads();
    // ---- what the step needs, and whether that can be had
    Sums total{0, 0, 0}, all{0, 0, 0};
    bool bad = count < 0 || count > p.free_capacity, full = false;
    const Entry e0 = load_entry<kRelease>(p, tid, seen);
    for (int b0 = 0; b0 < p.batch; b0 += kThreads) {
        const Entry e = b0 == 0 ? e0 : load_entry<kRelease>(p, b0 + tid, seen);
        bad |= e.bad || (b0 > 0 && e.on_none());
        full |= e.full;
        total = total + Sums{e.pages, e.moved, e.n};
    }
    const Sums mine0 = block_scan<kThreads / 32>(total, all, warp_sums);     // (sums of the sequences themselves, when each has a thread)
    bad = __syncthreads_or(bad || e0.on_none());
    if (kRelease) full = all.moved > INT32_MAX;               // (entries are counted in 32 bits from here on, and no stack takes so many)
    else full = __syncthreads_or(full) || all.moved > count || all.pages > p.bt_capacity || all.rows > p.row_capacity;
    if (bad || full) {                                        // nothing is taken: a step without pages and rows
        if (!kRelease)
            for (int b = tid; b <= p.batch; b += kThreads) {
                p.bt_indptr[b] = 0;
                if (p.new_indptr) p.new_indptr[b] = 0;
            }
        if (tid == 0 && p.status) atomicOr(p.status, 1 << (bad ? KAP_ERR_DEVICE_INDEX : KAP_ERR_CAPACITY));
        return;
    }
    // The entries moved by the sequences from b0 on, one for each thread, laid out one after the other: upto, first and request, and their number.
    Entry e = e0;
    Sums v = mine0;
    auto lay_out = [&](int b0) {
        Sums here = all;
        e = b0 == 0 ? e0 : load_entry<kRelease>(p, b0 + tid, nullptr);
        v = mine0;
        if (p.batch > kThreads) v = block_scan<kThreads / 32>(Sums{e.pages, e.moved, e.n}, here, warp_sums);
        upto[tid] = (int32_t)v.moved;
        first[tid] = kRelease ? e.pages : e.held;
        request[tid] = e.request;
        __syncthreads();
        return here;
    };
    auto entry_of = [&](int i) {
        const int lo = moved_by<kThreads>(upto, i), before = lo ? upto[lo - 1] : 0;
        return p.page_table + request[lo] * p.table_stride + first[lo] + (i - before);
    };
    Sums carry{0, 0, 0};
    if (kRelease) {
        // The i-th page, in the batch's order, becomes the i-th from the top of the larger stack.  Entries without a page (negative ones) are rare: every
        // entry is placed as if there were none (in front of nothing that is on the stack), and placed again, counted one by one, if there were.
        const long long room = (long long)p.free_capacity - count;
        const bool fits = all.moved <= room, early = fits && p.batch <= kThreads;      // early: the lengths are written beside the pages (512 sequences 0.3 us less)
        bool gone = false;
        for (int b0 = 0; b0 < p.batch; b0 += kThreads) {
            const Sums here = lay_out(b0);
            if (early && e.moved > 0) p.pages_held[e.request] = e.pages;
            for (int i = tid; i < (int)here.moved; i += kThreads) {
                const int32_t page = *entry_of(i);
                gone |= page < 0;
                if (fits) p.free_pages[count + all.moved - 1 - (carry.moved + i)] = page;
            }
            carry = carry + here;
            if (b0 + kThreads < p.batch) __syncthreads();
        }
        gone = __syncthreads_or(gone);
        long long back = all.moved;
        for (int pass = 0; gone && pass < 2; ++pass) {        // counted, then placed
            long long before = 0;
            for (int b0 = 0; b0 < p.batch; b0 += kThreads) {
                const Sums here = lay_out(b0);
                for (int i0 = 0; i0 < (int)here.moved; i0 += kThreads) {
                    const int32_t page = i0 + tid < (int)here.moved ? *entry_of(i0 + tid) : -1;
                    Sums round;
                    const Sums upto_here = block_scan<kThreads / 32>(Sums{page >= 0, 0, 0}, round, warp_sums);
                    if (pass == 1 && page >= 0) p.free_pages[count + back - (before + upto_here.pages)] = page;
                    before += round.pages;
                    __syncthreads();
                }
                __syncthreads();
            }
            back = before;
            if (back > room) break;
        }
        if (back > room) {
            if (tid == 0 && p.status) atomicOr(p.status, 1 << KAP_ERR_CAPACITY);
            return;
        }
        for (int b0 = 0; b0 < p.batch && !early; b0 += kThreads) {
            e = b0 == 0 ? e0 : load_entry<true>(p, b0 + tid, nullptr);
            if (e.moved > 0) p.pages_held[e.request] = e.pages;
        }
        if (tid == 0 && back > 0) *p.free_count = (int32_t)(count + back);
        return;
    }
    // ---- the state and the prefix sums
    if (tid == 0) {
        p.bt_indptr[0] = 0;
        if (p.new_indptr) p.new_indptr[0] = 0;
    }
    for (int b0 = 0; b0 < p.batch; b0 += kThreads) {
        const Sums here = lay_out(b0);
        const int b = b0 + tid;
        if (b < p.batch) {
            p.bt_indptr[b + 1] = (int32_t)(carry.pages + v.pages);
            if (p.new_indptr) p.new_indptr[b + 1] = (int32_t)(carry.rows + v.rows);
            if (e.moved > 0) p.pages_held[e.request] = e.pages;
        }
        // the i-th page taken, in the batch's order, is the i-th from the top
        for (int i = tid; i < (int)here.moved; i += kThreads) *entry_of(i) = p.free_pages[count - 1 - (carry.moved + i)];
        carry = carry + here;
        if (b0 + kThreads < p.batch) __syncthreads();
    }
    if (tid == 0 && all.moved > 0) *p.free_count = (int32_t)(count - all.moved);
}

// the last sequence whose entries begin at or before i
__device__ __forceinline__ int owner_of(const int32_t* indptr, int lo, int hi, int i) {
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (indptr[mid] <= i) lo = mid;
        else hi = mid;
    }
    return lo;
}

constexpr int kFillStaged = 2048;                             // sequences whose offsets and requests are looked up in shared memory
__global__ void __launch_bounds__(kFillThreads)
kap_fill_tables_kernel(const TableParams p, const int list_blocks)
{
    __shared__ int32_t staged[kFillStaged + 1], staged_request[kFillStaged];
    const bool lists = (int)blockIdx.x < list_blocks, stage = p.batch <= kFillStaged;
    const int at = (lists ? blockIdx.x : blockIdx.x - list_blocks) * kFillEntries;
    // (It lets nothing start before it ends: attention kernels read block tables ahead of their dependency wait.)
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int32_t* indptr = lists ? p.bt_indptr : p.new_indptr;
    if (stage) {
        for (int b = threadIdx.x; b <= p.batch; b += kFillThreads) {
            staged[b] = indptr[b];
            if (b < p.batch) staged_request[b] = p.request ? p.request[b] : b;
        }
        __syncthreads();
        indptr = staged;
    }
    const int end = min(at + kFillEntries, indptr[p.batch]);
    if (at >= end) return;
    const int b1 = owner_of(indptr, 0, p.batch, end - 1) + 1;
    int b = owner_of(indptr, 0, b1, at);
#pragma unroll 4
    for (int i = at + threadIdx.x; i < end; i += kFillThreads) {
        if (i >= indptr[b + 1]) b = owner_of(indptr, b, b1, i);
        const int place = i - indptr[b];
        const long long row = (stage ? staged_request[b] : p.request ? p.request[b] : b) * p.table_stride;
        if (lists) {
            p.bt_pages[i] = p.page_table[row + place];
        } else {
            const int pos = p.ctx_len[b] + place;
            if (p.position) p.position[i] = pos;
            if (p.slot) p.slot[i] = (long long)p.page_table[row + pos / p.page_size] * p.page_size + pos % p.page_size;
        }
    }
}

bool misaligned(const void* a, uintptr_t bits) { return (reinterpret_cast<uintptr_t>(a) & bits) != 0; }

kap_status check_state(int32_t batch, int32_t page_size, const void* page_table, int32_t num_requests, int64_t table_stride, const void* pages_held,
                       const void* free_pages, int32_t free_capacity, const void* free_count, const int32_t* request, const int32_t* device_status) {
    if (batch < 0 || page_size <= 0 || num_requests < 0 || table_stride < 0 || free_capacity < 0)
        return fail(KAP_ERR_INVALID_ARG, "batch %d, page_size %d, %d requests of %lld pages, %d free pages", batch, page_size, num_requests, (long long)table_stride, free_capacity);
    if (num_requests > kMaxRequests || table_stride > INT32_MAX) return fail(KAP_ERR_UNSUPPORTED, "%d requests of %lld pages (at most %d)", num_requests, (long long)table_stride, kMaxRequests);
    if (batch > num_requests) return fail(KAP_ERR_INVALID_ARG, "%d sequences of %d requests", batch, num_requests);
    if (batch > 0 && (!page_table || !pages_held || !free_pages || !free_count)) return fail(KAP_ERR_INVALID_ARG, "NULL pointer");
    for (const void* a : {page_table, pages_held, free_pages, free_count, (const void*)request, (const void*)device_status})
        if (misaligned(a, 3)) return fail(KAP_ERR_INVALID_ARG, "an index array is not 4-byte aligned");
    return KAP_OK;
}

template <bool kRelease>
kap_status launch(const TableParams& p, cudaStream_t stream) {
    const bool few = p.batch <= kFewThreads;
    auto* kernel = few ? kap_tables_kernel<kRelease, kFewThreads> : kap_tables_kernel<kRelease, kTableThreads>;
    const size_t smem = (size_t)(p.num_requests + 31) / 32 * 4;
    if (smem > 32 * 1024) {                                   // with the kernel's own arrays more than the default 48 KiB
        // (always to the most that a call may need: another thread's call must not find less than it asked for)
        cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxRequests / 8);
        if (e != cudaSuccess) return fail(KAP_ERR_CUDA, "cudaFuncSetAttribute failed: %s", cudaGetErrorString(e));
    }
    kernel<<<1, few ? kFewThreads : kTableThreads, smem, stream>>>(p);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return fail(KAP_ERR_CUDA, "block table kernel launch failed: %s", cudaGetErrorString(e));
    count_launch();
    return KAP_OK;
}

}  // namespace
}  // namespace kap

using namespace kap;

extern "C" kap_status kap_build_block_tables(
    const int32_t* request, const int32_t* ctx_len, const int32_t* n_new, int32_t batch, int32_t page_size, int32_t* page_table,
    int32_t num_requests, int64_t table_stride, int32_t* pages_held, int32_t* free_pages, int32_t free_capacity, int32_t* free_count,
    int32_t* bt_indptr, int32_t* bt_pages, int64_t bt_capacity, int32_t* new_indptr, int64_t* slot, int32_t* position, int64_t row_capacity,
    int32_t* device_status, void* cuda_stream)
{
    kap_status st = check_state(batch, page_size, page_table, num_requests, table_stride, pages_held, free_pages, free_capacity, free_count, request, device_status);
    if (st != KAP_OK) return st;
    if (bt_capacity < 0 || row_capacity < 0) return fail(KAP_ERR_INVALID_ARG, "bt_capacity %lld, row_capacity %lld", (long long)bt_capacity, (long long)row_capacity);
    if (!bt_indptr || (batch > 0 && (!ctx_len || !bt_pages))) return fail(KAP_ERR_INVALID_ARG, "NULL pointer");
    if ((slot || position) && !new_indptr) return fail(KAP_ERR_INVALID_ARG, "slot and position need new_indptr");
    for (const void* a : {(const void*)ctx_len, (const void*)n_new, (const void*)bt_indptr, (const void*)bt_pages, (const void*)new_indptr, (const void*)position})
        if (misaligned(a, 3)) return fail(KAP_ERR_INVALID_ARG, "an index array is not 4-byte aligned");
    if (misaligned(slot, 7)) return fail(KAP_ERR_INVALID_ARG, "slot is not 8-byte aligned");
    TableParams p{};
    p.request = request; p.ctx_len = ctx_len; p.n_new = n_new; p.page_table = page_table; p.pages_held = pages_held;
    p.free_pages = free_pages; p.free_count = free_count; p.bt_indptr = bt_indptr; p.bt_pages = bt_pages; p.new_indptr = new_indptr;
    p.slot = reinterpret_cast<long long*>(slot); p.position = position; p.status = device_status;
    p.table_stride = table_stride; p.bt_capacity = bt_capacity < kMostEntries ? bt_capacity : kMostEntries;
    p.row_capacity = (slot || position) && row_capacity < kMostEntries ? row_capacity : kMostEntries;
    p.batch = batch; p.page_size = page_size; p.num_requests = num_requests; p.free_capacity = free_capacity;
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    if (batch == 0) {                                         // an empty table
        cudaError_t e = cudaMemsetAsync(bt_indptr, 0, sizeof(int32_t), stream);
        if (e == cudaSuccess && new_indptr) e = cudaMemsetAsync(new_indptr, 0, sizeof(int32_t), stream);
        return e == cudaSuccess ? KAP_OK : fail(KAP_ERR_CUDA, "cudaMemsetAsync failed: %s", cudaGetErrorString(e));
    }
    st = launch<false>(p, stream);
    if (st != KAP_OK) return st;
    const int64_t list_blocks = (p.bt_capacity + kFillEntries - 1) / kFillEntries;
    const int64_t row_blocks = slot || position ? (p.row_capacity + kFillEntries - 1) / kFillEntries : 0;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(list_blocks + row_blocks > 0 ? list_blocks + row_blocks : 1));
    cfg.blockDim = dim3(kFillThreads);
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = launch_programmatically() ? 1 : 0;
    cudaError_t e = cudaLaunchKernelEx(&cfg, kap_fill_tables_kernel, p, (int)list_blocks);
    if (e != cudaSuccess) return fail(KAP_ERR_CUDA, "block table kernel launch failed: %s", cudaGetErrorString(e));
    count_launch();
    return KAP_OK;
}

extern "C" kap_status kap_release_pages(
    const int32_t* request, int32_t n, const int32_t* keep_tokens, int32_t page_size, int32_t* page_table, int32_t num_requests, int64_t table_stride,
    int32_t* pages_held, int32_t* free_pages, int32_t free_capacity, int32_t* free_count, int32_t* device_status, void* cuda_stream)
{
    kap_status st = check_state(n, page_size, page_table, num_requests, table_stride, pages_held, free_pages, free_capacity, free_count, request, device_status);
    if (st != KAP_OK) return st;
    if (misaligned(keep_tokens, 3)) return fail(KAP_ERR_INVALID_ARG, "an index array is not 4-byte aligned");
    if (n == 0) return KAP_OK;
    TableParams p{};
    p.request = request; p.ctx_len = keep_tokens; p.page_table = page_table; p.pages_held = pages_held;
    p.free_pages = free_pages; p.free_count = free_count; p.status = device_status; p.table_stride = table_stride;
    p.batch = n; p.page_size = page_size; p.num_requests = num_requests; p.free_capacity = free_capacity;
    return launch<true>(p, (cudaStream_t)cuda_stream);
}
