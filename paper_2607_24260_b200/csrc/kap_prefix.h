// Work-list structures of kap_shared_prefix_attn, shared by its host scheduler and its kernels.
#pragma once
#include "kap_internal.h"

namespace kap {

constexpr int kPrefixStepPages = 5;                    // a step of the tcgen05 kernel: 80 tokens
constexpr int kPrefixStepTokens = kPrefixStepPages * kPageSize;
constexpr int kPrefixTileRows = 128;                   // query rows of one tile (TMEM lanes)
constexpr int kPrefixUnitRows = 2 * kPrefixTileRows;
// Ring of the split kernel, 8 KiB a slot.  More for grids that leave SMs room only cost start-up (4 sequences with 512 shared tokens, 96
// CTAs: 8.3 us with 8 slots, 8.5 with 12, 9.2 with 24).
constexpr int kPrefixRingSlots = 8;

enum { kSegPair = 1, kSegTwoStates = 2 };

struct alignas(16) PrefixSegment {                     // what one CTA of the tcgen05 kernel does of one unit
    int32_t seq;                                       // sequence whose block table is read (from its first page on)
    int32_t kv_head, flags;
    int32_t n_pages;                                   // of the shared prefix
    int32_t step_begin, step_end;                      // steps of it
    int32_t tok_row0, rows;                            // token row of q that holds the unit's first query row; query rows
    int32_t state_row0;                                // first row of its state(s) in the partial buffer
    int32_t pad[3];
};
static_assert(sizeof(PrefixSegment) == 48, "segments are read as three 16-byte pieces");
static_assert(sizeof(MergeGroup) == sizeof(WorkItem), "the workspace's three metadata arrays have max_items entries of one size");

struct alignas(16) PrefixUnit { int32_t state_row0, rows, n_states, pad; };
struct alignas(16) PrefixSeq {                         // where the merge pass finds a sequence's states
    int32_t row0, list_pages;
    int32_t own_unit0, prefix_unit0;                   // unit of KV head 0, or -1
    int32_t n_blocks, block_rows;                      // prefix units per KV head and their query rows
    int32_t group_row0, pad;                           // the group's first token row
};
struct PrefixRow { int32_t seq, back; };               // a token row's sequence, and its place minus the last row's

struct PrefixSchedule {
    std::vector<PrefixSegment> segments;               // of the tcgen05 kernel
    std::vector<int32_t> cta_begin;                    // [n_cta + 1], n_cta = 0: nothing for it
    std::vector<WorkItem> items;                       // of the split kernel: group: 1 a prefix, 2 one warp per KV head;
                                                       // split = first state row; n_splits = first row of q
    std::vector<PrefixUnit> units;
    std::vector<PrefixSeq> seqs;
    std::vector<PrefixRow> rows;
    int32_t n_cta = 0, total_rows = 0;
    int64_t state_rows = 0;
};
// Places of the arrays inside the workspace's metadata: items and segments in the first array, units in the second, sequences,
// rows and CTA ranges in the third.
struct PrefixLayout {
    size_t segments, rows, ctas, first_bytes, second_bytes, third_bytes;
    PrefixLayout(size_t n_items, size_t n_segments, size_t n_units, size_t batch, size_t total_rows, size_t n_cta) {
        segments = n_items * sizeof(WorkItem);
        first_bytes = segments + n_segments * sizeof(PrefixSegment);
        second_bytes = n_units * sizeof(PrefixUnit);
        rows = batch * sizeof(PrefixSeq);
        ctas = rows + total_rows * sizeof(PrefixRow);
        third_bytes = ctas + (n_cta + 1) * sizeof(int32_t);
    }
};
inline PrefixLayout prefix_layout(const PrefixSchedule& s) {
    return PrefixLayout(s.items.size(), s.segments.size(), s.units.size(), s.seqs.size(), s.rows.size(), (size_t)s.n_cta);
}

kap_status build_prefix_schedule(int32_t batch, const int32_t* list_len, const int32_t* n_q, int32_t n_groups,
                                 const int32_t* group_indptr, const int32_t* prefix_pages, int32_t hq, int32_t hkv,
                                 int32_t sm_count, PrefixSchedule& out);
int64_t prefix_items_needed(const PrefixSchedule& s, int32_t max_rows);

}  // namespace kap
