// Work-list structures of kap_shared_prefix_attn, shared by its host scheduler and its kernels.
#pragma once
#include "kap_internal.h"

namespace kap {

constexpr int kPrefixStepPages = 4;                    // a step: 64 tokens
constexpr int kPrefixStepTokens = kPrefixStepPages * kPageSize;
constexpr int kPrefixTileRows = 128;                   // query rows of one tile (TMEM lanes)
constexpr int kPrefixUnitRows = 2 * kPrefixTileRows;

enum { kSegPrefix = 1, kSegPair = 2, kSegTwoStates = 4 };

struct alignas(16) PrefixSegment {                     // what one CTA does of one unit
    int32_t seq;                                       // sequence whose block table is read
    int32_t kv_head, flags;
    int32_t first_page, n_pages;                       // the unit's pages in that table
    int32_t step_begin, step_end;                      // steps of the unit
    int32_t tok_row0;                                  // token row of q that holds the unit's first query row
    int32_t rows, n_q;                                 // query rows; rows per sequence (own parts only)
    int32_t state_row0;                                // first row of its state(s) in the partial buffer
    int32_t pad[5];
};
static_assert(sizeof(PrefixSegment) == 64, "segments are read as four 16-byte pieces");

struct alignas(16) PrefixUnit { int32_t state_row0, rows, n_states, pad; };
struct alignas(16) PrefixSeq {                         // where the merge pass finds a sequence's states
    int32_t row0, n_q;
    int32_t own_unit0, prefix_unit0;                   // unit of KV head 0, or -1
    int32_t n_pairs, group_row0;                       // prefix units per KV head; the group's first token row
    int32_t list_pages, pad;
};
struct PrefixRow { int32_t seq, back; };               // a token row's sequence, and its place minus the last row's

struct PrefixSchedule {
    std::vector<PrefixSegment> segments;
    std::vector<PrefixUnit> units;
    std::vector<PrefixSeq> seqs;
    std::vector<PrefixRow> rows;
    std::vector<int32_t> cta_begin;                    // [n_cta + 1]
    int32_t n_cta = 0, total_rows = 0;
    int64_t state_rows = 0;
};
// sequences, rows and CTA ranges travel as one block
inline size_t prefix_blob_bytes(const PrefixSchedule& s) {
    return s.seqs.size() * sizeof(PrefixSeq) + s.rows.size() * sizeof(PrefixRow) + s.cta_begin.size() * sizeof(int32_t);
}

kap_status build_prefix_schedule(int32_t batch, const int32_t* list_len, const int32_t* n_q, int32_t n_groups,
                                 const int32_t* group_indptr, const int32_t* prefix_pages, int32_t hq, int32_t hkv,
                                 int32_t cta_slots, PrefixSchedule& out);
int64_t prefix_items_needed(const PrefixSchedule& s, int32_t max_rows);

}  // namespace kap
