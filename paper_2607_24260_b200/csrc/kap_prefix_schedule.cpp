// The work list of kap_shared_prefix_attn (host code, no GPU).
//
// Units of work: a shared prefix for one KV head and up to 256 of the group's query rows (two tiles of 128),
// or one sequence's own pages for one KV head.  A unit is a run of steps of 64 tokens (four pages); all units
// laid end to end form a tape, which is cut into one piece per CTA of nearly equal cost, so that a long prefix is
// spread over the whole device and many short own parts are dealt out in runs.  What a CTA gets of one unit is
// a segment; every segment leaves un-normalised states (m, l, O) that the merge pass joins.
#include <algorithm>
#include <exception>

#include "kap_prefix.h"

namespace kap {

namespace {

struct Unit {
    int32_t seq, kv_head, first_page, n_pages, tok_row0, rows, flags, n_q, merge_unit;
    int32_t steps() const { return (n_pages + kPrefixStepPages - 1) / kPrefixStepPages; }
};

// Costs in thirds of a 64-token step of two row tiles (about 1300 cycles of the tensor core).  A step of a single
// tile is bound by its 32 KiB from memory; a segment pays for its query tile, the pipeline's fill and its states.
constexpr int64_t kPairCost = 3, kSoloCost = 3, kSegmentCost = 6;

}  // namespace

kap_status build_prefix_schedule(int32_t batch, const int32_t* list_len, const int32_t* n_q, int32_t n_groups,
                                 const int32_t* group_indptr, const int32_t* prefix_pages, int32_t hq, int32_t hkv,
                                 int32_t cta_slots, PrefixSchedule& out)
{
    if (batch < 0 || n_groups < 0 || (batch > 0 && (!list_len || !n_q || !group_indptr || !prefix_pages)))
        return fail(KAP_ERR_INVALID_ARG, "NULL pointer, batch %d or n_groups %d", batch, n_groups);
    if (hq <= 0 || hkv <= 0 || hq % hkv) return fail(KAP_ERR_INVALID_ARG, "head counts %d / %d", hq, hkv);
    const int32_t G = hq / hkv;
    if (kRowTile % G) return fail(KAP_ERR_UNSUPPORTED, "group size %d must divide %d", G, kRowTile);
    if (batch > 0 && (n_groups < 1 || group_indptr[0] != 0 || group_indptr[n_groups] != batch))
        return fail(KAP_ERR_INVALID_ARG, "group_indptr must run from 0 to the batch size %d", batch);
    for (int32_t b = 0; b < batch; ++b) {
        if (list_len[b] <= 0 || n_q[b] < 1 || list_len[b] > 0x7fffffff / kPageSize) return fail(KAP_ERR_INVALID_ARG, "sequence %d: list_len %d, n_q %d", b, list_len[b], n_q[b]);
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

    out = PrefixSchedule();
    std::vector<Unit> units;
    auto add = [&](Unit u) {
        u.merge_unit = (int32_t)units.size();
        units.push_back(u);
    };
    out.seqs.resize((size_t)batch);
    int32_t row = 0;
    for (int32_t i = 0; i < n_groups && batch > 0; ++i) {
        const int32_t b0 = group_indptr[i], b1 = group_indptr[i + 1], row0 = row;
        for (int32_t b = b0; b < b1; ++b) {
            PrefixSeq& s = out.seqs[(size_t)b];
            s = PrefixSeq{row, n_q[b], -1, -1, 0, row0, list_len[b], 0};
            for (int32_t j = 0; j < n_q[b]; ++j) out.rows.push_back(PrefixRow{b, j + 1 - n_q[b]});
            row += n_q[b];
        }
        // a prefix that only one sequence reads is part of that sequence's own pages
        const int32_t shared = b1 - b0 > 1 ? prefix_pages[i] : 0;
        if (shared > 0) {
            const int32_t rows = (row - row0) * G, pairs = (rows + kPrefixUnitRows - 1) / kPrefixUnitRows;
            for (int32_t b = b0; b < b1; ++b) {
                out.seqs[(size_t)b].prefix_unit0 = (int32_t)units.size();
                out.seqs[(size_t)b].n_pairs = pairs;
            }
            for (int32_t g = 0; g < hkv; ++g)
                for (int32_t p = 0; p < pairs; ++p) {
                    const int32_t r0 = p * kPrefixUnitRows, n = std::min(kPrefixUnitRows, rows - r0);
                    add(Unit{b0, g, 0, shared, row0 + r0 / G, n, kSegPrefix | (n > kPrefixTileRows ? kSegPair : 0), 0, 0});
                }
        }
        for (int32_t b = b0; b < b1; ++b) {
            PrefixSeq& s = out.seqs[(size_t)b];
            if (list_len[b] <= shared) continue;
            s.own_unit0 = (int32_t)units.size();
            for (int32_t g = 0; g < hkv; ++g)
                add(Unit{b, g, shared, list_len[b] - shared, s.row0, n_q[b] * G, 0, n_q[b], 0});
        }
    }
    out.total_rows = row;
    out.units.resize(units.size());

    // shared prefixes first (long, bound by the tensor cores), then the own parts
    std::stable_sort(units.begin(), units.end(), [](const Unit& a, const Unit& b) { return (a.flags & kSegPrefix) > (b.flags & kSegPrefix); });
    auto step_cost = [](const Unit& u) { return u.flags & kSegPair ? kPairCost : kSoloCost; };
    int64_t cost = 0, steps = 0;
    for (const Unit& u : units) { cost += u.steps() * step_cost(u) + kSegmentCost; steps += u.steps(); }
    const int32_t n_cta = (int32_t)std::max<int64_t>(1, std::min<int64_t>(cta_slots, steps));
    cost += (n_cta - 1) * kSegmentCost;                        // a cut unit starts once more
    int64_t spent = 0;                                         // cost of everything handed out so far
    int32_t cta = 0;
    out.cta_begin.push_back(0);
    int64_t state_rows = 0;
    for (const Unit& u : units) {
        PrefixUnit& mu = out.units[(size_t)u.merge_unit];
        mu.state_row0 = (int32_t)state_rows; mu.rows = u.rows; mu.n_states = 0; mu.pad = 0;
        for (int32_t at = 0; at < u.steps();) {
            // steps that still fit this CTA's share; the last CTA takes what is left
            int64_t end = cost * (cta + 1) / n_cta;
            int64_t fit = (end - spent - kSegmentCost + step_cost(u) / 2) / step_cost(u);
            if (cta + 1 < n_cta && fit < 1 && spent > cost * cta / n_cta) {   // not even one: the next CTA's
                ++cta;
                out.cta_begin.push_back((int32_t)out.segments.size());
                continue;
            }
            const int32_t n = cta + 1 == n_cta ? u.steps() - at : (int32_t)std::min<int64_t>(std::max<int64_t>(fit, 1), u.steps() - at);
            const bool two = !(u.flags & kSegPair) && n > 1;   // a single tile's steps alternate between the two streams
            PrefixSegment s{};
            s.seq = u.seq; s.kv_head = u.kv_head; s.flags = u.flags | (two ? kSegTwoStates : 0);
            s.first_page = u.first_page; s.n_pages = u.n_pages; s.step_begin = at; s.step_end = at + n;
            s.tok_row0 = u.tok_row0; s.rows = u.rows; s.n_q = u.n_q;
            s.state_row0 = (int32_t)(state_rows + (int64_t)mu.n_states * u.rows);
            mu.n_states += two ? 2 : 1;
            out.segments.push_back(s);
            at += n;
            spent += n * step_cost(u) + kSegmentCost;
        }
        state_rows += (int64_t)mu.n_states * u.rows;
        if (state_rows > 0x7fffffff) return fail(KAP_ERR_CAPACITY, "the schedule needs %lld state rows", (long long)state_rows);
    }
    out.cta_begin.push_back((int32_t)out.segments.size());
    out.n_cta = (int32_t)out.cta_begin.size() - 1;
    out.state_rows = state_rows;
    return KAP_OK;
}

int64_t prefix_items_needed(const PrefixSchedule& s, int32_t max_rows) {
    auto up = [](int64_t bytes) { return (bytes + (int64_t)sizeof(WorkItem) - 1) / (int64_t)sizeof(WorkItem); };
    int64_t n = std::max<int64_t>(1, (s.state_rows + max_rows - 1) / max_rows);
    n = std::max(n, up((int64_t)(s.segments.size() * sizeof(PrefixSegment))));
    n = std::max(n, up((int64_t)(s.units.size() * sizeof(PrefixUnit))));
    return std::max(n, up((int64_t)prefix_blob_bytes(s)));
}

}  // namespace kap

extern "C" kap_status kap_shared_prefix_items(
    int32_t batch, const int32_t* list_len, const int32_t* n_q, int32_t n_groups, const int32_t* group_indptr,
    const int32_t* prefix_pages, int32_t num_q_heads, int32_t num_kv_heads, int32_t max_rows_per_item, int32_t cta_slots,
    int32_t* max_items)
{
    using namespace kap;
    if (!max_items || max_rows_per_item <= 0 || cta_slots <= 0) return fail(KAP_ERR_INVALID_ARG, "NULL pointer or sizes below 1");
    try {
        PrefixSchedule s;
        kap_status st = build_prefix_schedule(batch, list_len, n_q, n_groups, group_indptr, prefix_pages, num_q_heads, num_kv_heads, cta_slots, s);
        if (st != KAP_OK) return st;
        const int64_t n = prefix_items_needed(s, max_rows_per_item);
        if (n > 0x7fffffff) return fail(KAP_ERR_CAPACITY, "the schedule needs %lld items", (long long)n);
        *max_items = (int32_t)n;
    } catch (const std::exception& e) {                        // no exception leaves a C entry point
        return fail(KAP_ERR_CAPACITY, "the schedule does not fit the host's memory: %s", e.what());
    }
    return KAP_OK;
}
