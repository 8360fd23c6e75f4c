// The work list of kap_shared_prefix_attn (host code, no GPU).
//
// A group's shared pages are read once per KV head for all of the group's query rows.  With more than 32 rows they go to
// the tcgen05 kernel, in blocks of up to 256 rows (two tiles of 128) and steps of 80 tokens; with fewer, and for the pages that a
// sequence has of its own, to the split kernel, whose unit is one (rows, KV head, slice of a page list).  Every piece leaves
// un-normalised states (m, l, O) that the merge pass joins.
#include <algorithm>
#include <exception>
#include <functional>

#include "kap_prefix.h"

namespace kap {

namespace {

// Row counts up to which the split kernel takes a prefix.  Measured on B200 (8 KV heads, one group; split / tcgen05, us a call): 16 rows
// 8.3 / 12.8 at 512 tokens, 31 / 41 at 32K; 32 rows 10.3 / 13.4 and 35 / 40; 64 rows 13.9 / 14.7 and 53 / 42.
constexpr int32_t kSplitRows = 2 * kRowTile;
constexpr int32_t kSplitCtasPerSm = 3;
constexpr int32_t kMinSplitPages = 4;                          // a page for each of a CTA's warps
constexpr int32_t kMaxSplitPages = 1024;                       // page ids a CTA holds: 1600
// Short parts of at most 16 rows may go four KV heads to a CTA, one per warp, instead of a CTA each: for many short lists a CTA is
// mostly start-up (256 sequences with up to 19 own pages on a prefix of 8K: the call takes 72 us, with a CTA for each head 83).  A warp alone takes about a
// microsecond a page, so long lists do not belong there.
constexpr int32_t kByHeadPages = 48;
// What a CTA of the split kernel takes, in pages that one warp group streams (about a microsecond each): its start and its end as much
// as five.  Measured on B200: 384 slices of 16 pages of 32 rows (two groups, one wave) 14.5 us, 768 of 8 pages 21.5; 384 of 16 pages
// of 4 rows (four groups) 8.
constexpr int32_t kSliceTime = 5;
// A segment of the tcgen05 kernel pays for its query tiles, the pipeline's fill and its states about as much as for two steps.
constexpr int64_t kSegmentSteps = 2;
constexpr int32_t kMaxLists = 1 << 23;
constexpr int32_t kMaxCtaSlots = 4096;

struct Unit {                                                  // of the tcgen05 kernel
    int32_t seq, kv_head, n_pages, tok_row0, rows, unit;
};
struct Tape {                                                  // row blocks that walk over the same pages side by side
    int32_t steps, first_unit, n_units;                        // consecutive entries of the unit list
};

// CTAs that walk over the same pages side by side, for different row blocks, so that the pages come from memory once: the
// largest width up to eight that wastes at most 3 % more CTA time than the best one (blocks that do not fill the last
// bundle, SMs that do not fill one).
int32_t bundle_width(const std::vector<std::pair<int32_t, int64_t>>& groups /* (row blocks, steps) */, int32_t sm_count) {
    double waste[9], best = 1e300;
    for (int32_t w = 1; w <= 8; ++w) {
        double used = 0, need = 0;
        for (const auto& g : groups) {
            used += (double)((g.first + w - 1) / w * w) * (double)g.second;
            need += (double)g.first * (double)g.second;
        }
        waste[w] = w > sm_count || need == 0 ? 1e300 : used / need * sm_count / (sm_count / w * w);
        best = std::min(best, waste[w]);
    }
    for (int32_t w = 8; w > 1; --w)
        if (waste[w] <= 1.03 * best) return w;
    return 1;
}

}  // namespace

kap_status build_prefix_schedule(int32_t batch, const int32_t* list_len, const int32_t* n_q, int32_t n_groups,
                                 const int32_t* group_indptr, const int32_t* prefix_pages, int32_t hq, int32_t hkv,
                                 int32_t sm_count, PrefixSchedule& out)
{
    if (batch < 0 || n_groups < 0 || (batch > 0 && (!list_len || !n_q || !group_indptr || !prefix_pages)))
        return fail(KAP_ERR_INVALID_ARG, "NULL pointer, batch %d or n_groups %d", batch, n_groups);
    if (hq <= 0 || hkv <= 0 || hq % hkv) return fail(KAP_ERR_INVALID_ARG, "head counts %d / %d", hq, hkv);
    const int32_t G = hq / hkv;
    if (kRowTile % G) return fail(KAP_ERR_UNSUPPORTED, "group size %d must divide %d", G, kRowTile);
    if (batch > 0 && (n_groups < 1 || group_indptr[0] != 0 || group_indptr[n_groups] != batch))
        return fail(KAP_ERR_INVALID_ARG, "group_indptr must run from 0 to the batch size %d", batch);
    // (a list is a sequence's pages for one KV head; the counts below stay within 32 bits with room to spare)
    if ((int64_t)batch * hkv > kMaxLists) return fail(KAP_ERR_CAPACITY, "%d sequences x %d KV heads exceed %d lists", batch, hkv, kMaxLists);
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
    out.seqs.resize((size_t)batch);
    std::vector<Unit> tc;
    std::vector<std::pair<int32_t, int64_t>> widths;
    struct Part { int32_t seq, kv_head, first_page, n_pages, rows, n_q, prefix, row0, unit; };
    std::vector<Part> parts;                                   // of the split kernel
    std::vector<int32_t> blocks_of;                            // per tcgen05 group: row blocks
    int32_t row = 0;
    for (int32_t i = 0; i < n_groups && batch > 0; ++i) {
        const int32_t b0 = group_indptr[i], b1 = group_indptr[i + 1], row0 = row;
        // a prefix that only one sequence reads is part of that sequence's own pages
        const int32_t shared = b1 - b0 > 1 ? prefix_pages[i] : 0;
        for (int32_t b = b0; b < b1; ++b) {
            out.seqs[(size_t)b] = PrefixSeq{row, list_len[b], -1, -1, 0, 1, row0, 0};
            for (int32_t j = 0; j < n_q[b]; ++j) out.rows.push_back(PrefixRow{b, j + 1 - n_q[b]});
            row += n_q[b];
        }
        if (shared > 0) {
            const int32_t rows = (row - row0) * G;
            const bool split = rows <= kSplitRows;
            const int32_t block = split ? rows : kPrefixUnitRows, blocks = (rows + block - 1) / block;
            for (int32_t b = b0; b < b1; ++b) {
                PrefixSeq& s = out.seqs[(size_t)b];
                s.prefix_unit0 = (int32_t)out.units.size(); s.n_blocks = blocks; s.block_rows = block;
            }
            for (int32_t g = 0; g < hkv; ++g)
                for (int32_t k = 0; k < blocks; ++k) {
                    const int32_t n = std::min(block, rows - k * block), unit = (int32_t)out.units.size();
                    out.units.push_back(PrefixUnit{0, n, 0, 0});
                    if (split) parts.push_back(Part{b0, g, 0, shared, n, row - row0, 1, row0, unit});
                    else tc.push_back(Unit{b0, g, shared, row0 + k * block / G, n, unit});
                }
            if (!split) {
                widths.emplace_back(blocks, (int64_t)hkv * ((shared + kPrefixStepPages - 1) / kPrefixStepPages));
                for (int32_t g = 0; g < hkv; ++g) blocks_of.push_back(blocks);
            }
        }
        for (int32_t b = b0; b < b1; ++b) {
            if (list_len[b] <= shared) continue;
            out.seqs[(size_t)b].own_unit0 = (int32_t)out.units.size();
            for (int32_t g = 0; g < hkv; ++g) {
                parts.push_back(Part{b, g, shared, list_len[b] - shared, n_q[b] * G, n_q[b], 0, out.seqs[(size_t)b].row0, (int32_t)out.units.size()});
                out.units.push_back(PrefixUnit{0, n_q[b] * G, 0, 0});
            }
        }
    }
    out.total_rows = row;
    int64_t state_rows = 0;

    // ---- split kernel: near-equal slices, the longest first, cut where a simulated run ends soonest
    const int64_t slots = (int64_t)sm_count * kSplitCtasPerSm;
    struct Plan { int32_t chunk, limit; };                     // pages a slice; pages up to which parts go four heads to a CTA
    auto slices = [](const Part& p, int32_t chunk) { return (p.n_pages + chunk - 1) / chunk; };
    auto shares_cta = [&](const Part& p, int32_t limit) { return hkv % 4 == 0 && !p.prefix && p.rows <= kRowTile && p.n_pages <= limit; };
    std::vector<int32_t> times;
    std::vector<int64_t> ends;
    auto makespan = [&](const Plan& plan) {
        times.clear();
        int64_t total = 0;
        for (size_t i = 0; i < parts.size(); ++i) {
            const Part& p = parts[i];
            const bool by_head = shares_cta(p, plan.limit);
            if (by_head && p.kv_head % 4) continue;
            const int32_t tiles = (p.rows + kRowTile - 1) / kRowTile, groups = by_head ? 1 : tiles == 1 ? 4 : tiles == 2 ? 2 : 1;
            const int32_t n = by_head ? 1 : slices(p, plan.chunk), most = (p.n_pages + n - 1) / n;
            for (int32_t k = 0; k < n; ++k) times.push_back(kSliceTime + (most + groups - 1) / groups);
            total += (int64_t)n * times.back();
        }
        if ((int64_t)times.size() > 8 * slots) return total / slots + kSliceTime;       // many waves: the sum decides
        std::sort(times.begin(), times.end(), std::greater<int32_t>());
        ends.assign((size_t)slots, 0);                         // a heap: the CTA place that is free first takes the next slice
        int64_t last = 0;
        for (int32_t t : times) {
            std::pop_heap(ends.begin(), ends.end(), std::greater<int64_t>());
            ends.back() += t;
            last = std::max(last, ends.back());
            std::push_heap(ends.begin(), ends.end(), std::greater<int64_t>());
        }
        return last;
    };
    Plan plan{kMaxSplitPages, 0};
    if (!parts.empty()) {
        int64_t best = makespan(plan);
        for (int32_t limit = 0; limit <= kByHeadPages; limit += limit < 16 ? 4 : 16)
            for (int32_t chunk = kMinSplitPages; chunk <= kMaxSplitPages; chunk += std::max(2, chunk / 3)) {
                const Plan other{chunk, limit};
                const int64_t t = makespan(other);
                if (t < best) { best = t; plan = other; }
            }
    }
    struct Timed { WorkItem item; int32_t pages; };            // pages that the busiest warp streams
    std::vector<Timed> timed;
    for (size_t i = 0; i < parts.size();) {
        const Part& p = parts[i];
        const bool by_head = shares_cta(p, plan.limit);
        const int32_t n = by_head ? 1 : slices(p, plan.chunk), heads = by_head ? 4 : 1;   // (a part's heads follow one another)
        for (int32_t h = 0; h < heads; ++h) {
            PrefixUnit& u = out.units[(size_t)parts[i + (size_t)h].unit];
            u.state_row0 = (int32_t)(state_rows + (int64_t)h * p.rows); u.n_states = n;
        }
        for (int32_t k = 0; k < n; ++k) {
            const int32_t from = (int32_t)((int64_t)p.n_pages * k / n), to = (int32_t)((int64_t)p.n_pages * (k + 1) / n);
            const int32_t group = (p.prefix ? 1 : 0) | (by_head ? 2 : 0);
            timed.push_back(Timed{WorkItem{p.seq, p.kv_head, p.first_page + from, p.first_page + to, group,
                                           (int32_t)(state_rows + (int64_t)k * p.rows), p.row0, p.n_q}, by_head ? to - from : (to - from + 3) / 4});
        }
        state_rows += (int64_t)n * heads * p.rows;
        if (state_rows > 0x7fffffff) return fail(KAP_ERR_CAPACITY, "the schedule needs %lld state rows", (long long)state_rows);
        i += (size_t)heads;
    }
    std::stable_sort(timed.begin(), timed.end(), [](const Timed& a, const Timed& b) { return a.pages > b.pages; });
    for (const Timed& t : timed) out.items.push_back(t.item);

    // ---- tcgen05 kernel: the tapes of all (group, KV head, bundle of row blocks) end to end, cut into equal pieces; bundle b of
    // `width` CTAs takes piece b, CTA p of it row block p
    if (!tc.empty()) {
        const int32_t width = bundle_width(widths, sm_count);
        std::vector<Tape> tapes;
        int64_t cost = 0, steps = 0;
        for (size_t at = 0, k = 0; at < tc.size(); ++k) {
            const int32_t blocks = blocks_of[k];
            for (int32_t j = 0; j < blocks; j += width) {
                Tape t{(tc[at].n_pages + kPrefixStepPages - 1) / kPrefixStepPages, (int32_t)at + j, std::min(width, blocks - j)};
                cost += t.steps + kSegmentSteps;
                steps += t.steps;
                tapes.push_back(t);
            }
            at += (size_t)blocks;
        }
        const int32_t bundles = (int32_t)std::max<int64_t>(1, std::min<int64_t>(sm_count / width, steps));
        cost += (bundles - 1) * kSegmentSteps;                 // a cut tape starts once more
        std::vector<std::vector<PrefixSegment>> per_cta((size_t)bundles * width);
        int64_t spent = 0;
        int32_t bundle = 0;
        for (const Tape& t : tapes) {
            std::vector<int64_t> first((size_t)t.n_units, -1);
            for (int32_t at = 0; at < t.steps;) {
                const int64_t fit = cost * (bundle + 1) / bundles - spent - kSegmentSteps;   // steps that still fit this bundle's share
                if (bundle + 1 < bundles && fit < 1 && spent > cost * bundle / bundles) { ++bundle; continue; }
                const int32_t n = bundle + 1 == bundles ? t.steps - at : (int32_t)std::min<int64_t>(std::max<int64_t>(fit, 1), t.steps - at);
                for (int32_t p = 0; p < t.n_units; ++p) {
                    const Unit& u = tc[(size_t)(t.first_unit + p)];
                    const bool pair = u.rows > kPrefixTileRows, two = !pair && n > 1;   // a single tile's steps alternate between the streams
                    PrefixSegment s{};
                    s.seq = u.seq; s.kv_head = u.kv_head; s.flags = (pair ? kSegPair : 0) | (two ? kSegTwoStates : 0);
                    s.n_pages = u.n_pages; s.step_begin = at; s.step_end = at + n; s.tok_row0 = u.tok_row0; s.rows = u.rows;
                    s.state_row0 = out.units[(size_t)u.unit].n_states;     // the state's number for now
                    s.pad[0] = u.unit;
                    out.units[(size_t)u.unit].n_states += two ? 2 : 1;
                    per_cta[(size_t)bundle * width + p].push_back(s);
                }
                at += n;
                spent += n + kSegmentSteps;
            }
        }
        for (const Unit& u : tc) {
            PrefixUnit& mu = out.units[(size_t)u.unit];
            mu.state_row0 = (int32_t)state_rows;
            state_rows += (int64_t)mu.n_states * mu.rows;
            if (state_rows > 0x7fffffff) return fail(KAP_ERR_CAPACITY, "the schedule needs %lld state rows", (long long)state_rows);
        }
        out.n_cta = bundles * width;
        out.cta_begin.push_back(0);
        for (auto& list : per_cta) {
            for (PrefixSegment& s : list) {
                const PrefixUnit& mu = out.units[(size_t)s.pad[0]];
                s.state_row0 = mu.state_row0 + s.state_row0 * mu.rows;
                s.pad[0] = 0;
                out.segments.push_back(s);
            }
            out.cta_begin.push_back((int32_t)out.segments.size());
        }
    }
    out.state_rows = state_rows;
    return KAP_OK;
}

int64_t prefix_items_needed(const PrefixSchedule& s, int32_t max_rows) {
    auto up = [](size_t bytes) { return (int64_t)((bytes + sizeof(WorkItem) - 1) / sizeof(WorkItem)); };
    const PrefixLayout at = prefix_layout(s);
    int64_t n = std::max<int64_t>(1, (s.state_rows + max_rows - 1) / max_rows);
    n = std::max(n, up(at.first_bytes));
    n = std::max(n, up(at.second_bytes));
    return std::max(n, up(at.third_bytes));
}

}  // namespace kap

extern "C" kap_status kap_shared_prefix_items(
    int32_t batch, const int32_t* list_len, const int32_t* n_q, int32_t n_groups, const int32_t* group_indptr,
    const int32_t* prefix_pages, int32_t num_q_heads, int32_t num_kv_heads, int32_t max_rows_per_item, int32_t cta_slots,
    int32_t* max_items)
{
    using namespace kap;
    if (!max_items || max_rows_per_item <= 0 || cta_slots <= 0 || cta_slots > kMaxCtaSlots)
        return fail(KAP_ERR_INVALID_ARG, "NULL pointer, sizes below 1 or more than %d cta_slots", kMaxCtaSlots);
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
