// Runs the schedule of attention calls on the CPU, in both forms, and checks what the launched workgroups and the join of parts would then do, column by column: every row
// of the call has its result written once, from its keys, each taken once.  (tests/test_attention_schedule.py)
// Lists are heap blocks of exactly their capacity, filled with garbage, so that with a sanitizer an access past one ends the run, and an entry that nobody wrote
// is seen.  Standard input: KIND DTYPE T S HEADS KV_HEADS GROUPS MAX_KEYS, then seg_start[S + 1], seg_prefill_len[S] and, where KIND is 2, kv_len[S], group_start[GROUPS + 1]
// (if GROUPS) and group_prefix_len[GROUPS].  KIND 1: prompts, 2: over pages; 11 and 12: the same on tables that are malformed, where rows may have any result, but every index has to stay
// within bounds.  KIND 22: no tables follow; whether the sizes fit, the workgroups that a call over pages launches, and the capacities of its tiles, units, merges and parts.  One line for each call: direct, split, join launch, units, units of the grid, entries of the join, and "ok" or what is wrong.
#include "emulated_hip.hpp"

#include "../paper_2605_14217_amd/csrc/attention_plan.hpp"

#include <algorithm>
#include <cstring>
#include <map>
#include <string>

using namespace preft;

template <typename T> struct Block {             // heap memory of exactly n, of bytes that are no sensible entry
    std::vector<T> v;
    explicit Block(size_t n) : v(n) { if (n) std::memset((void *)v.data(), 0x9d, n * sizeof(T)); }
    T *p() { return v.data(); }
};

struct Span { int32_t from, to; };
struct Column { std::vector<Span> direct; int written = 0; };

static std::string check(int kind, int dtype, int32_t T, int32_t S, int32_t heads, int32_t kv_heads, int32_t groups, int64_t max_keys, const std::vector<int32_t> &start,
                         const std::vector<int32_t> &prefill, const std::vector<int32_t> &kv, const std::vector<int32_t> &gstart, const std::vector<int32_t> &gprefix,
                         bool malformed, std::string &facts)
{
    const Layout l = kind == 1 ? prompt_layout(T, S, heads, kv_heads) : cached_layout(T, S, heads, kv_heads, 64, groups);
    AttnLists x = lists_of(l, reinterpret_cast<void *>(4096));        // for its capacities
    Block<int32_t> report(HEADER_INTS), header(HEADER_INTS), tiles(S + groups + 1), rows_before(S + 1), group_of(S), group_list(groups), group_slot(groups), group_low(groups);
    Block<AttnUnit> units(l.unit_cap);
    Block<AttnMerge> merges(l.merge_cap);
    Block<int2> group_rows(l.group_row_cap);
    x.header = header.p(); x.units = units.p(); x.merges = merges.p(); x.group_rows = group_rows.p(); x.tiles = tiles.p(); x.rows_before = rows_before.p();
    x.group_of = group_of.p(); x.group_list = group_list.p(); x.group_slot = group_slot.p(); x.group_low = group_low.p(); x.report = report.p(); x.part_o = nullptr; x.part_ml = nullptr;
    AttnScheduleArgs s = {};
    s.seg_start = start.data(); s.seg_prefill_len = prefill.data(); s.S = S; s.T = T; s.heads = heads; s.kv_heads = kv_heads; s.group = heads / kv_heads; s.l = x;
    if (kind == 1) {
        prompt_rules(s, dtype);
    } else {
        s.kv_len = kv.data(); s.group_start = gstart.data(); s.group_prefix = gprefix.data(); s.n_groups = groups;
        cached_rules(s, dtype, max_keys);
    }
    const Plan p = plan_of(s);
    if (!p.split) s.can_split = 0;
    std::vector<AttnUnit> run;                        // the units that the launched workgroups process
    if (p.direct) {
        for (int64_t unit = 0; unit < p.units; ++unit) {
            AttnUnit u = {};
            bool found = false;
            emulated::run_block(64, (unsigned)(unit * kv_heads), (unsigned)(p.units * kv_heads), [&] {
                AttnUnit mine;
                const bool f = attn_direct_unit(s, (int32_t)unit, 0, false, mine);
                if (emulated::lane() == 17) { found = f; if (f) u = mine; }
            });
            if (found) run.push_back(u);
        }
    } else {
        emulated::run_block((unsigned)schedule_threads(s), 0, 1, [&] { attn_schedule_kernel(s); });
        const int32_t n = header.v[AH_UNITS], alone = header.v[AH_SHORT];
        if (n < 0 || n > l.unit_cap || alone < 0 || alone > n) return "header counts";
        for (int64_t unit = 0; unit < p.units; ++unit)
            for (int w = 0; w < 4; ++w) {
                const int64_t i = unit < alone ? unit : alone + 4 * (unit - alone) + w;
                if ((unit < alone && w > 0) || i >= n) continue;
                run.push_back(units.v[(size_t)i]);
            }
    }
    const int32_t joins = header.v[AH_JOINS], listed = header.v[AH_UNITS], G = s.group;
    facts = std::to_string(p.direct) + " " + std::to_string(p.split) + " " + std::to_string(p.merge) + " " + std::to_string(listed) + " " + std::to_string(p.units) + " " + std::to_string(p.merge ? joins : 0);
    if (joins < 0 || joins > l.merge_cap) return "entries of the join";

    // what the units do, for key/value head 0 and for the last
    std::map<std::pair<int32_t, int32_t>, Column> out;           // {row, query head of the key/value head}
    struct Part { std::vector<Span> keys; int32_t row, head; };
    std::map<int64_t, Part> parts;                                // of key/value head 0, by its place
    for (const AttnUnit &u : run) {
        if (u.ncols == 0) { if (!malformed) return "a unit without columns"; continue; }
        if (u.ncols < 0 || u.ncols > ATTN_COLS || u.head0 < 0 || u.head0 >= G) return "columns of a unit";
        if (u.table < 0 || u.table >= (kind == 1 ? T : S)) return "a unit's table";
        if (u.key0 < 0 || u.key1 < u.key0 || u.key1 > s.max_keys || (kind == 1 && (int64_t)u.table + u.key1 > T)) return "keys of a unit";
        if (u.slot >= 0 && (int64_t)u.slot + (int64_t)u.ncols * kv_heads > l.slot_cap) return "a unit's parts";
        for (int32_t c = 0; c < u.ncols; ++c) {
            const int32_t i = (u.head0 + c) / G, head = (u.head0 + c) % G;
            int32_t row, lim;
            if (u.row0 >= 0) {
                row = u.row0 + i; lim = u.lim0 + i;
            } else {
                const int64_t at = (int64_t)-1 - u.row0 + i;
                if (malformed && (at < 0 || at >= l.group_row_cap)) continue;       // the kernel keeps to the list
                if (at < 0 || at >= l.group_row_cap) return "rows of a group's unit";
                row = group_rows.v[at].x; lim = group_rows.v[at].y;
            }
            if (malformed) continue;
            if (row < 0 || row >= T) return "a unit's row";
            const Span keys = {u.key0, std::min(lim, u.key1)};
            if (u.slot < 0) {
                Column &o = out[{row, head}];
                ++o.written;
                if (keys.from < keys.to) o.direct.push_back(keys);
            } else {
                const int64_t at = (int64_t)u.slot + c;
                if (parts.count(at)) return "two parts in one place";
                parts[at] = Part{{keys}, row, head};
            }
        }
    }
    // the join
    if (p.merge)
        for (int32_t e = 0; e < joins; ++e) {
            const AttnMerge &j = merges.v[e];
            if (j.parts < 0 || j.group_parts < 0 || j.parts > p.units || j.group_parts > p.units) return "parts of an entry that nobody wrote";
            if (j.parts + j.group_parts == 0) continue;
            if (j.ncols < 0 || j.ncols > ATTN_COLS || j.col0 < 0 || j.group_col0 < 0) return "columns of an entry";
            for (int32_t c = 0; c < j.ncols; ++c) {
                const int32_t gc = j.group_col0 + c, tile = gc / ATTN_COLS, width = std::min(ATTN_COLS, j.group_cols - tile * ATTN_COLS);
                const int64_t group = (int64_t)j.group_slot + (int64_t)tile * ATTN_COLS * kv_heads * j.group_parts + gc % ATTN_COLS, mine = (int64_t)j.slot + c;
                const int32_t row = j.row0 + (j.col0 + c) / G, head = (j.col0 + c) % G;
                if (malformed) continue;
                Column &o = out[{row, head}];
                ++o.written;
                for (int32_t k = 0; k < j.parts + j.group_parts; ++k) {
                    const int64_t at = k < j.parts ? mine + (int64_t)k * j.ncols * kv_heads : group + (int64_t)(k - j.parts) * width * kv_heads;
                    const auto it = parts.find(at);
                    if (it == parts.end()) return "a part that nobody wrote";
                    if (it->second.row != row || it->second.head != head) return "another column's part";
                    for (const Span &sp : it->second.keys)
                        if (sp.from < sp.to) o.direct.push_back(sp);
                }
            }
        }
    if (malformed) return "ok";
    // what the call has to do
    size_t wanted = 0;
    for (int32_t sg = 0; sg < S; ++sg) {
        const int32_t lo = start[sg], hi = start[sg + 1], prompt = std::max(0, std::min(prefill[sg], hi - lo));
        const int32_t first = kind == 1 ? lo : lo + prompt, end = kind == 1 ? lo + prompt : hi;
        for (int32_t row = first; row < end; ++row) {
            const int64_t lim = kind == 1 ? row - lo + 1 : std::max((int64_t)0, std::min((int64_t)kv[sg], (int64_t)s.max_keys) - (end - 1 - row));
            for (int32_t h = 0; h < G; ++h) {
                ++wanted;
                const auto it = out.find({row, h});
                if (it == out.end()) return "row " + std::to_string(row) + " is not written";
                if (it->second.written != 1) return "row " + std::to_string(row) + " is written " + std::to_string(it->second.written) + " times";
                auto &d = it->second.direct;
                std::sort(d.begin(), d.end(), [](const Span &a, const Span &b) { return a.from < b.from; });
                int64_t at = 0;
                for (const Span &sp : d) {
                    if (sp.from != at) return "row " + std::to_string(row) + ": keys from " + std::to_string(at);
                    at = sp.to;
                }
                if (at != lim) return "row " + std::to_string(row) + " sees " + std::to_string(at) + " keys of " + std::to_string(lim);
            }
        }
    }
    if (wanted != out.size()) return "rows that are not the call's are written";
    return "ok";
}

int main()
{
    int kind, dtype;
    long long T, S, heads, kv_heads, groups, max_keys;
    while (std::scanf("%d %d %lld %lld %lld %lld %lld %lld", &kind, &dtype, &T, &S, &heads, &kv_heads, &groups, &max_keys) == 8) {
        auto read = [](long long n) {
            std::vector<int32_t> v((size_t)n);
            for (int32_t &x : v)
                if (std::scanf("%d", &x) != 1) std::exit(2);
            return v;
        };
        if (kind == 22) {
            AttnScheduleArgs s = {};
            const Layout l = cached_layout(T, S, heads, kv_heads, 64, groups);
            s.S = (int32_t)S; s.T = (int32_t)T; s.n_groups = (int32_t)groups; s.heads = (int32_t)heads; s.kv_heads = (int32_t)kv_heads; s.group = (int32_t)(heads / kv_heads);
            s.l = lists_of(l, reinterpret_cast<void *>(4096));
            cached_rules(s, dtype, max_keys);
            const Layout wide = cached_layout(T, S, heads, kv_heads, 128, groups);
            const bool one_place = l.header == wide.header && l.units == wide.units && l.group_low == wide.group_low;
            std::printf("%d %lld %d %d %d %d %s\n", sizes_fit(T, S, heads, groups), (long long)(plan_of(s).units * kv_heads), l.tile_cap, l.unit_cap, l.merge_cap, l.slot_cap,
                        one_place ? "ok" : "schedules of other head sizes stand elsewhere");
            continue;
        }
        const auto start = read(S + 1), prefill = read(S);
        const bool malformed = kind > 10;
        kind %= 10;
        const auto kv = read(kind == 2 ? S : 0), gstart = read(kind == 2 && groups ? groups + 1 : 0), gprefix = read(kind == 2 ? groups : 0);
        std::string facts;
        const std::string what = check(kind, dtype, (int32_t)T, (int32_t)S, (int32_t)heads, (int32_t)kv_heads, (int32_t)groups, max_keys, start, prefill, kv, gstart, gprefix, malformed, facts);
        std::printf("%s %s\n", facts.c_str(), what.c_str());
        std::fflush(stdout);
    }
    return 0;
}
