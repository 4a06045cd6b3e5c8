// How an attention call runs, decided on the host from its sizes: the layout of the workspace, whether workgroups find their units themselves, how many there
// are, and whether parts are joined.  Needs no device.
#pragma once
#include "../../include/preft.h"
#include "attention_schedule.hpp"

namespace preft {

// Bounds on the lists, for tables that are well-formed:
//   column tiles   T G / 128 + one part-filled tile a segment, and the same of groups; of segments and groups, no more than rows have any;
//   units          a tile of n key tiles is cut into ceil(n / range) < 1 + n / range ranges, and range is at least the estimate of all tiles' n times
//                  kv_heads / TARGET.  That estimate, from the first and the last tile of a segment, is short by up to two a tile of a causal prompt (list), and
//                  at least half of what counting every tile of a segment like its last gives (direct);
//   part columns   a tile that is cut has at most twice n / range parts of at most 128 columns; rows of groups have one of their own and their group's.
//
// The workspace holds, behind the header that preft_schedule_counts reads, a header, lists and parts of each kind of call: in a mixed step both kinds find their own
// schedule again in every layer.  The prompts' come first, since their size does not depend on the groups of the other call.
struct Layout {
    int32_t tile_cap, unit_cap, merge_cap, group_row_cap, slot_cap;
    size_t header, units, merges, group_rows, tiles, rows_before, group_of, group_list, group_slot, group_low, part_ml, part_o, end;
};

// of one kind of call, from byte `at` on; slots: part columns, but those of groups' rows
inline Layout layout_from(size_t at, int64_t slots, int64_t T, int64_t S, int64_t heads, int64_t kv_heads, int64_t D, int64_t groups)
{
    Layout l;
    const int64_t G = heads / kv_heads, cols = T * G;
    const int64_t seg_tiles = cols / ATTN_COLS + (S < T ? S : T);
    const int64_t tiles = groups > 0 ? 2 * seg_tiles + (groups < T ? groups : T) : seg_tiles;
    l.tile_cap = (int32_t)tiles;
    l.unit_cap = (int32_t)(3 * tiles + 2 * ((ATTN_TARGET + kv_heads - 1) / kv_heads) + 2);
    l.merge_cap = (int32_t)seg_tiles;
    l.group_row_cap = groups > 0 ? (int32_t)(T < ATTN_GROUP_ROWS ? T : ATTN_GROUP_ROWS) : 0;
    l.slot_cap = (int32_t)(slots + 2 * l.group_row_cap * heads);
    auto take = [&](size_t bytes) { const size_t p = at; at = (at + bytes + 63) & ~(size_t)63; return p; };
    l.header = take(HEADER_INTS * 4);
    l.units = take((size_t)l.unit_cap * sizeof(AttnUnit));
    l.merges = take((size_t)l.merge_cap * sizeof(AttnMerge));
    l.group_rows = take((size_t)l.group_row_cap * sizeof(int2));
    l.tiles = take((size_t)(S + groups + 1) * 4);
    l.rows_before = take(groups > 0 ? (size_t)(S + 1) * 4 : 0);
    l.group_of = take(groups > 0 ? (size_t)S * 4 : 0);
    l.group_list = take((size_t)groups * 4);
    l.group_slot = take((size_t)groups * 4);
    l.group_low = take((size_t)groups * 4);
    l.part_ml = take((size_t)l.slot_cap * sizeof(float2));
    l.part_o = take((size_t)l.slot_cap * D * 4);
    l.end = at;
    return l;
}

// Prompts are cut only where they are long on average and their tiles do not fill half the chip: a prompt has tiles by its rows as it has keys, and a
// merge launch with nothing to join costs 4 us of the 10 that a batch of chat-length prompts takes (8 heads over 2 of 128: 4000 rows 66 us, uncut 74; 6000 rows
// 115 uncut, cut 132; 32 heads over 8, 1200 rows: 30 uncut, cut 75).
inline bool prompts_are_cut(int64_t tiles, int64_t kv_heads, int64_t T, int64_t S) { return tiles * kv_heads <= ATTN_TARGET / 2 && T >= 512 * S; }

// Parts have room for the largest heads, so that the other kind's schedule stands in one place: layers whose heads differ in size take the same.
inline Layout prompt_layout(int64_t T, int64_t S, int64_t heads, int64_t kv_heads)
{
    const Layout l = layout_from(HEADER_INTS * 4, 0, T, S, heads, kv_heads, ATTN_MAX_DIM, 0);
    if (!prompts_are_cut(l.tile_cap, kv_heads, T, S)) return l;
    // n tiles of all heads, up to TARGET / 2 of them, and spread = TARGET - n: n + 2 spread = 2 TARGET - n units at most (they are searched for, not listed)
    return layout_from(HEADER_INTS * 4, 2 * ATTN_TARGET * ATTN_COLS, T, S, heads, kv_heads, ATTN_MAX_DIM, 0);
}

// ends where the workspace does
inline Layout cached_layout(int64_t T, int64_t S, int64_t heads, int64_t kv_heads, int64_t D, int64_t groups)
{
    const int64_t cols = T * (heads / kv_heads);
    return layout_from(prompt_layout(T, S, heads, kv_heads).end, 4 * ATTN_TARGET * (cols < ATTN_COLS ? cols : ATTN_COLS), T, S, heads, kv_heads, D, groups);
}

inline AttnLists lists_of(const Layout &l, void *workspace)
{
    char *p = (char *)workspace;
    AttnLists r;
    r.report = (int32_t *)p;
    r.header = (int32_t *)(p + l.header);
    r.units = (AttnUnit *)(p + l.units);
    r.merges = (AttnMerge *)(p + l.merges);
    r.group_rows = (int2 *)(p + l.group_rows);
    r.tiles = (int32_t *)(p + l.tiles);
    r.rows_before = (int32_t *)(p + l.rows_before);
    r.group_of = (int32_t *)(p + l.group_of);
    r.group_list = (int32_t *)(p + l.group_list);
    r.group_slot = (int32_t *)(p + l.group_slot);
    r.group_low = (int32_t *)(p + l.group_low);
    r.part_ml = (float2 *)(p + l.part_ml);
    r.part_o = (float *)(p + l.part_o);
    r.tile_cap = l.tile_cap; r.unit_cap = l.unit_cap; r.merge_cap = l.merge_cap; r.group_row_cap = l.group_row_cap; r.slot_cap = l.slot_cap;
    return r;
}

// so that counts of columns, part columns and workgroups (three a tile and key/value head at most) stay below 2^31
inline bool sizes_fit(int64_t T, int64_t S, int64_t heads, int64_t groups) { return T * heads < (1ll << 28) && S + groups < (1ll << 28); }

// How a call runs: its units found by the workgroups themselves or listed by the schedule kernel, its keys cut into ranges or not, and whether there may be parts to
// join: of keys that are cut, and of rows of groups, whose shared keys are a part of their own whether anything is cut or not.
struct Plan { bool direct, split, merge; int64_t units, tiles; };

// The workgroups that the keys are spread over.  n tiles of about the same work, cut into ranges of 1/spread of it all, make up to n + spread units: no more than run
// side by side where spread = ATTN_TARGET - n (eight decode rows over 8000..30 000 keys: 124 us, spread over all 512 workgroups 147).  Wide tiles are cut no shorter than
// min_wide, fewer key tiles the fewer of them there are; a key tile of f32 takes longer, and counts for four (one prompt of 800 rows, 14 heads: 34 us at 2 key tiles,
// 36 at 4, 60 uncut).
inline void spread(AttnScheduleArgs &s, int dtype)
{
    const int64_t n = (int64_t)s.l.tile_cap * s.kv_heads, least = dtype == PREFT_BF16 ? 2 : 1, wide = dtype == PREFT_BF16 ? n / 8 : n / 32, most = 8 * least;
    s.spread = (int32_t)(n > ATTN_TARGET ? ATTN_TARGET : ATTN_TARGET - n > ATTN_TARGET / 2 ? ATTN_TARGET - n : ATTN_TARGET / 2);
    s.min_tiles = (int32_t)least;
    s.min_wide = (int32_t)(wide > most ? most : wide < least ? least : wide);
}

// A prompt call of T rows: what its schedule goes by.
inline void prompt_rules(AttnScheduleArgs &s, int dtype)
{
    s.max_keys = s.T;
    s.dtype = dtype;
    s.can_split = prompts_are_cut(s.l.tile_cap, s.kv_heads, s.T, s.S);
    spread(s, dtype);
    s.min_tiles = s.min_wide;
}

// A schedule is of one type of pages.
constexpr int32_t ATTN_MX_TYPE = 0x10;

// A call over pages; most_keys: what a row of the block table has room for.
inline void cached_rules(AttnScheduleArgs &s, int dtype, int64_t most_keys)
{
    s.max_keys = (int32_t)(most_keys < (1 << 30) ? most_keys : (1 << 30));
    s.dtype = dtype;
    s.can_split = 1;
    const bool mx = (dtype & ATTN_MX_TYPE) != 0;
    const int64_t n = (int64_t)s.l.tile_cap * s.kv_heads;
    // A second unit on a compute unit takes of the first one's time, and a part has to be written and joined: 16 requests of 40 rows over 1500 tokens, 24 key tiles, 41 us, in two parts 52;
    // over 3000 tokens 70 and 73.  A key tile of f32 queries takes three times as long (20 requests of 20 rows over 1300..2600 tokens: 150, cut 81).
    s.fill = mx && n > ATTN_TARGET / 8 && n < ATTN_TARGET && (int64_t)s.T * s.group > (int64_t)s.S * ATTN_FEW_COLS ? ((dtype & 1) == PREFT_BF16 ? 24 : 8) : 0;
    spread(s, mx ? PREFT_BF16 : dtype);                   // over 4-bit pages the products are bf16's, whatever the queries are
}

// Few segments and workgroups: the schedule kernel's launch is a third of the call (one decode row over 1500 keys: 17.0 us with it, 11.7 without; 40 chat-length
// prompts 12.1 and 7.7); with more than two rounds of workgroups each one's search, about a microsecond, costs as much, and the order by time pays.  For decode rows,
// whose keys are cut one by one then, it does from one round on (64 rows over 4000..16 000 keys: 487 us without the kernel, 468 with it).
// The workgroups sum the work of all tiles in 31 bits: where tables are so long that it may not fit, the schedule kernel does it in 64.
// Keys are cut where the tiles alone do not fill the chip and some tile may be longer than a range.
inline Plan plan_of(const AttnScheduleArgs &s)
{
    Plan p;
    const int64_t key_tiles = ((int64_t)s.max_keys + ATTN_KEYS - 1) / ATTN_KEYS;
    p.tiles = s.l.tile_cap;
    const bool narrow = (int64_t)s.T * s.group <= (int64_t)s.S * ATTN_FEW_COLS;
    p.split = s.can_split && key_tiles > 2 * s.min_tiles;
    p.merge = p.split || s.n_groups > 0;
    p.direct = s.n_groups == 0 && s.S <= ATTN_DIRECT && p.tiles * s.kv_heads <= (narrow && s.can_split ? 1 : 2) * ATTN_TARGET &&
               p.tiles * (key_tiles + 1) <= INT32_MAX;
    const int64_t ranges = (ATTN_TARGET + s.kv_heads - 1) / s.kv_heads;
    p.units = !p.split ? p.tiles : p.direct ? p.tiles + 2 * ranges + 2 : 3 * p.tiles + ranges + 2;
    const int64_t most = p.tiles * ((key_tiles + s.min_tiles - 1) / s.min_tiles);
    if (p.split && p.units > most) p.units = most;
    return p;
}

// One workgroup: a thread for every item or tile, as far as there are.
inline int schedule_threads(const AttnScheduleArgs &s)
{
    const int64_t items = (int64_t)s.S + s.n_groups, n = items > s.l.tile_cap ? items : s.l.tile_cap;
    return n >= SCHED_THREADS ? SCHED_THREADS : n <= 256 ? 256 : (int)((n + 63) / 64 * 64);
}

}  // namespace preft
