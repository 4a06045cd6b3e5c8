// Schedule of an attention call: segment tables -> work units (a tile of query columns and a range of keys) and merges.
//
// The columns of a segment are its (row, query head of the key/value head) pairs, column c = row * G + head: G query heads share every key that is
// read, and a decode row fills G columns of a tile instead of one.  Units are cut into tiles of 128 columns, and along the keys into ranges of
// about total / TARGET each where there are too few tiles to fill the chip; the ranges' parts are joined by the merge kernel.
// Rows of a group see their shared first keys through units of the group, which carry the rows of all its members.
#pragma once
#include "common.hpp"
#include "block_scan.hpp"

namespace preft {

constexpr int ATTN_COLS      = 128;   // columns of a unit (four wavefronts of 32)
constexpr int ATTN_FEW_COLS  = 32;    // up to here the four wavefronts of a unit share the keys instead
constexpr int ATTN_KEYS      = 64;    // keys of a tile
constexpr int ATTN_MAX_DIM   = 128;   // largest head size
constexpr int ATTN_TARGET    = 512;   // workgroups that run side by side: two on each of 256 compute units
constexpr int ATTN_GROUP_ROWS = 4096; // rows of groups that are listed; the rest see their prefix by themselves
constexpr int ATTN_MIN_PREFIX = 64;   // shorter prefixes are not worth a part of their own
constexpr int ATTN_SHORT     = 12;    // key tiles: up to here a unit of few columns is one wavefront's, where there are many of them
constexpr int ATTN_SCAN      = 4096;  // items whose tile offsets are kept in LDS
constexpr int ATTN_DIRECT    = 256;   // segments of a call whose workgroups find their unit by themselves, four a lane

struct AttnUnit {
    int32_t table;     // row of the block table; packed keys: the row of key 0
    int32_t head0;     // column c of the unit is query head (head0 + c) % G of row (head0 + c) / G
    int32_t ncols;     // 1..ATTN_COLS
    int32_t key0, key1;
    int32_t row0;      // batch row of the unit's row 0, the next ones follow; a group: -1 - (its entry in the row list)
    int32_t lim0;      // row i sees keys below lim0 + i; a group: every row sees those below
    int32_t slot;      // first part column, head-major; -1: the unit writes the result
};
struct AttnMerge {
    int32_t row0, col0, ncols;
    int32_t parts, slot;                                   // of the segment's own keys
    int32_t group_parts, group_slot, group_col0, group_cols;
    int32_t pad[3];
};

struct AttnLists {
    int32_t   *report;     // what preft_schedule_counts reads: units, joined tiles and tiles of the last schedule, and the marks of refused calls
    int32_t   *header;     // HEADER_INTS ints of this kind of call
    AttnUnit  *units;
    AttnMerge *merges;
    int2      *group_rows; // {batch row, keys it sees}
    int32_t   *tiles;      // [S + groups + 1] first column tile of every item
    int32_t   *rows_before;// [S + 1]
    int32_t   *group_of;   // [S]
    int32_t   *group_list; // [groups] first entry in group_rows, or -1
    int32_t   *group_slot; // [groups] first part column of the group's units
    int32_t   *group_low;  // [groups] keys that all of the group's rows see
    float     *part_o;     // [slots][head_dim]
    float2    *part_ml;    // [slots] {largest exponent, sum}
    int32_t    tile_cap, unit_cap, merge_cap, group_row_cap, slot_cap;
};

constexpr int AH_UNITS = 0, AH_MERGES = 1, AH_TILES = 2, AH_KIND = 3, AH_GROUPS = 4, AH_T = 5, AH_S = 6, AH_HEADS = 7, AH_DTYPE = 8, AH_KV_HEADS = 9, AH_SHORT = 10, AH_JOINS = 11, AH_KEYS = 12;      // AH_SHORT: first unit that is one wavefront's; AH_JOINS: entries of merges

struct AttnScheduleArgs {
    const int32_t *seg_start, *seg_prefill_len;            // seg_prefill_len may be null in a cached call
    const int32_t *kv_len;                                 // null: packed whole prompts
    const int32_t *group_start, *group_prefix;
    int32_t S, T, n_groups, heads, kv_heads, group, max_keys, dtype, can_split, min_tiles, min_wide, spread;    // group: heads / kv_heads; spread: workgroups that a range's length is meant for
    AttnLists l;
};

struct AttnItem { int32_t row0, rows, lim0, key0, key1; };

// Entry i of a table of offsets, each cut to 0..most, and the next: does it go back?  Where none does, segments (and groups) are disjoint, and every bound on lists,
// sums and grids follows from T and S; a call with an offset that goes back has no units.  All other entries of the tables are cut to what exists.
__device__ __forceinline__ bool goes_back_at(const int32_t *start, int32_t i, int32_t most) { return max(0, min(start[i + 1], most)) < max(0, min(start[i], most)); }

__device__ __forceinline__ AttnItem attn_segment(const AttnScheduleArgs &a, int32_t s)
{
    AttnItem r;
    const int32_t lo = max(0, min(a.seg_start[s], a.T)), hi = max(lo, min(a.seg_start[s + 1], a.T));
    const int32_t prompt = a.seg_prefill_len ? max(0, min(a.seg_prefill_len[s], hi - lo)) : 0;
    if (a.kv_len) {
        const int32_t kv = max(0, min(a.kv_len[s], a.max_keys));
        r.row0 = lo + prompt;
        r.rows = hi - r.row0;
        r.lim0 = kv - r.rows + 1;
        r.key1 = kv;
    } else {
        r.row0 = lo;
        r.rows = prompt;
        r.lim0 = 1;
        r.key1 = prompt;
    }
    r.key0 = 0;
    return r;
}

__device__ __forceinline__ int32_t key_tiles(int32_t key0, int32_t key1) { return key1 > key0 ? (key1 - 1) / ATTN_KEYS - key0 / ATTN_KEYS + 1 : 0; }

// A part of a wide tile is 64 KB written and read again, which on a full chip takes the time of some 14 key tiles: cut only where tiles are few, or this one long.
// (16 requests of 40 rows over 100..2000 tokens: 56 us, cut by `range` 85; one prompt of 900 rows 23 us, cut by 8 key tiles 37; of 2000 rows and 8 heads 33 us cut by 8, uncut 40.)
__device__ __forceinline__ int32_t wide_range(const AttnScheduleArgs &a, int32_t range)
{
    return max(a.min_wide, a.spread <= ATTN_TARGET / 2 ? min(range, INT32_MAX / 2) * 2 : range);
}
__device__ __forceinline__ int32_t ranges_of(int32_t tiles, int32_t range) { return tiles > range ? (int32_t)((uint32_t)(tiles - 1) / (uint32_t)range) + 1 : 1; }
// where part k of `parts` of n tiles begins: the first n % parts have one more
__device__ __forceinline__ int32_t part_begin(int32_t n, int32_t parts, int32_t k)
{
    const int32_t each = (int32_t)((uint32_t)n / (uint32_t)parts);
    return each * k + min(k, n - each * parts);
}

// what a later call and the join go by; joined: tiles of more than one part
__device__ __forceinline__ void attn_header(const AttnScheduleArgs &a, int32_t units, int32_t alone, int32_t tiles, int32_t joined, int32_t joins)
{
    int32_t *h = a.l.header, *r = a.l.report;
    const int32_t kind = a.kv_len ? 2 : 1;
    r[AH_UNITS] = units; r[AH_MERGES] = joined; r[AH_TILES] = tiles; r[HDR_ALL] = ATTN_REPORT; r[ATTN_MARKS + kind] = 0;
    h[AH_UNITS] = units; h[AH_SHORT] = alone; h[AH_TILES] = tiles; h[AH_MERGES] = joined; h[AH_JOINS] = joins;
    h[AH_KIND] = kind; h[AH_DTYPE] = a.dtype; h[AH_KEYS] = a.max_keys; h[AH_GROUPS] = a.n_groups; h[AH_T] = a.T; h[AH_S] = a.S; h[AH_HEADS] = a.heads; h[AH_KV_HEADS] = a.kv_heads;
}

// Whether the header's schedule is that of a call with these sizes.  The type and the room of the block table are among them: ranges, and with them the grid and
// whether parts are joined, go by both.  Compared as a whole: behind && it would be a chain of trips to memory.
__device__ __forceinline__ bool attn_schedule_fits(const AttnScheduleArgs &a)
{
    const PREFT_CONST int32_t *h = as_const(a.l.header);
    return ((h[AH_KIND] ^ (a.kv_len ? 2 : 1)) | (h[AH_GROUPS] ^ a.n_groups) | (h[AH_T] ^ a.T) | (h[AH_S] ^ a.S) | (h[AH_HEADS] ^ a.heads) | (h[AH_DTYPE] ^ a.dtype) |
            (h[AH_KV_HEADS] ^ a.kv_heads) | (h[AH_KEYS] ^ a.max_keys)) == 0;
}

struct AttnGroup { int32_t begin, end, rows, prefix; };

__device__ __forceinline__ AttnGroup attn_group(const AttnScheduleArgs &a, int32_t g)
{
    AttnGroup m;
    m.begin = max(0, min(a.group_start[g], a.S));
    m.end = max(m.begin, min(a.group_start[g + 1], a.S));
    m.rows = a.l.rows_before[m.end] - a.l.rows_before[m.begin];
    m.prefix = max(0, min(a.group_prefix[g], a.max_keys));
    return m;
}

// last i of [0, n) with first[i] <= x; first[0] <= x
template <typename P>
__device__ __forceinline__ int32_t last_at_or_before(P first, int32_t n, int32_t x)
{
    int32_t lo = 0, hi = n;
    while (hi - lo > 1) {
        const int32_t mid = (lo + hi) >> 1;
        if (first[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}

// One workgroup: the lists are a few kilobytes, and what a step waits for is the chain of reads and barriers, not the work.
// Units stand in the order of falling time (counting sort over 256 classes): the longest of a causal prompt begin first and the short ones fill the ends.
// (Wide units, bound by the matrix cores, and narrow ones, bound by memory, in turns, so that a compute unit has one of each: 229 us against 187 on 256 rows of
// 64 heads with prefixes of 8192 -- the wide ones then end late.)  Their order does not change a result: every unit has an output or part of its own.
__global__ __launch_bounds__(SCHED_THREADS) void attn_schedule_kernel(AttnScheduleArgs a)
{
    __shared__ int32_t lds[32];
    __shared__ int32_t first_tile[ATTN_SCAN + 1];
    __shared__ int32_t bins[512];
    __shared__ int32_t n_units, n_long, n_merges, n_slots, goes_back;
    __shared__ unsigned long long cost_sum;
    const int tid = threadIdx.x, nt = blockDim.x;
    const int32_t G = a.group, items = a.S + a.n_groups;
    const bool in_lds = items <= ATTN_SCAN;
    if (tid == 0) { n_merges = 0; n_slots = 0; cost_sum = 0; goes_back = 0; }
    for (int b = tid; b < 512; b += nt) bins[b] = 0;
    // Whether offsets go back is known after the first loop over them; its sums wrap where they do.  All threads then leave: true for them all.
    bool back = false;
    auto nothing_to_run = [&]() {
        if (back) goes_back = 1;                           // set to 0 before a barrier of the loop
        __syncthreads();
        if (goes_back && tid == 0) attn_header(a, 0, 0, 0, 0, 0);
        return goes_back != 0;
    };

    // groups: how many rows each has, and where they stand in the row list
    if (a.n_groups > 0) {
        uint32_t rows_carry = 0;
        for (int32_t s0 = 0; s0 < a.S; s0 += nt) {
            const int32_t s = s0 + tid;
            int32_t total;
            const int32_t rows = s < a.S ? attn_segment(a, s).rows : 0;
            back = back || (s < a.S && goes_back_at(a.seg_start, s, a.T));
            const int32_t before = block_exclusive_scan(rows, lds, &total);
            if (s < a.S) a.l.rows_before[s] = (int32_t)(rows_carry + (uint32_t)before);
            rows_carry += (uint32_t)total;
        }
        if (tid == 0) a.l.rows_before[a.S] = (int32_t)rows_carry;
        for (int32_t g = tid; g < a.n_groups; g += nt) back = back || goes_back_at(a.group_start, g, a.S);
        if (nothing_to_run()) return;
        int32_t carry = 0;
        for (int32_t g0 = 0; g0 < a.n_groups; g0 += nt) {
            const int32_t g = g0 + tid;
            int32_t rows = 0, total;
            if (g < a.n_groups) {
                const AttnGroup m = attn_group(a, g);
                rows = m.prefix >= ATTN_MIN_PREFIX && m.rows >= 2 ? m.rows : 0;
            }
            const int32_t before = block_exclusive_scan(rows, lds, &total);
            const int64_t end = (int64_t)carry + before + rows;
            if (g < a.n_groups) {
                a.l.group_list[g] = rows > 0 && end <= a.l.group_row_cap ? carry + before : -1;
                a.l.group_low[g] = max(0, min(a.group_prefix[g], a.max_keys));
            }
            carry = (int32_t)min((int64_t)INT32_MAX / 2, (int64_t)carry + total);
        }
        __syncthreads();
    }

    // items: column tiles, and the work of all
    uint32_t carry = 0;
    unsigned long long cost = 0;
    for (int32_t i0 = 0; i0 < items; i0 += nt) {
        const int32_t i = i0 + tid;
        int32_t tiles = 0, total;
        if (i < a.S) {
            AttnItem it = attn_segment(a, i);
            back = back || goes_back_at(a.seg_start, i, a.T);
            if (a.n_groups > 0) {
                const int32_t g = last_at_or_before(a.group_start, a.n_groups, i);
                const AttnGroup m = attn_group(a, g);
                const bool in = m.begin <= i && i < m.end && a.l.group_list[g] >= 0;
                a.l.group_of[i] = in ? g : -1;
                if (in) {
                    const int32_t at = a.l.group_list[g] + a.l.rows_before[i] - a.l.rows_before[m.begin];
                    for (int32_t r = 0; r < it.rows; ++r)
                        if (at + r < a.l.group_row_cap) a.l.group_rows[at + r] = make_int2(it.row0 + r, min(it.lim0 + r, m.prefix));
                    if (it.rows > 0 && it.lim0 < m.prefix) atomicMin(&a.l.group_low[g], it.lim0);
                    it.key0 = m.prefix;
                }
            }
            tiles = it.rows > 0 ? (int32_t)(((int64_t)it.rows * G + ATTN_COLS - 1) / ATTN_COLS) : 0;
            // a causal prompt: tiles see half of the keys on average
            if (tiles > 0) {
                const int32_t low = min(it.key1, it.lim0 + (int32_t)(min((int64_t)it.rows * G, (int64_t)ATTN_COLS) - 1) / G);
                cost += (unsigned long long)tiles * (unsigned)(key_tiles(it.key0, low) + key_tiles(it.key0, it.key1) + 1) / 2;
            }
        } else if (i < items) {
            const int32_t g = i - a.S;
            if (a.l.group_list[g] >= 0) {
                const AttnGroup m = attn_group(a, g);
                tiles = (int32_t)(((int64_t)m.rows * G + ATTN_COLS - 1) / ATTN_COLS);
                cost += (unsigned long long)tiles * (unsigned)key_tiles(0, m.prefix);
            }
        }
        const int32_t before = block_exclusive_scan(tiles, lds, &total);
        if (i < items) {
            const int32_t first = (int32_t)(carry + (uint32_t)before);
            if (in_lds) first_tile[i] = first;
            else a.l.tiles[i] = first;
        }
        carry += (uint32_t)total;
    }
    for (int off = 32; off > 0; off >>= 1) cost += __shfl_xor(cost, off, 64);
    if ((tid & 63) == 0) atomicAdd(&cost_sum, cost);
    if (nothing_to_run()) return;
    const int32_t n_tiles = min((int32_t)carry, a.l.tile_cap);
    // a range of keys: no shorter than the whole work over the workgroups it is meant for
    // (Wide and narrow tiles each for themselves: 206 us against 173 on 256 rows of 64 heads with prefixes of 8192.  All workgroups are wide ones then at first, and memory
    // waits for the narrow ones.)
    int32_t range = INT32_MAX;
    if (a.can_split) {
        const unsigned long long even = (cost_sum * (unsigned)a.kv_heads + a.spread - 1) / (unsigned)a.spread;
        range = max(a.min_tiles, (int32_t)min(even, (unsigned long long)INT32_MAX));
    }
    if (a.n_groups > 0) {                                  // a group's parts stand together, tile by tile: its members find them by their columns
        int64_t base = 0;
        for (int32_t g0 = 0; g0 < a.n_groups; g0 += nt) {
            const int32_t g = g0 + tid;
            int64_t need = 0;
            if (g < a.n_groups && a.l.group_list[g] >= 0) {
                const AttnGroup m = attn_group(a, g);
                need = (int64_t)m.rows * G * a.kv_heads * ranges_of(key_tiles(0, m.prefix), range);
            }
            int32_t total;
            const int32_t before = block_exclusive_scan((int32_t)min(need, (int64_t)a.l.slot_cap), lds, &total);
            if (g < a.n_groups) a.l.group_slot[g] = (int32_t)min(base + before, (int64_t)INT32_MAX / 2);
            base += total;
        }
        if (tid == 0) n_slots = (int32_t)min(base, (int64_t)INT32_MAX / 2);
        __syncthreads();
    }

    struct Tile {
        AttnUnit u;
        int32_t n, splits, cls, key0, key1, group_ranges, col0, rows0, i, g, begin, group_cols;
        bool parts;
    };
    auto describe = [&](int32_t t) {
        Tile d;
        const int32_t i = in_lds ? last_at_or_before(first_tile, items, t) : last_at_or_before(a.l.tiles, items, t);
        const int32_t tile = t - (in_lds ? first_tile[i] : a.l.tiles[i]);
        AttnItem it;
        AttnGroup m = {0, 0, 0, 0};
        d.i = i; d.g = -1; d.group_ranges = 0;
        if (i < a.S) {
            it = attn_segment(a, i);
            if (a.n_groups > 0) d.g = a.l.group_of[i];
            if (d.g >= 0) {
                m = attn_group(a, d.g);
                it.key0 = m.prefix;
                d.group_ranges = ranges_of(key_tiles(0, m.prefix), range);
            }
            d.u.table = a.kv_len ? i : it.row0;
        } else {
            m = attn_group(a, i - a.S);
            it.row0 = 0; it.rows = m.rows; it.key0 = 0; it.key1 = m.prefix;
            d.u.table = min(m.begin, a.S - 1);
        }
        d.begin = m.begin; d.group_cols = m.rows * G;
        d.col0 = tile * ATTN_COLS;
        d.rows0 = it.row0;
        const int32_t first = d.col0 / G;
        d.u.ncols = min(ATTN_COLS, it.rows * G - d.col0);
        d.u.head0 = d.col0 - first * G;
        d.key0 = it.key0; d.key1 = it.key1;
        if (i < a.S) {
            d.u.row0 = it.row0 + first;
            d.u.lim0 = it.lim0 + first;
            d.key1 = min(d.key1, d.u.lim0 + (d.u.head0 + d.u.ncols - 1) / G);
        } else {
            d.u.row0 = -1 - (a.l.group_list[i - a.S] + first);
            d.u.lim0 = __hip_atomic_load(&a.l.group_low[i - a.S], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        d.n = key_tiles(d.key0, d.key1);
        d.splits = d.n == 0 && d.g >= 0 ? 0 : ranges_of(d.n, i < a.S && d.u.ncols > ATTN_FEW_COLS ? wide_range(a, range) : range);      // 0: the group's part is all there is
        d.parts = d.splits > 1 || d.g >= 0 || i >= a.S;
        const int32_t each = d.splits > 0 ? (int32_t)((uint32_t)d.n / (uint32_t)d.splits) : 0;
        // by time: 64 keys of a wide unit take 2.5 times those of a narrow one; short units stand at the end
        const bool narrow = d.u.ncols <= ATTN_FEW_COLS, brief = narrow && each <= ATTN_SHORT;
        const int32_t time = narrow && !brief ? each * 2 / 5 : each;
        d.cls = (brief ? 256 : 0) + 255 - (time < 128 ? time : min(255, 128 + (time - 128) / 16));
        return d;
    };
    Tile d;
    for (int32_t t = tid; t < n_tiles; t += nt) {
        d = describe(t);
        if (d.splits > 0) atomicAdd(&bins[d.cls], d.splits);
    }
    __syncthreads();
    {
        int32_t total;
        const int32_t v0 = tid < 256 ? bins[2 * tid] : 0, v1 = tid < 256 ? bins[2 * tid + 1] : 0;
        const int32_t before = block_exclusive_scan(v0 + v1, lds, &total);
        if (tid < 256) { bins[2 * tid] = before; bins[2 * tid + 1] = before + v0; }
        if (tid == 0) n_units = total;
        if (tid == 128) n_long = before;
        __syncthreads();
    }
    for (int32_t t = tid; t < n_tiles; t += nt) {
        if (n_tiles > nt) d = describe(t);                     // else every thread has its only one still
        const int32_t at = d.splits > 0 ? atomicAdd(&bins[d.cls], d.splits) : 0, step = d.u.ncols * a.kv_heads;
        int32_t slot = -1;
        if (d.i >= a.S) slot = a.l.group_slot[d.i - a.S] + d.col0 * a.kv_heads * d.splits;
        else if (d.parts) slot = atomicAdd(&n_slots, d.splits * step);
        const bool fits = !d.parts || (slot >= 0 && (int64_t)slot + (int64_t)d.splits * step <= a.l.slot_cap);   // always so: the bounds in attention_plan.hpp
        const int32_t first = d.key0 / ATTN_KEYS;
        for (int32_t k = 0; k < d.splits; ++k) {
            AttnUnit u = d.u;
            const int64_t k0 = first + part_begin(d.n, d.splits, k), k1 = first + part_begin(d.n, d.splits, k + 1);
            u.key0 = max(d.key0, (int32_t)(k0 * ATTN_KEYS));
            u.key1 = max(u.key0, (int32_t)min((int64_t)d.key1, k1 * ATTN_KEYS));
            u.slot = d.parts ? slot + k * step : -1;
            if (!fits) { u.slot = 0; u.ncols = 0; }
            if (at + k < a.l.unit_cap) a.l.units[at + k] = u;
        }
        if (d.parts && d.i < a.S && fits) {
            AttnMerge j;
            j.row0 = d.rows0; j.col0 = d.col0; j.ncols = d.u.ncols; j.parts = d.splits; j.slot = slot;
            j.group_parts = d.group_ranges; j.group_slot = d.g >= 0 ? a.l.group_slot[d.g] : 0;
            j.group_col0 = d.g >= 0 ? (a.l.rows_before[d.i] - a.l.rows_before[d.begin]) * G + d.col0 : 0;
            j.group_cols = d.group_cols;
            j.pad[0] = j.pad[1] = j.pad[2] = 0;
            const int32_t to = atomicAdd(&n_merges, 1);
            if (to < a.l.merge_cap) a.l.merges[to] = j;
        }
    }
    __syncthreads();
    if (tid == 0) {
        const int32_t units = min(n_units, a.l.unit_cap), joins = min(n_merges, a.l.merge_cap);
        // enough short ones that a wavefront each fills the chip: 2048 wavefronts run side by side
        attn_header(a, units, (units - n_long) * a.kv_heads >= 2 * ATTN_TARGET ? min(n_long, units) : units, n_tiles, joins, joins);
    }
}

// ---------------------------------------------------------------------------------------
// Without a schedule kernel: a wavefront finds the unit of its workgroup from the tables by itself, in a microsecond where the
// kernel would take six, and the first unit of a tile leaves the entry of its merge.  For calls of few segments and workgroups, without groups.  All tiles of a segment are cut into as many ranges, so that the sums over the
// segments before are all it takes.
// ---------------------------------------------------------------------------------------
struct AttnDirect {
    AttnItem it;
    int32_t s, tile, part, parts;      // parts 1: the unit writes the result
    int32_t tiles_before;              // of the segments before
    int32_t slot;                      // first part column of the segment
    int32_t units, tiles, joined;      // of the call, for index 0
    bool found;
};

// inclusive sums over the lanes, of which only the first `n` hold anything (a step of a few requests does not wait for six exchanges)
__device__ __forceinline__ int32_t wave_inclusive(int32_t v, int32_t n)
{
    const int lane = threadIdx.x & 63;
    for (int off = 1; off < n; off <<= 1) {
        const int32_t up = __shfl_up(v, off, 64);
        if (lane >= off) v += up;
    }
    return v;
}

// the unit `index` of the call
__device__ __forceinline__ AttnDirect attn_direct(const AttnScheduleArgs &a, int32_t index)
{
    constexpr int EACH = ATTN_DIRECT / 64;
    const int lane = threadIdx.x & 63, G = a.group;
    AttnItem it[EACH];
    int32_t tiles[EACH];
    uint32_t cost = 0;
    bool back = false;
#pragma unroll
    for (int c = 0; c < EACH; ++c) {
        it[c] = AttnItem{0, 0, 0, 0, 0};
        tiles[c] = 0;
        if (c * 64 >= a.S) continue;
        const int32_t s = c * 64 + lane;
        if (s < a.S) {
            it[c] = attn_segment(a, s);
            back = back || goes_back_at(a.seg_start, s, a.T);
        }
        tiles[c] = (it[c].rows * G + ATTN_COLS - 1) / ATTN_COLS;
        if (tiles[c] > 0) {
            const int32_t low = min(it[c].key1, it[c].lim0 + (min(it[c].rows * G, ATTN_COLS) - 1) / G);
            cost += (uint32_t)(((int64_t)tiles[c] * (key_tiles(0, low) + key_tiles(0, it[c].key1) + 1)) / 2);      // all of them fit 31 bits: plan_of
        }
    }
    AttnDirect r = {};
    if (__any(back)) return r;
    int32_t range = INT32_MAX;
    if (a.can_split) {
        const int32_t n = min(a.S, 64);
        cost = (uint32_t)__builtin_amdgcn_readlane(wave_inclusive((int32_t)cost, n), n - 1);
        range = max(a.min_tiles, (int32_t)min(((uint64_t)cost * (uint32_t)a.kv_heads + a.spread - 1) / (uint32_t)a.spread, (uint64_t)INT32_MAX));
    }
    int32_t before = 0, slots = 0, tiles_before = 0;
#pragma unroll
    for (int c = 0; c < EACH; ++c) {
        if (c * 64 >= a.S) continue;
        const int32_t parts = ranges_of(key_tiles(0, it[c].key1), it[c].rows * G > ATTN_FEW_COLS ? wide_range(a, range) : range), units = tiles[c] * parts;
        const int32_t need = parts > 1 ? (int32_t)min((int64_t)it[c].rows * G * parts * a.kv_heads, (int64_t)a.l.slot_cap) : 0;
        const int32_t lanes = min(a.S - c * 64, 64);
        const int32_t upto = wave_inclusive(units, lanes), slot = a.can_split ? wave_inclusive(need, lanes) : 0;
        const int32_t tile = a.can_split ? wave_inclusive(tiles[c], lanes) : upto;
        const uint64_t past = __ballot(lane < lanes && before + upto > index);
        if (!r.found && past != 0) {
            const int at = __builtin_ctzll(past);
            auto of = [&](int32_t v) { return __builtin_amdgcn_readlane(v, at); };
            const int32_t i = index - before - (of(upto) - of(units));
            r.found = true;
            r.s = c * 64 + at;
            r.it.row0 = of(it[c].row0); r.it.rows = of(it[c].rows); r.it.lim0 = of(it[c].lim0); r.it.key0 = 0; r.it.key1 = of(it[c].key1);
            r.parts = of(parts);
            r.tile = r.parts == 1 ? i : (int32_t)((uint32_t)i / (uint32_t)r.parts);
            r.part = i - r.tile * r.parts;
            r.tiles_before = tiles_before + of(tile) - of(tiles[c]);
            r.slot = slots + of(slot) - of(need);
        }
        before += __builtin_amdgcn_readlane(upto, lanes - 1);
        slots += __builtin_amdgcn_readlane(slot, lanes - 1);
        tiles_before += __builtin_amdgcn_readlane(tile, lanes - 1);
        if (index == 0) {
            r.joined += __builtin_amdgcn_readlane(wave_inclusive(parts > 1 ? tiles[c] : 0, lanes), lanes - 1);
        }
    }
    r.units = before;
    r.tiles = tiles_before;
    return r;
}

__device__ __forceinline__ AttnUnit attn_unit_of(const AttnScheduleArgs &a, const AttnDirect &d)
{
    const int32_t G = a.group;
    AttnUnit u;
    // the last tile of a causal prompt sees the most keys: it begins first
    const int32_t tiles = (d.it.rows * G + ATTN_COLS - 1) / ATTN_COLS, tile = tiles - 1 - d.tile;
    const int32_t col0 = tile * ATTN_COLS, first = col0 / G;
    u.table = a.kv_len ? d.s : d.it.row0;
    u.ncols = min(ATTN_COLS, d.it.rows * G - col0);
    u.head0 = col0 - first * G;
    u.row0 = d.it.row0 + first;
    u.lim0 = d.it.lim0 + first;
    const int32_t key1 = min(d.it.key1, u.lim0 + (u.head0 + u.ncols - 1) / G), n = key_tiles(0, key1);
    const int32_t k0 = part_begin(n, d.parts, d.part), k1 = part_begin(n, d.parts, d.part + 1);
    u.key0 = k0 * ATTN_KEYS;
    u.key1 = max(u.key0, (int32_t)min((int64_t)key1, (int64_t)k1 * ATTN_KEYS));
    u.slot = -1;
    if (d.parts > 1) {
        u.slot = d.slot + col0 * d.parts * a.kv_heads + d.part * u.ncols * a.kv_heads;
        if (u.slot < 0 || (int64_t)u.slot + (int64_t)u.ncols * a.kv_heads > a.l.slot_cap) u.ncols = 0;      // never so: the bounds in attention_plan.hpp
    }
    return u;
}

// The unit that a workgroup of a direct call finds; false: none.  The first workgroup leaves the header that a later call asks for, unless it is there already (`ready`), and
// a tile's first unit the entry of its merge.
__device__ __forceinline__ bool attn_direct_unit(const AttnScheduleArgs &a, int32_t unit, int32_t kv_head, bool ready, AttnUnit &u)
{
    const AttnDirect d = attn_direct(a, unit);
    if (!ready && unit == 0 && kv_head == 0 && threadIdx.x == 0) attn_header(a, d.units, d.units, d.tiles, d.joined, min(d.tiles, a.l.merge_cap));
    if (!d.found) return false;
    u = attn_unit_of(a, d);
    if (a.can_split && d.part == 0 && kv_head == 0 && threadIdx.x == 0) {
        const int32_t tile = (d.it.rows * a.group + ATTN_COLS - 1) / ATTN_COLS - 1 - d.tile, to = d.tiles_before + tile;
        AttnMerge j = {};
        j.row0 = d.it.row0; j.col0 = tile * ATTN_COLS; j.ncols = u.ncols; j.group_cols = ATTN_COLS;
        j.parts = d.parts > 1 ? d.parts : 0;
        j.slot = d.slot + j.col0 * d.parts * a.kv_heads;
        if (to < a.l.merge_cap) a.l.merges[to] = j;
    }
    return true;
}

}  // namespace preft
