// C entry points of attention: argument checks, the layout of the workspace, launches.  See include/preft.h for the contract.
#include "../../include/preft.h"

#include "attention_common.hpp"
#include "attention_kernel.hpp"

#include <cmath>

namespace {

using namespace preft;

// Bounds on the lists, for tables that are well-formed:
//   column tiles   T G / 128 + one part-filled tile a segment, and the same of groups;
//   units          a tile of n key tiles is cut into ceil(n / range) < 1 + n / range ranges, and range is at least the estimate of all tiles' n times
//                  kv_heads / TARGET.  That estimate, from the first and the last tile of a segment, is short by up to two a tile of a causal prompt (list), and
//                  at least half of what counting every tile of a segment like its last gives (direct);
//   part columns   a tile that is cut has at most twice n / range parts of at most 128 columns; rows of groups have one of their own and their group's.
struct Layout {
    int32_t tile_cap, unit_cap, merge_cap, group_row_cap, slot_cap;
    size_t units, merges, group_rows, tiles, rows_before, group_of, group_list, group_slot, group_low, part_ml, part_o, bytes;
};

Layout layout_of(int64_t T, int64_t S, int64_t heads, int64_t kv_heads, int64_t D, int64_t groups)
{
    Layout l;
    const int64_t G = heads / kv_heads, cols = T * G;
    const int64_t seg_tiles = cols / ATTN_COLS + (S < T ? S : T);
    const int64_t tiles = groups > 0 ? 2 * seg_tiles + groups : seg_tiles;
    l.tile_cap = (int32_t)tiles;
    l.unit_cap = (int32_t)(3 * tiles + 2 * ((ATTN_TARGET + kv_heads - 1) / kv_heads) + 2);
    l.merge_cap = (int32_t)seg_tiles;
    l.group_row_cap = groups > 0 ? (int32_t)(T < ATTN_GROUP_ROWS ? T : ATTN_GROUP_ROWS) : 0;
    l.slot_cap = (int32_t)(4 * ATTN_TARGET * (cols < ATTN_COLS ? cols : ATTN_COLS) + 2 * l.group_row_cap * heads);
    size_t at = HEADER_INTS * 4;
    auto take = [&](size_t bytes) { const size_t p = at; at = (at + bytes + 63) & ~(size_t)63; return p; };
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
    l.bytes = at;
    return l;
}

AttnLists lists_of(const Layout &l, void *workspace)
{
    char *p = (char *)workspace;
    AttnLists r;
    r.header = (int32_t *)p;
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
bool sizes_fit(int64_t T, int64_t S, int64_t heads, int64_t groups) { return T * heads < (1ll << 28) && S + groups < (1ll << 28); }

// How a call runs: its units found by the workgroups themselves or listed by the schedule kernel, its keys cut into ranges or not.
struct Plan { bool direct, split; int64_t units, tiles; };

// The workgroups that the keys are spread over.  n tiles of about the same work, cut into ranges of 1/spread of it all, make up to n + spread units: no more than run
// side by side where spread = ATTN_TARGET - n (eight decode rows over 8000..30 000 keys: 124 us, spread over all 512 workgroups 147).  Wide tiles are cut no shorter than
// min_wide, fewer key tiles the fewer of them there are; a key tile of f32 takes longer, and counts for four (one prompt of 800 rows, 14 heads: 34 us at 2 key tiles,
// 36 at 4, 60 uncut).
void spread(AttnScheduleArgs &s, int dtype)
{
    const int64_t n = (int64_t)s.l.tile_cap * s.kv_heads, least = dtype == PREFT_BF16 ? 2 : 1, wide = dtype == PREFT_BF16 ? n / 8 : n / 32, most = 8 * least;
    s.spread = (int32_t)(n > ATTN_TARGET ? ATTN_TARGET : ATTN_TARGET - n > ATTN_TARGET / 2 ? ATTN_TARGET - n : ATTN_TARGET / 2);
    s.min_tiles = (int32_t)least;
    s.min_wide = (int32_t)(wide > most ? most : wide < least ? least : wide);
}

// Few segments and workgroups: the schedule kernel's launch is a third of the call (one decode row over 1500 keys: 17.0 us with it, 11.7 without; 40 chat-length
// prompts 12.1 and 7.7); with more than two rounds of workgroups each one's search, about a microsecond, costs as much, and the order by time pays.  For decode rows,
// whose keys are cut one by one then, it does from one round on (64 rows over 4000..16 000 keys: 487 us without the kernel, 468 with it).
// Keys are cut where the tiles alone do not fill the chip and some tile may be longer than a range.
Plan plan_of(const AttnScheduleArgs &s, int64_t most_keys)
{
    Plan p;
    const int64_t key_tiles = (most_keys + ATTN_KEYS - 1) / ATTN_KEYS;
    p.tiles = s.l.tile_cap;
    const bool narrow = (int64_t)s.T * s.group <= (int64_t)s.S * ATTN_FEW_COLS;
    p.split = s.can_split && key_tiles > 2 * s.min_tiles;
    p.direct = s.n_groups == 0 && s.S <= ATTN_DIRECT && p.tiles * s.kv_heads <= (narrow && s.can_split ? 1 : 2) * ATTN_TARGET;
    const int64_t ranges = (ATTN_TARGET + s.kv_heads - 1) / s.kv_heads;
    p.units = !p.split ? p.tiles : p.direct ? p.tiles + 2 * ranges + 2 : 3 * p.tiles + ranges + 2;
    const int64_t most = p.tiles * ((key_tiles + s.min_tiles - 1) / s.min_tiles);
    if (p.split && p.units > most) p.units = most;
    return p;
}

template <typename E, int D, bool PAGED, bool DIRECT>
int launch(const AttnArgs &a, const Plan &p, hipStream_t st)
{
    hipLaunchKernelGGL((attention_kernel<E, D, PAGED, DIRECT>), dim3((unsigned)(p.units * a.kv_heads)), dim3(256), 0, st, a);
    if (p.split) {
        const unsigned tiles = (unsigned)(a.l.merge_cap < 1024 ? a.l.merge_cap : 1024);
        const unsigned z = tiles * (unsigned)a.kv_heads < 256 && (int64_t)a.T * a.group > 4 ? 16u : 1u;      // workgroups that share a tile's columns
        hipLaunchKernelGGL((attention_merge_kernel<E, D>), dim3(tiles, (unsigned)a.kv_heads, z), dim3(256), 0, st, a, PAGED ? 2 : 1);
    }
    return launched();
}

template <bool PAGED, bool DIRECT>
int launch_typed(const AttnArgs &a, int dtype, int32_t head_dim, const Plan &p, hipStream_t st)
{
    if (dtype == PREFT_BF16)
        return head_dim == 128 ? launch<__bf16, 128, PAGED, DIRECT>(a, p, st) : launch<__bf16, 64, PAGED, DIRECT>(a, p, st);
    return head_dim == 128 ? launch<float, 128, PAGED, DIRECT>(a, p, st) : launch<float, 64, PAGED, DIRECT>(a, p, st);
}

template <bool PAGED>
int run(AttnArgs &a, int dtype, int32_t head_dim, int mode, int64_t most_keys, hipStream_t st)
{
    Plan p = plan_of(a.s, most_keys);
    if (!p.split) a.s.can_split = 0;
    a.ready = mode & PREFT_SCHEDULE_READY;
    if (p.direct) return launch_typed<PAGED, true>(a, dtype, head_dim, p, st);
    if (!a.ready) {
        const int64_t items = (int64_t)a.s.S + a.s.n_groups, n = items > a.l.tile_cap ? items : a.l.tile_cap;
        const int threads = n >= SCHED_THREADS ? SCHED_THREADS : n <= 256 ? 256 : (int)((n + 63) / 64 * 64);
        hipLaunchKernelGGL(attn_schedule_kernel, dim3(1), dim3(threads), 0, st, a.s);
    }
    return launch_typed<PAGED, false>(a, dtype, head_dim, p, st);
}

int check_call(int32_t T, int32_t S, int32_t heads, int32_t kv_heads, int32_t head_dim, int32_t groups, float scale, int dtype, int mode)
{
    if (T < 0 || S < 0 || groups < 0 || (mode & ~PREFT_SCHEDULE_READY) != 0 || !(scale > 0.0f) || !std::isfinite(scale)) return PREFT_EINVAL;
    const int rc = check_heads(heads, kv_heads, head_dim, dtype);
    if (rc != PREFT_OK) return rc;
    return sizes_fit(T, S, heads, groups) ? PREFT_OK : PREFT_ETOOLARGE;
}

}  // namespace

extern "C" {

size_t preft_attention_workspace_bytes(int32_t T, int32_t S, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t n_groups)
{
    if (T < 0 || S < 0 || n_groups < 0 || check_heads(n_heads, n_kv_heads, head_dim, PREFT_F32) != PREFT_OK || !sizes_fit(T, S, n_heads, n_groups)) return 0;
    return layout_of(T, S, n_heads, n_kv_heads, head_dim, n_groups).bytes;
}

int preft_prompt_attention(void *out, int64_t ldo, const void *q, int64_t ldq, const void *k, int64_t ldk, const void *v, int64_t ldv, int32_t T,
                           int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, const int32_t *seg_start, const int32_t *seg_prefill_len, int32_t S,
                           float scale, int dtype, int mode, void *workspace, size_t workspace_bytes, void *stream)
{
    int rc = check_call(T, S, n_heads, n_kv_heads, head_dim, 0, scale, dtype, mode);
    if (rc != PREFT_OK) return rc;
    if (T == 0 || S == 0) return PREFT_OK;
    if (!seg_start || !seg_prefill_len) return PREFT_EINVAL;
    const int64_t wq = (int64_t)n_heads * head_dim, wk = (int64_t)n_kv_heads * head_dim;
    if ((rc = check_rows(out, ldo, wq, dtype)) != PREFT_OK || (rc = check_rows(q, ldq, wq, dtype)) != PREFT_OK ||
        (rc = check_rows(k, ldk, wk, dtype)) != PREFT_OK || (rc = check_rows(v, ldv, wk, dtype)) != PREFT_OK) return rc;
    if (rows_meet(out, ldo, wq, q, ldq, wq, T, dtype) || rows_meet(out, ldo, wq, k, ldk, wk, T, dtype) || rows_meet(out, ldo, wq, v, ldv, wk, T, dtype))
        return PREFT_EINVAL;
    const Layout l = layout_of(T, S, n_heads, n_kv_heads, head_dim, 0);
    if (!workspace || !aligned_workspace(workspace) || workspace_bytes < l.bytes) return PREFT_EWORKSPACE;
    const int64_t e = elem_bytes(dtype);
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    AttnArgs a = {};
    a.q = q; a.k = k; a.v = v; a.out = out;
    a.ldq = ldq * e; a.ldk = ldk * e; a.ldv = ldv * e; a.ldo = ldo * e;
    a.T = T; a.S = S; a.heads = n_heads; a.kv_heads = n_kv_heads; a.group = n_heads / n_kv_heads;
    a.per_head = ((1u << 21) + (uint32_t)a.group - 1) / (uint32_t)a.group;
    a.scale_log2 = scale * 1.44269504088896340736f;
    a.l = lists_of(l, workspace);
    AttnScheduleArgs &s = a.s;
    s.seg_start = seg_start; s.seg_prefill_len = seg_prefill_len; s.S = S; s.T = T; s.heads = n_heads; s.kv_heads = n_kv_heads; s.group = a.group;
    s.max_keys = T; s.l = a.l;
    // Cut only where the prompts are long on average and their tiles do not fill half the chip: a prompt has tiles by its rows as it has keys, and a
    // merge launch with nothing to join costs 4 us of the 10 that a batch of chat-length prompts takes (8 heads over 2 of 128: 4000 rows 66 us, uncut 74; 6000 rows
    // 115 uncut, cut 132; 32 heads over 8, 1200 rows: 30 uncut, cut 75).
    s.can_split = (int64_t)l.tile_cap * n_kv_heads <= ATTN_TARGET / 2 && T >= 512 * (int64_t)S;
    spread(s, dtype);
    s.min_tiles = s.min_wide;
    return run<false>(a, dtype, head_dim, mode, T, st);
}

int preft_cached_attention(void *out, int64_t ldo, const void *q, int64_t ldq, int32_t T, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                           const int32_t *seg_start, const int32_t *seg_prefill_len, const int32_t *kv_len, int32_t S, const void *k_cache,
                           const void *v_cache, int32_t n_pages, int32_t page_size, const int32_t *block_table, int64_t ld_table, int32_t max_pages,
                           const int32_t *group_start, const int32_t *group_prefix_len, int32_t n_groups, float scale, int dtype, int mode,
                           void *workspace, size_t workspace_bytes, void *stream)
{
    int rc = check_call(T, S, n_heads, n_kv_heads, head_dim, n_groups, scale, dtype, mode);
    if (rc != PREFT_OK) return rc;
    if (n_pages < 0 || max_pages < 0 || ld_table < max_pages) return PREFT_EINVAL;
    const int shift = page_shift_of(page_size);
    if (shift < 0) return PREFT_EUNSUPPORTED;
    if (T == 0 || S == 0) return PREFT_OK;
    if (!seg_start || !kv_len || (n_groups > 0 && (!group_start || !group_prefix_len))) return PREFT_EINVAL;
    const int64_t wq = (int64_t)n_heads * head_dim, wk = (int64_t)n_kv_heads * head_dim, e = elem_bytes(dtype);
    if ((rc = check_rows(out, ldo, wq, dtype)) != PREFT_OK || (rc = check_rows(q, ldq, wq, dtype)) != PREFT_OK) return rc;
    const bool keys = n_pages > 0 && max_pages > 0;               // without pages every row sees no key
    if (keys && (!k_cache || !v_cache || !block_table)) return PREFT_EINVAL;
    if (keys && ((reinterpret_cast<uintptr_t>(k_cache) | reinterpret_cast<uintptr_t>(v_cache)) & 15) != 0) return PREFT_EALIGN;
    if (rows_meet(out, ldo, wq, q, ldq, wq, T, dtype)) return PREFT_EINVAL;
    const int64_t cache = (int64_t)n_pages * page_size * wk * e;
    const Span o = {out, ((int64_t)(T - 1) * ldo + wq) * e};
    if (keys && (o.meets({k_cache, cache}) || o.meets({v_cache, cache}))) return PREFT_EINVAL;
    const Layout l = layout_of(T, S, n_heads, n_kv_heads, head_dim, n_groups);
    if (!workspace || !aligned_workspace(workspace) || workspace_bytes < l.bytes) return PREFT_EWORKSPACE;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    AttnArgs a = {};
    a.q = q; a.k = k_cache; a.v = v_cache; a.out = out; a.ldq = ldq * e; a.ldo = ldo * e;
    a.table = block_table; a.ld_table = ld_table; a.n_pages = n_pages; a.page_shift = shift;
    a.T = T; a.S = S; a.heads = n_heads; a.kv_heads = n_kv_heads; a.group = n_heads / n_kv_heads; a.n_groups = n_groups;
    a.per_head = ((1u << 21) + (uint32_t)a.group - 1) / (uint32_t)a.group;
    a.scale_log2 = scale * 1.44269504088896340736f;
    a.l = lists_of(l, workspace);
    AttnScheduleArgs &s = a.s;
    s.seg_start = seg_start; s.seg_prefill_len = seg_prefill_len; s.kv_len = kv_len; s.group_start = group_start; s.group_prefix = group_prefix_len;
    s.S = S; s.T = T; s.n_groups = n_groups; s.heads = n_heads; s.kv_heads = n_kv_heads; s.group = a.group; s.l = a.l;
    const int64_t most = (int64_t)max_pages << shift;
    s.max_keys = keys ? (int32_t)(most < (1 << 30) ? most : (1 << 30)) : 0;
    s.can_split = 1;
    spread(s, dtype);
    return run<true>(a, dtype, head_dim, mode, s.max_keys, st);
}

}  // extern "C"
