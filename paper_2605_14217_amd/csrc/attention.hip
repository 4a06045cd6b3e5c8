// C entry points of attention: argument checks, the layout of the workspace, launches.  See include/preft.h for the contract.
#include "../../include/preft.h"

#include "attention_common.hpp"
#include "attention_kernel.hpp"

#include <cmath>

namespace {

using namespace preft;

// Work ranges may be cut where the tiles of all segments are few.  Bounds on the lists, for tables that are well-formed:
//   column tiles   T G / 128 + one part-filled tile a segment, and the same of groups;
//   units          a tile is cut into ceil(n / range) <= 1 + n / range ranges, and the n of all tiles add up to at most TARGET / kv_heads ranges
//                  and one more a tile (the estimate of a causal prompt's work is half a tile off each way);
//   part columns   a tile that is cut has at most twice n / range parts of at most 128 columns; rows of groups have one of their own and their group's.
struct Layout {
    int32_t tile_cap, unit_cap, merge_cap, group_row_cap, slot_cap;
    size_t units, merges, group_rows, tiles, rows_before, group_of, group_list, group_slot, part_ml, part_o, bytes;
};

Layout layout_of(int64_t T, int64_t S, int64_t heads, int64_t kv_heads, int64_t D, int64_t groups)
{
    Layout l;
    const int64_t G = heads / kv_heads, cols = T * G;
    const int64_t seg_tiles = cols / ATTN_COLS + (S < T ? S : T);
    const int64_t tiles = groups > 0 ? 2 * seg_tiles + groups : seg_tiles;
    l.tile_cap = (int32_t)tiles;
    l.unit_cap = (int32_t)(2 * tiles + ATTN_TARGET + 64);
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
    r.part_ml = (float2 *)(p + l.part_ml);
    r.part_o = (float *)(p + l.part_o);
    r.tile_cap = l.tile_cap; r.unit_cap = l.unit_cap; r.merge_cap = l.merge_cap; r.group_row_cap = l.group_row_cap; r.slot_cap = l.slot_cap;
    return r;
}

bool sizes_fit(int64_t T, int64_t S, int64_t heads, int64_t groups) { return T * heads < (1ll << 30) && S + groups < (1ll << 28); }

template <typename E, int D, bool PAGED>
int launch(const AttnArgs &a, bool split, hipStream_t st)
{
    const unsigned units = split ? (unsigned)a.l.unit_cap : (unsigned)a.l.tile_cap;
    hipLaunchKernelGGL((attention_kernel<E, D, PAGED>), dim3(units * (unsigned)a.kv_heads), dim3(256), 0, st, a);
    if (split) {
        const unsigned x = a.l.merge_cap < 1024 ? (unsigned)a.l.merge_cap : 1024u;
        const unsigned z = x * (unsigned)a.kv_heads < 512 && (int64_t)a.T * (a.heads / a.kv_heads) > 4 ? 8u : 1u;
        hipLaunchKernelGGL((attention_merge_kernel<E, D>), dim3(x, (unsigned)a.kv_heads, z), dim3(256), 0, st, a, PAGED ? 2 : 1);
    }
    return launched();
}

template <bool PAGED>
int dispatch(const AttnArgs &a, int dtype, int32_t head_dim, bool split, hipStream_t st)
{
    if (dtype == PREFT_BF16) return head_dim == 128 ? launch<__bf16, 128, PAGED>(a, split, st) : launch<__bf16, 64, PAGED>(a, split, st);
    return head_dim == 128 ? launch<float, 128, PAGED>(a, split, st) : launch<float, 64, PAGED>(a, split, st);
}

void launch_schedule(const AttnScheduleArgs &s, hipStream_t st)
{
    const int64_t n = (int64_t)s.S + s.n_groups > s.l.tile_cap ? (int64_t)s.S + s.n_groups : s.l.tile_cap;
    const int threads = n >= SCHED_THREADS ? SCHED_THREADS : n <= 256 ? 256 : (int)((n + 63) / 64 * 64);
    hipLaunchKernelGGL(attn_schedule_kernel, dim3(1), dim3(threads), 0, st, s);
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
    const bool split = (int64_t)l.tile_cap * n_kv_heads < 4 * ATTN_TARGET;     // else there are tiles enough
    if (!(mode & PREFT_SCHEDULE_READY)) {
        AttnScheduleArgs s = {};
        s.seg_start = seg_start; s.seg_prefill_len = seg_prefill_len; s.S = S; s.T = T; s.heads = n_heads; s.kv_heads = n_kv_heads;
        s.max_keys = T; s.can_split = split; s.min_tiles = 8; s.l = a.l;
        launch_schedule(s, st);
    }
    return dispatch<false>(a, dtype, head_dim, split, st);
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
    a.table = block_table; a.ld_table = ld_table; a.n_pages = n_pages; a.page_shift = shift; a.max_pages = max_pages;
    a.T = T; a.S = S; a.heads = n_heads; a.kv_heads = n_kv_heads; a.group = n_heads / n_kv_heads; a.n_groups = n_groups;
    a.per_head = ((1u << 21) + (uint32_t)a.group - 1) / (uint32_t)a.group;
    a.scale_log2 = scale * 1.44269504088896340736f;
    a.l = lists_of(l, workspace);
    if (!(mode & PREFT_SCHEDULE_READY)) {
        AttnScheduleArgs s = {};
        s.seg_start = seg_start; s.seg_prefill_len = seg_prefill_len; s.kv_len = kv_len; s.group_start = group_start; s.group_prefix = group_prefix_len;
        s.S = S; s.T = T; s.n_groups = n_groups; s.heads = n_heads; s.kv_heads = n_kv_heads;
        const int64_t most = (int64_t)max_pages << shift;
        s.max_keys = keys ? (int32_t)(most < (1 << 30) ? most : (1 << 30)) : 0;
        s.can_split = 1; s.min_tiles = 4; s.l = a.l;
        launch_schedule(s, st);
    }
    return dispatch<true>(a, dtype, head_dim, true, st);
}

}  // extern "C"
