// C entry points of attention: argument checks and launches.  See include/preft.h for the contract.
#include "../../include/preft.h"

#include "attention_common.hpp"
#include "attention_kernel.hpp"
#include "attention_mx.hpp"
#include "attention_plan.hpp"

#include <algorithm>
#include <cmath>

namespace {

using namespace preft;

enum Keys { PACKED, PAGES, MX_PAGES };                           // where a call's keys are

template <typename E, int D, int KEYS, bool DIRECT>
int launch(AttnArgs &a, const Plan &p, hipStream_t st)
{
    // a launch has fewer than 2^32 threads (HIP): units of 2^23 workgroups at once
    const int64_t most = (1 << 23) / a.s.kv_heads;
    for (int64_t first = 0; first < p.units; first += most) {
        const dim3 grid((unsigned)(std::min(p.units - first, most) * a.s.kv_heads));
        a.first = (int32_t)first;
        if constexpr (KEYS == MX_PAGES) launch_mx_attention(a, (int)sizeof(E), D, DIRECT, grid, st);
        else hipLaunchKernelGGL((attention_kernel<E, D, KEYS == PAGES, DIRECT>), grid, dim3(256), 0, st, a);
    }
    if (p.merge) {
        const unsigned tiles = (unsigned)(a.s.l.merge_cap < 1024 ? a.s.l.merge_cap : 1024);
        unsigned z = tiles * (unsigned)a.s.kv_heads < 256 && (int64_t)a.s.T * a.s.group > 4 ? 16u : 1u;      // workgroups that share a tile's columns
        // 4-bit pages: a wavefront takes a microsecond a column, and tiles of 16 columns and more on average are shared by up to 2048 workgroups in all (28 requests of 8 rows with 4 prefixes
        // of 10 544 tokens, 32 heads over 8: 74 us, of which the join took 19 of 84)
        if (KEYS == MX_PAGES && z == 1 && (int64_t)a.s.T * a.s.group >= 16 * (int64_t)a.s.l.merge_cap)
            z = std::max(1u, std::min(8u, 2048u / (tiles * (unsigned)a.s.kv_heads)));
        hipLaunchKernelGGL((attention_merge_kernel<E, D>), dim3(tiles, (unsigned)a.s.kv_heads, z), dim3(256), 0, st, a, KEYS == PACKED ? 1 : 2);
    }
    return launched();
}

template <int KEYS, bool DIRECT>
int launch_typed(AttnArgs &a, int dtype, int32_t head_dim, const Plan &p, hipStream_t st)
{
    if (dtype == PREFT_BF16)
        return head_dim == 128 ? launch<__bf16, 128, KEYS, DIRECT>(a, p, st) : launch<__bf16, 64, KEYS, DIRECT>(a, p, st);
    return head_dim == 128 ? launch<float, 128, KEYS, DIRECT>(a, p, st) : launch<float, 64, KEYS, DIRECT>(a, p, st);
}

template <int KEYS>
int run(AttnArgs &a, int dtype, int32_t head_dim, int mode, hipStream_t st)
{
    Plan p = plan_of(a.s);
    if (!p.split) a.s.can_split = 0;
    a.ready = mode & PREFT_SCHEDULE_READY;
    if (p.direct) return launch_typed<KEYS, true>(a, dtype, head_dim, p, st);
    if (!a.ready) {
        const int threads = schedule_threads(a.s);
        hipLaunchKernelGGL(attn_schedule_kernel, dim3(1), dim3(threads), 0, st, a.s);
    }
    return launch_typed<KEYS, false>(a, dtype, head_dim, p, st);
}

int check_call(int32_t T, int32_t S, int32_t heads, int32_t kv_heads, int32_t head_dim, int32_t groups, float scale, int dtype, int mode)
{
    if (T < 0 || S < 0 || groups < 0 || (mode & ~PREFT_SCHEDULE_READY) != 0 || !(scale > 0.0f) || !std::isfinite(scale)) return PREFT_EINVAL;
    const int rc = check_heads(heads, kv_heads, head_dim, dtype);
    if (rc != PREFT_OK) return rc;
    return sizes_fit(T, S, heads, groups) ? PREFT_OK : PREFT_ETOOLARGE;
}

int cached_call(Keys keys_in, void *out, int64_t ldo, const void *q, int64_t ldq, int32_t T, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                const int32_t *seg_start, const int32_t *seg_prefill_len, const int32_t *kv_len, int32_t S, const void *k_cache, const void *v_cache, int32_t n_pages,
                int32_t page_size, const int32_t *block_table, int64_t ld_table, int32_t max_pages, const int32_t *group_start, const int32_t *group_prefix_len,
                int32_t n_groups, float scale, int dtype, int mode, void *workspace, size_t workspace_bytes, void *stream)
{
    int rc = check_call(T, S, n_heads, n_kv_heads, head_dim, n_groups, scale, dtype, mode);
    if (rc != PREFT_OK) return rc;
    if (n_pages < 0 || max_pages < 0 || ld_table < max_pages) return PREFT_EINVAL;
    const int shift = page_shift_of(page_size);
    if (shift < 0) return PREFT_EUNSUPPORTED;
    if (T == 0 || S == 0) return PREFT_OK;
    if (!seg_start || !kv_len || (n_groups > 0 && (!group_start || !group_prefix_len))) return PREFT_EINVAL;
    const int64_t wq = (int64_t)n_heads * head_dim, e = elem_bytes(dtype);
    if ((rc = check_rows(out, ldo, wq, dtype)) != PREFT_OK || (rc = check_rows(q, ldq, wq, dtype)) != PREFT_OK) return rc;
    const bool keys = n_pages > 0 && max_pages > 0;               // without pages every row sees no key
    if (keys && (!k_cache || !v_cache || !block_table)) return PREFT_EINVAL;
    if (keys && ((reinterpret_cast<uintptr_t>(k_cache) | reinterpret_cast<uintptr_t>(v_cache)) & 15) != 0) return PREFT_EALIGN;
    if (rows_meet(out, ldo, wq, q, ldq, wq, T, dtype)) return PREFT_EINVAL;
    const int64_t token = keys_in == MX_PAGES ? head_dim / 2 + head_dim / MX4_BLOCK : head_dim * e, cache = (int64_t)n_pages * page_size * n_kv_heads * token;
    const Span o = {out, ((int64_t)(T - 1) * ldo + wq) * e};
    if (keys && (o.meets({k_cache, cache}) || o.meets({v_cache, cache}))) return PREFT_EINVAL;
    const Layout l = cached_layout(T, S, n_heads, n_kv_heads, head_dim, n_groups);
    if (!workspace || !aligned_workspace(workspace) || workspace_bytes < l.end) return PREFT_EWORKSPACE;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    AttnArgs a = {};
    a.q = q; a.k = k_cache; a.v = v_cache; a.out = out; a.ldq = ldq * e; a.ldo = ldo * e;
    a.table = block_table; a.ld_table = ld_table; a.n_pages = n_pages; a.page_shift = shift;
    a.scale_log2 = scale * 1.44269504088896340736f;
    AttnScheduleArgs &s = a.s;
    s.seg_start = seg_start; s.seg_prefill_len = seg_prefill_len; s.kv_len = kv_len; s.group_start = group_start; s.group_prefix = group_prefix_len;
    s.S = S; s.T = T; s.n_groups = n_groups; s.heads = n_heads; s.kv_heads = n_kv_heads; s.group = n_heads / n_kv_heads; s.l = lists_of(l, workspace);
    a.per_head = ((1u << 21) + (uint32_t)s.group - 1) / (uint32_t)s.group;
    const int64_t most_keys = keys ? (int64_t)max_pages << shift : 0;
    cached_rules(s, keys_in == MX_PAGES ? ATTN_MX_TYPE | dtype : dtype, most_keys);
    return keys_in == MX_PAGES ? run<MX_PAGES>(a, dtype, head_dim, mode, st) : run<PAGES>(a, dtype, head_dim, mode, st);
}

}  // namespace

extern "C" {

size_t preft_attention_workspace_bytes(int32_t T, int32_t S, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t n_groups)
{
    if (T < 0 || S < 0 || n_groups < 0 || check_heads(n_heads, n_kv_heads, head_dim, PREFT_F32) != PREFT_OK || !sizes_fit(T, S, n_heads, n_groups)) return 0;
    return cached_layout(T, S, n_heads, n_kv_heads, head_dim, n_groups).end;
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
    if (!workspace || !aligned_workspace(workspace) || workspace_bytes < cached_layout(T, S, n_heads, n_kv_heads, head_dim, 0).end) return PREFT_EWORKSPACE;
    const Layout l = prompt_layout(T, S, n_heads, n_kv_heads);
    const int64_t e = elem_bytes(dtype);
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    AttnArgs a = {};
    a.q = q; a.k = k; a.v = v; a.out = out;
    a.ldq = ldq * e; a.ldk = ldk * e; a.ldv = ldv * e; a.ldo = ldo * e;
    a.scale_log2 = scale * 1.44269504088896340736f;
    AttnScheduleArgs &s = a.s;
    s.seg_start = seg_start; s.seg_prefill_len = seg_prefill_len;
    s.S = S; s.T = T; s.heads = n_heads; s.kv_heads = n_kv_heads; s.group = n_heads / n_kv_heads; s.l = lists_of(l, workspace);
    a.per_head = ((1u << 21) + (uint32_t)s.group - 1) / (uint32_t)s.group;
    prompt_rules(s, dtype);
    return run<PACKED>(a, dtype, head_dim, mode, st);
}

int preft_cached_attention(void *out, int64_t ldo, const void *q, int64_t ldq, int32_t T, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                           const int32_t *seg_start, const int32_t *seg_prefill_len, const int32_t *kv_len, int32_t S, const void *k_cache,
                           const void *v_cache, int32_t n_pages, int32_t page_size, const int32_t *block_table, int64_t ld_table, int32_t max_pages,
                           const int32_t *group_start, const int32_t *group_prefix_len, int32_t n_groups, float scale, int dtype, int mode,
                           void *workspace, size_t workspace_bytes, void *stream)
{
    return cached_call(PAGES, out, ldo, q, ldq, T, n_heads, n_kv_heads, head_dim, seg_start, seg_prefill_len, kv_len, S, k_cache, v_cache, n_pages, page_size,
                       block_table, ld_table, max_pages, group_start, group_prefix_len, n_groups, scale, dtype, mode, workspace, workspace_bytes, stream);
}

int preft_cached_attention_mx(void *out, int64_t ldo, const void *q, int64_t ldq, int32_t T, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                           const int32_t *seg_start, const int32_t *seg_prefill_len, const int32_t *kv_len, int32_t S, const void *k_cache,
                           const void *v_cache, int32_t n_pages, int32_t page_size, const int32_t *block_table, int64_t ld_table, int32_t max_pages,
                           const int32_t *group_start, const int32_t *group_prefix_len, int32_t n_groups, float scale, int dtype, int mode,
                           void *workspace, size_t workspace_bytes, void *stream)
{
    return cached_call(MX_PAGES, out, ldo, q, ldq, T, n_heads, n_kv_heads, head_dim, seg_start, seg_prefill_len, kv_len, S, k_cache, v_cache, n_pages, page_size,
                       block_table, ld_table, max_pages, group_start, group_prefix_len, n_groups, scale, dtype, mode, workspace, workspace_bytes, stream);
}

}  // extern "C"
