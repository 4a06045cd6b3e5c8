// C entry points of attention: argument checks and launches.  See include/preft.h for the contract.
#include "../../include/preft.h"

#include "attention_common.hpp"
#include "attention_kernel.hpp"
#include "attention_plan.hpp"

#include <cmath>

namespace {

using namespace preft;

template <typename E, int D, bool PAGED, bool DIRECT>
int launch(const AttnArgs &a, const Plan &p, hipStream_t st)
{
    hipLaunchKernelGGL((attention_kernel<E, D, PAGED, DIRECT>), dim3((unsigned)(p.units * a.s.kv_heads)), dim3(256), 0, st, a);
    if (p.merge) {
        const unsigned tiles = (unsigned)(a.s.l.merge_cap < 1024 ? a.s.l.merge_cap : 1024);
        const unsigned z = tiles * (unsigned)a.s.kv_heads < 256 && (int64_t)a.s.T * a.s.group > 4 ? 16u : 1u;      // workgroups that share a tile's columns
        hipLaunchKernelGGL((attention_merge_kernel<E, D>), dim3(tiles, (unsigned)a.s.kv_heads, z), dim3(256), 0, st, a, PAGED ? 2 : 1);
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
int run(AttnArgs &a, int dtype, int32_t head_dim, int mode, hipStream_t st)
{
    Plan p = plan_of(a.s);
    if (!p.split) a.s.can_split = 0;
    a.ready = mode & PREFT_SCHEDULE_READY;
    if (p.direct) return launch_typed<PAGED, true>(a, dtype, head_dim, p, st);
    if (!a.ready) {
        const int threads = schedule_threads(a.s);
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
    return run<false>(a, dtype, head_dim, mode, st);
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
    cached_rules(s, dtype, keys ? (int64_t)max_pages << shift : 0);
    return run<true>(a, dtype, head_dim, mode, st);
}

}  // extern "C"
