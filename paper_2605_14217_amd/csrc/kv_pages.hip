// Pages of the key/value cache: block tables and slot maps from request lengths (preft_kv_plan), and the store of a
// batch's keys and values (preft_kv_store).  See include/preft.h for the contract of both.
#include "../../include/preft.h"

#include "attention_common.hpp"
#include "block_scan.hpp"

namespace {

using namespace preft;

struct PlanArgs {
    int64_t *slot_map;
    int32_t *positions, *kv_len, *table, *counts;
    const int32_t *seg_start, *ctx_len, *free_pages;
    int64_t  ld_table;
    int32_t  max_pages, S, T, n_free, page_shift;
};

// 1024 rows a workgroup of 512: of workgroups of 1024 threads a compute unit holds one, and 356 000 rows took two rounds (12.0 us).
constexpr int PLAN_THREADS = 512, PLAN_ROWS = 2;

struct PlanRequest { int32_t lo, hi, ctx, need, over; };     // rows, tokens before them, pages to begin within and beyond the table

__device__ __forceinline__ PlanRequest plan_request(const PlanArgs &a, int32_t s)
{
    PlanRequest r;
    const int32_t page = 1 << a.page_shift;
    r.lo = max(0, min(a.seg_start[s], a.T));
    r.hi = max(r.lo, min(a.seg_start[s + 1], a.T));
    r.ctx = max(0, min(a.ctx_len[s], INT32_MAX - (r.hi - r.lo)));
    const int32_t have = (int32_t)(((int64_t)r.ctx + page - 1) >> a.page_shift), want = (int32_t)(((int64_t)r.ctx + (r.hi - r.lo) + page - 1) >> a.page_shift);
    r.need = min(want, a.max_pages) - min(have, a.max_pages);
    r.over = want - have - r.need;
    return r;
}

// sum over the workgroup, for every thread; `lds`: one place a wavefront
__device__ __forceinline__ uint32_t block_sum(uint32_t v, uint32_t *lds)
{
    const int lane = threadIdx.x & 63, waves = blockDim.x >> 6;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    if (lane == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lane < waves ? lds[lane] : 0;
#pragma unroll
    for (int off = 8; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    return __shfl(v, 0, 64);
}

// have = ceil(ctx / page), want = ceil((ctx + n) / page), both cut at max_pages; page k of a request, have <= k < want, is
// free_pages[off + k - have] with off = sum of want - have over the requests before it.  (A new page has a row at its start: all sums are at most T.  Of
// requests that overlap they may wrap; a pick is compared unsigned, and stays within the list.)
// Latency is what bounds it: a handful of bytes per request, and a chain of reads.  Every workgroup therefore sums the requests before its rows by itself (twelve
// bytes each, from the cache, all reads in flight at once) instead of waiting for another launch to do it, keeps the requests that own its rows in LDS, and
// writes its rows; the last one sums all requests and writes kv_len and the counts.  32 requests, one row each: 4.2 us a call; 4096 requests and 356 000 rows:
// 9.2 us, where the 4.5 MB that it moves would take 1.
__global__ __launch_bounds__(PLAN_THREADS) void kv_plan_kernel(PlanArgs a)
{
    __shared__ int32_t lds[32];
    __shared__ uint32_t sums[4][PLAN_THREADS / 64], own_off[PLAN_THREADS];
    __shared__ int32_t own_start[PLAN_THREADS], own_end[PLAN_THREADS], own_ctx[PLAN_THREADS];
    const int32_t page = 1 << a.page_shift, n_threads = (int32_t)blockDim.x;
    const int32_t row0 = (int32_t)blockIdx.x * n_threads * PLAN_ROWS, row1 = min(a.T, row0 + n_threads * PLAN_ROWS);
    const bool last = blockIdx.x + 1 == gridDim.x;
    // requests that end before this workgroup's rows: their pages, and how many they are; all requests: their pages, and those that do not fit the table
    uint32_t off = 0, first = 0, all = 0, over = 0;
#pragma unroll 4
    for (int32_t s = (int32_t)threadIdx.x; s < a.S; s += n_threads) {
        const PlanRequest r = plan_request(a, s);
        if (r.hi <= row0) { off += (uint32_t)r.need; ++first; }
        all += (uint32_t)r.need;
        over += (uint32_t)r.over;
        if (last) a.kv_len[s] = r.ctx + (r.hi - r.lo);
    }
    if (row0 > 0) {                                    // else there are none before, but empty ones
        off = block_sum(off, sums[0]);
        first = block_sum(first, sums[1]);
    } else {
        off = 0;
        first = 0;
    }
    if (last) {
        all = block_sum(all, sums[2]);
        over = block_sum(over, sums[3]);
        if (threadIdx.x == 0) {
            const uint32_t taken = min((uint32_t)a.n_free, all);
            a.counts[0] = (int32_t)taken;
            a.counts[1] = (int32_t)(all - taken + over);
        }
    }
    int64_t slot[PLAN_ROWS];
    int32_t at[PLAN_ROWS];
#pragma unroll
    for (int i = 0; i < PLAN_ROWS; ++i) { slot[i] = -1; at[i] = 0; }
    for (int32_t s0 = (int32_t)first; s0 < a.S; s0 += n_threads) {          // more than once only where hundreds of requests without rows stand together
        const int32_t s = s0 + (int32_t)threadIdx.x;
        PlanRequest r = {};
        r.lo = INT32_MAX;
        if (s < a.S) r = plan_request(a, s);
        int32_t total;
        const int32_t here = block_exclusive_scan(r.need, lds, &total);        // its barriers also end the reads of the turn before
        own_start[threadIdx.x] = r.lo; own_end[threadIdx.x] = r.hi; own_ctx[threadIdx.x] = r.ctx; own_off[threadIdx.x] = off + (uint32_t)here;
        off += (uint32_t)total;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < PLAN_ROWS; ++i) {
            const int32_t row = row0 + i * n_threads + (int32_t)threadIdx.x;
            int32_t lo = 0, hi = n_threads;                        // the last request that starts at or before the row: an empty one never is
            while (hi - lo > 1) {
                const int32_t mid = (lo + hi) >> 1;
                if (own_start[mid] <= row) lo = mid; else hi = mid;
            }
            if (row >= row1 || own_start[lo] > row || row >= own_end[lo]) continue;
            at[i] = own_ctx[lo] + (row - own_start[lo]);
            const int32_t k = at[i] >> a.page_shift, have = (int32_t)(((int64_t)own_ctx[lo] + page - 1) >> a.page_shift);
            if (k >= a.max_pages) continue;
            int32_t *entry = a.table + (int64_t)(s0 + lo) * a.ld_table + k;
            int32_t p;
            if (k < have) {
                p = *entry;
            } else {
                const uint32_t pick = own_off[lo] + (uint32_t)(k - have);
                p = pick < (uint32_t)a.n_free ? a.free_pages[pick] : -1;
                if ((at[i] & (page - 1)) == 0) *entry = p;         // a new page has exactly one row at its start
            }
            if (p >= 0) slot[i] = ((int64_t)p << a.page_shift) + (at[i] & (page - 1));
        }
        if (a.seg_start[min(s0 + n_threads, a.S)] >= row1) break;
    }
#pragma unroll
    for (int i = 0; i < PLAN_ROWS; ++i) {
        const int32_t row = row0 + i * n_threads + (int32_t)threadIdx.x;
        if (row >= row1) continue;
        a.slot_map[row] = slot[i];
        a.positions[row] = at[i];
    }
}

struct StoreArgs {
    char *k_cache, *v_cache;
    const char *k, *v;
    const int64_t *slot_map;
    int64_t ldk, ldv;          // bytes
    int64_t n_slots;
    int32_t T, page_shift, heads, head_bytes;
};

// A copy: bound by memory.  A wavefront moves the k (grid.y = 0) or v row of one token, 16 bytes a lane; a head's row lands in one piece (page, head, position in the page,
// head_dim).  One row a wavefront: 33 rows of 8 heads of 128 in f32 in 3.8 us (four rows, all in flight: 5.2).  The pages are written with the non-temporal hint, so
// that the rows' keys and values, which attention reads next, stay in the caches: store and prompt attention of 36 864 rows together 558 us, 563 without the hint
// or with it on the loads too (the store alone 65.5 us, 4.6 TB/s; 71 and 63.8).
__global__ __launch_bounds__(256) void kv_store_kernel(StoreArgs a)
{
    const int lane = threadIdx.y & 63;
    const int32_t row = __builtin_amdgcn_readfirstlane((int32_t)(blockIdx.x * 4 + (threadIdx.y >> 6)));
    if (row >= a.T) return;
    const int64_t slot = as_const(a.slot_map)[row];
    if (slot < 0 || slot >= a.n_slots) return;
    const gcptr_t src = as_global((const void *)(blockIdx.y ? a.v : a.k)) + row * (blockIdx.y ? a.ldv : a.ldk);
    const gptr_t dst = as_global((void *)(blockIdx.y ? a.v_cache : a.k_cache)) + (slot >> a.page_shift) * (((int64_t)a.heads * a.head_bytes) << a.page_shift) +
                       (slot & ((1 << a.page_shift) - 1)) * a.head_bytes;
    const int32_t pieces = a.head_bytes / 16, n = a.heads * pieces;
#pragma unroll 2
    for (int32_t c = lane; c < n; c += 64) {
        const int32_t head = c / pieces;
        const int64_t to = (((int64_t)head * a.head_bytes) << a.page_shift) + (c - head * pieces) * 16;
        __builtin_nontemporal_store(ld16(src + c * 16), (PREFT_GLOBAL u32x4_t *)(dst + to));
    }
}

}  // namespace

extern "C" {

int preft_kv_plan(int64_t *slot_map, int32_t *positions, int32_t *kv_len, int32_t *block_table, int64_t ld_table, int32_t max_pages,
                  int32_t *counts, const int32_t *seg_start, const int32_t *ctx_len, int32_t S, int32_t T, const int32_t *free_pages,
                  int32_t n_free, int32_t page_size, void *stream)
{
    if (T < 0 || S < 0 || n_free < 0 || max_pages < 0 || ld_table < max_pages) return PREFT_EINVAL;
    const int shift = page_shift_of(page_size);
    if (shift < 0) return PREFT_EUNSUPPORTED;
    if (S == 0 || T == 0) {
        if (S == 0 && T == 0) return PREFT_OK;
        if (S == 0) return PREFT_EINVAL;               // rows of no request
    }
    if ((T > 0 && (!slot_map || !positions)) || !kv_len || !counts || !seg_start || !ctx_len || (max_pages > 0 && !block_table) ||
        (n_free > 0 && !free_pages)) return PREFT_EINVAL;
    PlanArgs a;
    a.slot_map = slot_map; a.positions = positions; a.kv_len = kv_len; a.table = block_table; a.counts = counts;
    a.seg_start = seg_start; a.ctx_len = ctx_len; a.free_pages = free_pages;
    a.ld_table = ld_table; a.max_pages = max_pages; a.S = S; a.T = T; a.n_free = n_free; a.page_shift = shift;
    const int32_t most = S > T ? S : T;                // a step of a few dozen rows: one small workgroup, no wavefronts to wait for at its barriers
    const int threads = most >= PLAN_THREADS ? PLAN_THREADS : (most + 63) / 64 * 64;
    const int64_t rows = (int64_t)threads * PLAN_ROWS;
    const unsigned grid = T > 0 ? (unsigned)((T + rows - 1) / rows) : 1u;
    hipLaunchKernelGGL(kv_plan_kernel, dim3(grid), dim3(threads), 0, reinterpret_cast<hipStream_t>(stream), a);
    return launched();
}

int preft_kv_store(void *k_cache, void *v_cache, int32_t n_pages, int32_t page_size, const void *k, int64_t ldk, const void *v, int64_t ldv,
                   int32_t T, int32_t n_kv_heads, int32_t head_dim, const int64_t *slot_map, int dtype, void *stream)
{
    if (T < 0 || n_pages < 0) return PREFT_EINVAL;
    const int shift = page_shift_of(page_size);
    int rc = check_heads(n_kv_heads, n_kv_heads, head_dim, dtype);
    if (rc != PREFT_OK) return rc;
    if (shift < 0) return PREFT_EUNSUPPORTED;
    if (T == 0) return PREFT_OK;
    if (!slot_map) return PREFT_EINVAL;
    const int64_t width = (int64_t)n_kv_heads * head_dim;
    if ((rc = check_rows(k, ldk, width, dtype)) != PREFT_OK || (rc = check_rows(v, ldv, width, dtype)) != PREFT_OK) return rc;
    if (n_pages == 0) return PREFT_OK;                 // no slot exists: nothing is written
    if (!k_cache || !v_cache) return PREFT_EINVAL;
    if (((reinterpret_cast<uintptr_t>(k_cache) | reinterpret_cast<uintptr_t>(v_cache)) & 15) != 0) return PREFT_EALIGN;
    const int64_t e = elem_bytes(dtype), cache = (int64_t)n_pages * page_size * width * e;
    const Span in[2] = {{k, ((int64_t)(T - 1) * ldk + width) * e}, {v, ((int64_t)(T - 1) * ldv + width) * e}};
    const Span out[2] = {{k_cache, cache}, {v_cache, cache}};
    if (out[0].meets(out[1])) return PREFT_EINVAL;
    for (const Span &o : out)
        for (const Span &i : in)
            if (o.meets(i)) return PREFT_EINVAL;
    StoreArgs a;
    a.k_cache = (char *)k_cache; a.v_cache = (char *)v_cache; a.k = (const char *)k; a.v = (const char *)v; a.slot_map = slot_map;
    a.ldk = ldk * e; a.ldv = ldv * e; a.n_slots = (int64_t)n_pages * page_size; a.T = T; a.page_shift = shift; a.heads = n_kv_heads;
    a.head_bytes = (int32_t)(head_dim * e);
    hipLaunchKernelGGL(kv_store_kernel, dim3((unsigned)(((int64_t)T + 3) / 4), 2), row_threads(), 0, reinterpret_cast<hipStream_t>(stream), a);
    return launched();
}

}  // extern "C"
