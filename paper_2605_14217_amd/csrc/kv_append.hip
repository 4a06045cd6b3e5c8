// Heads of queries and keys, normed and turned by their position: as rows (preft_qk_rotate), and on the way into pages of activations (preft_kv_append) or of
// 4-bit numbers (preft_kv_append_mx); and rows out of such pages (preft_kv_fetch_mx).  See include/preft.h for the contract.
#include "../../include/preft.h"

#include "attention_common.hpp"
#include "mx4.hpp"

#include <cmath>

namespace {

using namespace preft;

enum Pages { NO_PAGES, PLAIN_PAGES, MX4_PAGES };

struct HeadsArgs {
    const char *q, *k, *v, *q_weight, *k_weight;
    char *q_out, *k_out, *k_cache, *v_cache;
    int64_t ldq, ldk, ldv, ldqo, ldko;       // bytes
    const int32_t *positions;
    const int64_t *slot_map;
    const float *rotation;                   // [n_positions][rot]: cosines, sines
    int64_t n_slots;
    double eps;
    int32_t T, q_heads, kv_heads, n_positions, rot, page_shift, splits;
};

// A head is spread over LANES lanes, two pieces of 16 bytes each: with the first half's and the second half's elements (or neighbours) of a pair in one lane a head is
// turned without an exchange, and its norm takes log2(LANES) of them.
template <typename E, int D> struct Heads {
    static constexpr int ELEM = sizeof(E), PE = 16 / ELEM;        // elements of a piece
    static constexpr int ROW = D * ELEM, LANES = ROW / 32, AT_ONCE = 64 / LANES;
};

template <typename E> __device__ __forceinline__ void widen(u32x4_t v, float *x)
{
    if constexpr (sizeof(E) == 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = bf16_lo(v[i]); x[2 * i + 1] = bf16_hi(v[i]); }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(v[i]);
    }
}
template <typename E> __device__ __forceinline__ u32x4_t narrow(const float *x)
{
    u32x4_t v;
    if constexpr (sizeof(E) == 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __float_as_uint(x[i]);
    }
    return v;
}

// What a lane does to its share of every head of a row.
template <typename E, int D, bool HALVES> struct Turn {
    using H = Heads<E, D>;
    static constexpr int PE = H::PE;
    int   lo, hi;                  // bytes of the two pieces in a head
    bool  turns;
    float c[PE], s[PE];            // of the lane's pairs

    __device__ __forceinline__ void init(const HeadsArgs &a, int32_t position)
    {
        const int j = (threadIdx.y & 63) % H::LANES, half = a.rot / PE / 2;      // the first `half` lanes of a head turn theirs
        turns = j < half;
        lo = 16 * (HALVES && turns ? j : 2 * j);
        hi = 16 * (HALVES && turns ? j + half : 2 * j + 1);
        if (turns) {
            const gcptr_t row = as_global((const void *)(a.rotation + (int64_t)position * a.rot)) + j * PE * 4;
#pragma unroll
            for (int i = 0; i < PE; i += 4) {
                widen<float>(ld16(row + i * 4), c + i);
                widen<float>(ld16(row + a.rot * 2 + i * 4), s + i);
            }
        }
    }

    // x: the lane's 2 PE elements of a head; w: their weights.  In 64 bits, rounded once.
    __device__ __forceinline__ void apply(float *x, const float *w, bool normed, double eps) const
    {
        double h[2 * PE];
#pragma unroll
        for (int i = 0; i < 2 * PE; ++i) h[i] = x[i];
        if (normed) {
            double sum = 0;
#pragma unroll
            for (int i = 0; i < 2 * PE; ++i) sum = __builtin_fma(h[i], h[i], sum);
#pragma unroll
            for (int off = H::LANES / 2; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
            const double f = 1.0 / __builtin_sqrt(sum * (1.0 / D) + eps);
#pragma unroll
            for (int i = 0; i < 2 * PE; ++i) h[i] = h[i] * f * (double)w[i];
        }
        if (turns) {
#pragma unroll
            for (int i = 0; i < PE; ++i) {
                double &a = h[HALVES ? i : 2 * i], &b = h[HALVES ? PE + i : 2 * i + 1];
                const double u = a * c[i] - b * s[i], v = b * c[i] + a * s[i];
                a = u;
                b = v;
            }
        }
#pragma unroll
        for (int i = 0; i < 2 * PE; ++i) x[i] = (float)h[i];
    }
};

// A lane's 32 consecutive bytes of a head become numbers of 4 bits: `codes`, and in the first lane of each 32 numbers their power.
template <typename E, int D> struct Mx4Put {
    using H = Heads<E, D>;
    static constexpr int N = 2 * H::PE, SHARE = MX4_BLOCK / N;    // numbers of a lane; lanes that share a power

    static __device__ __forceinline__ void put(gptr_t head, int64_t page_shift, int32_t in, float *x, bool there)
    {
        const int j = (threadIdx.y & 63) % H::LANES;
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
#pragma unroll
        for (int off = 1; off < SHARE; off <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, off, 64));
        const uint32_t power = mx4_power(top);
        const float inv = mx4_inverse(power);
        uint32_t codes[N / 8];
#pragma unroll
        for (int i = 0; i < N / 8; ++i) {
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = x[8 * i + e] * inv;
            codes[i] = mx4_pack(y);
        }
        if (!there) return;
        const gptr_t to = head + (int64_t)in * (D / 2) + j * (N / 2);
        if constexpr (N == 16) *(PREFT_GLOBAL u32x2_t *)to = u32x2_t{codes[0], codes[1]};
        else *(PREFT_GLOBAL uint32_t *)to = codes[0];
        if (j % SHARE == 0) *(PREFT_GLOBAL uint8_t *)(head + ((int64_t)(D / 2) << page_shift) + (int64_t)in * Mx4Page<D>::POWERS + j / SHARE) = (uint8_t)power;
    }
};

// what a wavefront's lanes have written to LDS is there for its other lanes
__device__ __forceinline__ void wave_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// ---------------------------------------------------------------------------------------
// n = w h / sqrt(mean(h^2) + eps), (a, b) <- (a c - b s, b c + a s), one pass: every head is read once and written once (keys twice where their rows are wanted too), so bytes bound it, and
// the 64-bit arithmetic, which puts each number on the side of a border of 4-bit numbers that the formula does, hides behind them.  A wavefront takes a row, 64 / LANES heads at a time, with
// the row's cosines and sines in registers; rows too few to fill the chip are spread over several (4096 wavefronts in all), and a single row is one launch's latency.  heads_kernel on
//   17 100 rows of 64 + 8 heads of 128, bf16, 639 MB in and out                            125-128 us, 5.0 TB/s (a copy: 4.8)
//   37 100 rows of 32 + 8 heads, values beside, keys and values to pages and keys kept     183-186 us, 5.3 TB/s
//   12 350 rows of 64 + 8 heads, values beside, to 4-bit pages                             107-110 us, 4.4 TB/s
//   one row of 32 + 8 heads                                                                2.8-3.2 us
// and whole calls of f32 rows, twice the bytes: the first 250 us, 5.1 TB/s, the second 381, 5.2, the third and the fetch of its rows 227, 4.6.
// ---------------------------------------------------------------------------------------
template <typename E, int D, int PAGES, bool HALVES>
__global__ __launch_bounds__(256) void heads_kernel(HeadsArgs a)
{
    using H = Heads<E, D>;
    constexpr int PE = H::PE;
    __shared__ __align__(16) char lds[PAGES == MX4_PAGES ? 4 * 2048 : 16];
    const int wave = threadIdx.y >> 6, lane = threadIdx.y & 63, h = lane / H::LANES, j = lane % H::LANES;
    const uint32_t task = (uint32_t)__builtin_amdgcn_readfirstlane((int32_t)(blockIdx.x * 4 + wave)), at = task / (uint32_t)a.splits;
    if (at >= (uint32_t)a.T) return;
    const int32_t row = (int32_t)at, part = (int32_t)(task - at * (uint32_t)a.splits);
    int32_t position = 0;
    if (a.positions) {
        position = as_const(a.positions)[row];
        if (position < 0) return;                             // padding
        position = min(position, a.n_positions - 1);
    }
    int64_t slot = -1;
    if constexpr (PAGES != NO_PAGES) {
        slot = as_const(a.slot_map)[row];
        if (slot >= a.n_slots) slot = -1;
    }
    const bool stored = slot >= 0;
    const int32_t in = (int32_t)(slot & (((int64_t)1 << a.page_shift) - 1));
    const int64_t head_bytes = PAGES == MX4_PAGES ? Mx4Page<D>::head_bytes(a.page_shift) : (int64_t)H::ROW << a.page_shift;
    const int64_t page = stored ? (slot >> a.page_shift) * a.kv_heads * head_bytes : 0;
    Turn<E, D, HALVES> turn;
    turn.init(a, position);
    const int32_t q_units = (a.q_heads + H::AT_ONCE - 1) / H::AT_ONCE, kv_units = (a.kv_heads + H::AT_ONCE - 1) / H::AT_ONCE;
    const int32_t units = q_units + kv_units + (PAGES != NO_PAGES ? kv_units : 0);
    for (int32_t u = part; u < units; u += a.splits) {
        if (u < q_units + kv_units) {
            const bool is_q = u < q_units;
            if (!is_q && !stored && !a.k_out) continue;
            const int32_t head = (is_q ? u : u - q_units) * H::AT_ONCE + h, heads = is_q ? a.q_heads : a.kv_heads;
            const bool there = head < heads;
            const gcptr_t from = as_global((const void *)(is_q ? a.q : a.k)) + row * (is_q ? a.ldq : a.ldk) + (int64_t)min(head, heads - 1) * H::ROW;
            const char *weight = is_q ? a.q_weight : a.k_weight;
            float x[2 * PE], w[2 * PE];
            widen<E>(ld16(from + turn.lo), x);
            widen<E>(ld16(from + turn.hi), x + PE);
            if (weight) {
                widen<E>(ld16(as_global((const void *)weight) + turn.lo), w);
                widen<E>(ld16(as_global((const void *)weight) + turn.hi), w + PE);
            }
            turn.apply(x, w, weight != nullptr, a.eps);
            const u32x4_t lo = narrow<E>(x), hi = narrow<E>(x + PE);
            char *rows = is_q ? a.q_out : a.k_out;
            if (rows && there) {
                const gptr_t to = as_global((void *)rows) + row * (is_q ? a.ldqo : a.ldko) + head * H::ROW;
                st16(to + turn.lo, lo);
                st16(to + turn.hi, hi);
            }
            if (PAGES == NO_PAGES || is_q || !stored) continue;
            const gptr_t to = as_global((void *)a.k_cache) + page + head * head_bytes;
            if constexpr (PAGES == PLAIN_PAGES) {
                if (there) {
                    st16(to + (int64_t)in * H::ROW + turn.lo, lo);
                    st16(to + (int64_t)in * H::ROW + turn.hi, hi);
                }
            } else {
                char *mine = lds + wave * 2048;               // in the order of the elements again; nobody else's
                *(u32x4_t *)(mine + h * H::ROW + turn.lo) = lo;
                *(u32x4_t *)(mine + h * H::ROW + turn.hi) = hi;
                wave_fence();
                widen<E>(*(const u32x4_t *)(mine + h * H::ROW + j * 32), x);
                widen<E>(*(const u32x4_t *)(mine + h * H::ROW + j * 32 + 16), x + PE);
                wave_fence();
                Mx4Put<E, D>::put(to, a.page_shift, in, x, there);
            }
        } else {
            if (!stored) continue;
            const int32_t head = (u - q_units - kv_units) * H::AT_ONCE + h;
            const bool there = head < a.kv_heads;
            const gcptr_t from = as_global((const void *)a.v) + row * a.ldv + (int64_t)min(head, a.kv_heads - 1) * H::ROW + j * 32;
            const u32x4_t lo = ld16(from), hi = ld16(from + 16);
            const gptr_t to = as_global((void *)a.v_cache) + page + head * head_bytes;
            if constexpr (PAGES == PLAIN_PAGES) {
                if (there) {
                    st16(to + (int64_t)in * H::ROW + j * 32, lo);
                    st16(to + (int64_t)in * H::ROW + j * 32 + 16, hi);
                }
            } else if constexpr (PAGES == MX4_PAGES) {
                float x[2 * PE];
                widen<E>(lo, x);
                widen<E>(hi, x + PE);
                Mx4Put<E, D>::put(to, a.page_shift, in, x, there);
            }
        }
    }
}

struct FetchArgs {
    char *k, *v;
    const char *k_cache, *v_cache;
    const int64_t *slot_map;
    int64_t ldk, ldv, n_slots;               // ld: bytes
    int32_t T, kv_heads, page_shift;
};

// A wavefront takes a row of keys or values, 64 / LANES heads at a time, a lane 32 bytes of what it writes: bound by these (12 350 rows of 8 heads of 128, keys and values, bf16: 16 us, 4.0 TB/s;
// 224 rows 2.6 us).
template <typename E, int D>
__global__ __launch_bounds__(256) void mx4_fetch_kernel(FetchArgs a)
{
    using H = Heads<E, D>;
    constexpr int N = 2 * H::PE, SHARE = MX4_BLOCK / N;
    const int lane = threadIdx.y & 63, h = lane / H::LANES, j = lane % H::LANES;
    const uint32_t at = (uint32_t)__builtin_amdgcn_readfirstlane((int32_t)(blockIdx.x * 4 + (threadIdx.y >> 6)));
    if (at >= (uint32_t)a.T) return;
    const int32_t row = (int32_t)at;
    const int64_t slot = as_const(a.slot_map)[row];
    if (slot < 0 || slot >= a.n_slots) return;
    const int32_t in = (int32_t)(slot & (((int64_t)1 << a.page_shift) - 1));
    const int64_t head_bytes = Mx4Page<D>::head_bytes(a.page_shift), page = (slot >> a.page_shift) * a.kv_heads * head_bytes;
    const gcptr_t cache = as_global((const void *)(blockIdx.y ? a.v_cache : a.k_cache)) + page;
    const gptr_t rows = as_global((void *)(blockIdx.y ? a.v : a.k)) + row * (blockIdx.y ? a.ldv : a.ldk);
    for (int32_t head = h; head < a.kv_heads; head += H::AT_ONCE) {
        const gcptr_t from = cache + head * head_bytes;
        const gcptr_t numbers = from + (int64_t)in * (D / 2) + j * (N / 2);
        const float scale = mx4_scale(*(const PREFT_GLOBAL uint8_t *)(from + ((int64_t)(D / 2) << a.page_shift) + (int64_t)in * Mx4Page<D>::POWERS + j / SHARE));
        const gptr_t to = rows + head * H::ROW + j * 32;
        if constexpr (sizeof(E) == 2) {
            const u32x2_t c = ld8(numbers);
            st16(to, mx4_bf16(c[0], scale));
            st16(to + 16, mx4_bf16(c[1], scale));
        } else {
            const uint32_t c = ld4(numbers);
            const u32x4_t v = mx4_bf16(c, scale);
            st16(to, u32x4_t{v[0] << 16, v[0] & 0xffff0000u, v[1] << 16, v[1] & 0xffff0000u});
            st16(to + 16, u32x4_t{v[2] << 16, v[2] & 0xffff0000u, v[3] << 16, v[3] & 0xffff0000u});
        }
    }
}

template <int PAGES, bool HALVES>
int launch_heads(const HeadsArgs &a, int dtype, int32_t head_dim, hipStream_t st)
{
    const dim3 grid((unsigned)(((int64_t)a.T * a.splits + 3) / 4)), block = row_threads();
    if (dtype == PREFT_BF16) {
        if (head_dim == 128) hipLaunchKernelGGL((heads_kernel<__bf16, 128, PAGES, HALVES>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((heads_kernel<__bf16, 64, PAGES, HALVES>), grid, block, 0, st, a);
    } else {
        if (head_dim == 128) hipLaunchKernelGGL((heads_kernel<float, 128, PAGES, HALVES>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((heads_kernel<float, 64, PAGES, HALVES>), grid, block, 0, st, a);
    }
    return launched();
}

// Rows that a call writes over its own input do so in place; any other overlap is refused.
bool in_place(const void *out, int64_t ldo, const void *in, int64_t ldi) { return out == in && ldo == ldi; }

struct Rows { const void *p; int64_t ld, width; };
bool apart(const Rows &a, const Rows &b, int64_t T, int dtype) { return !a.p || !b.p || !rows_meet(a.p, a.ld, a.width, b.p, b.ld, b.width, T, dtype); }

int run_heads(Pages pages, void *k_cache, void *v_cache, int32_t n_pages, int32_t page_size, void *q_out, int64_t ldqo, const void *q, int64_t ldq, void *k_out,
              int64_t ldko, const void *k, int64_t ldk, const void *v, int64_t ldv, int32_t T, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
              const int64_t *slot_map, const void *q_weight, const void *k_weight, float eps, const int32_t *positions, const float *rotation, int32_t n_positions,
              int32_t rotary_dim, int pairs, int dtype, void *stream)
{
    if (T < 0 || n_pages < 0 || n_heads < 0 || n_heads > PREFT_MAX_HEADS || n_kv_heads < 0 || n_kv_heads > PREFT_MAX_HEADS) return PREFT_EINVAL;
    if (dtype != PREFT_F32 && dtype != PREFT_BF16) return PREFT_EINVAL;
    if (pairs != PREFT_PAIRS_HALVES && pairs != PREFT_PAIRS_ADJACENT) return PREFT_EINVAL;
    if (!(eps >= 0.0f) || !std::isfinite(eps)) return PREFT_EINVAL;
    if (head_dim != 64 && head_dim != 128) return PREFT_EUNSUPPORTED;
    if (rotary_dim < 0 || rotary_dim > head_dim) return PREFT_EINVAL;
    if (rotary_dim % 16 != 0) return PREFT_EUNSUPPORTED;
    const int shift = pages == NO_PAGES ? 0 : page_shift_of(page_size);
    if (shift < 0) return PREFT_EUNSUPPORTED;
    if (pages != NO_PAGES && n_kv_heads == 0) return PREFT_EINVAL;
    if (T == 0) return PREFT_OK;
    if (rotary_dim > 0 && (!positions || !rotation || n_positions < 1)) return PREFT_EINVAL;
    const int64_t wq = (int64_t)n_heads * head_dim, wk = (int64_t)n_kv_heads * head_dim, e = elem_bytes(dtype);
    int rc;
    if (n_heads > 0 && ((rc = check_rows(q_out, ldqo, wq, dtype)) != PREFT_OK || (rc = check_rows(q, ldq, wq, dtype)) != PREFT_OK)) return rc;
    if (n_kv_heads > 0 && (rc = check_rows(k, ldk, wk, dtype)) != PREFT_OK) return rc;
    if (n_kv_heads > 0 && (k_out || pages == NO_PAGES) && (rc = check_rows(k_out, ldko, wk, dtype)) != PREFT_OK) return rc;
    if (pages != NO_PAGES && (rc = check_rows(v, ldv, wk, dtype)) != PREFT_OK) return rc;
    if (((reinterpret_cast<uintptr_t>(q_weight) | reinterpret_cast<uintptr_t>(k_weight) | (rotary_dim > 0 ? reinterpret_cast<uintptr_t>(rotation) : 0)) & 15) != 0)
        return PREFT_EALIGN;
    const Rows qo = {n_heads > 0 ? q_out : nullptr, ldqo, wq}, qi = {n_heads > 0 ? q : nullptr, ldq, wq}, ko = {n_kv_heads > 0 ? k_out : nullptr, ldko, wk},
               ki = {n_kv_heads > 0 ? k : nullptr, ldk, wk}, vi = {pages != NO_PAGES ? v : nullptr, ldv, wk};
    if (!apart(qo, ko, T, dtype) || !apart(qo, ki, T, dtype) || !apart(qo, vi, T, dtype) || !apart(ko, qi, T, dtype) || !apart(ko, vi, T, dtype)) return PREFT_EINVAL;
    if (qo.p && !in_place(q_out, ldqo, q, ldq) && !apart(qo, qi, T, dtype)) return PREFT_EINVAL;
    if (ko.p && !in_place(k_out, ldko, k, ldk) && !apart(ko, ki, T, dtype)) return PREFT_EINVAL;
    HeadsArgs a = {};
    if (pages != NO_PAGES) {
        if (!slot_map || (n_pages > 0 && (!k_cache || !v_cache))) return PREFT_EINVAL;
        if (((reinterpret_cast<uintptr_t>(k_cache) | reinterpret_cast<uintptr_t>(v_cache)) & 15) != 0) return PREFT_EALIGN;
        const int64_t token = pages == MX4_PAGES ? head_dim / 2 + head_dim / MX4_BLOCK : head_dim * e;
        const int64_t cache = (int64_t)n_pages * page_size * n_kv_heads * token;
        const Span caches[2] = {{k_cache, cache}, {v_cache, cache}};
        if (n_pages > 0 && caches[0].meets(caches[1])) return PREFT_EINVAL;
        for (const Span &c : caches)
            for (const Rows &r : {qo, qi, ko, ki, vi})
                if (n_pages > 0 && r.p && c.meets({r.p, ((int64_t)(T - 1) * r.ld + r.width) * e})) return PREFT_EINVAL;
        a.n_slots = (int64_t)n_pages * page_size;
    }
    a.q = (const char *)q; a.k = (const char *)k; a.v = (const char *)v; a.q_weight = (const char *)q_weight; a.k_weight = (const char *)k_weight;
    a.q_out = (char *)q_out; a.k_out = (char *)k_out; a.k_cache = (char *)k_cache; a.v_cache = (char *)v_cache;
    a.ldq = ldq * e; a.ldk = ldk * e; a.ldv = ldv * e; a.ldqo = ldqo * e; a.ldko = ldko * e;
    a.positions = positions; a.slot_map = slot_map; a.rotation = rotation; a.eps = eps;
    a.T = T; a.q_heads = n_heads; a.kv_heads = n_kv_heads; a.n_positions = n_positions; a.rot = rotary_dim; a.page_shift = shift;
    const int64_t at_once = 64 / (head_dim * e / 32), units = (n_heads + at_once - 1) / at_once + (n_kv_heads + at_once - 1) / at_once * (pages == NO_PAGES ? 1 : 2);
    if (units == 0) return PREFT_OK;
    // a row's heads are spread over wavefronts where rows are too few to fill the chip
    int64_t splits = 4096 / T;
    a.splits = (int32_t)(splits < 1 ? 1 : splits > units ? units : splits);
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    const bool halves = pairs == PREFT_PAIRS_HALVES;
    switch (pages) {
    case NO_PAGES: return halves ? launch_heads<NO_PAGES, true>(a, dtype, head_dim, st) : launch_heads<NO_PAGES, false>(a, dtype, head_dim, st);
    case PLAIN_PAGES: return halves ? launch_heads<PLAIN_PAGES, true>(a, dtype, head_dim, st) : launch_heads<PLAIN_PAGES, false>(a, dtype, head_dim, st);
    default: return halves ? launch_heads<MX4_PAGES, true>(a, dtype, head_dim, st) : launch_heads<MX4_PAGES, false>(a, dtype, head_dim, st);
    }
}

}  // namespace

extern "C" {

int preft_qk_rotate(void *q_out, int64_t ldqo, const void *q, int64_t ldq, void *k_out, int64_t ldko, const void *k, int64_t ldk, int32_t T, int32_t n_heads,
                    int32_t n_kv_heads, int32_t head_dim, const void *q_weight, const void *k_weight, float eps, const int32_t *positions, const float *rotation,
                    int32_t n_positions, int32_t rotary_dim, int pairs, int dtype, void *stream)
{
    return run_heads(NO_PAGES, nullptr, nullptr, 0, 0, q_out, ldqo, q, ldq, k_out, ldko, k, ldk, nullptr, 0, T, n_heads, n_kv_heads, head_dim, nullptr, q_weight, k_weight,
                     eps, positions, rotation, n_positions, rotary_dim, pairs, dtype, stream);
}

int preft_kv_append(void *k_cache, void *v_cache, int32_t n_pages, int32_t page_size, void *q_out, int64_t ldqo, const void *q, int64_t ldq, void *k_out, int64_t ldko,
                    const void *k, int64_t ldk, const void *v, int64_t ldv, int32_t T, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, const int64_t *slot_map,
                    const void *q_weight, const void *k_weight, float eps, const int32_t *positions, const float *rotation, int32_t n_positions, int32_t rotary_dim,
                    int pairs, int dtype, void *stream)
{
    return run_heads(PLAIN_PAGES, k_cache, v_cache, n_pages, page_size, q_out, ldqo, q, ldq, k_out, ldko, k, ldk, v, ldv, T, n_heads, n_kv_heads, head_dim, slot_map,
                     q_weight, k_weight, eps, positions, rotation, n_positions, rotary_dim, pairs, dtype, stream);
}

int preft_kv_append_mx(void *k_cache, void *v_cache, int32_t n_pages, int32_t page_size, void *q_out, int64_t ldqo, const void *q, int64_t ldq, void *k_out,
                        int64_t ldko, const void *k, int64_t ldk, const void *v, int64_t ldv, int32_t T, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                        const int64_t *slot_map, const void *q_weight, const void *k_weight, float eps, const int32_t *positions, const float *rotation,
                        int32_t n_positions, int32_t rotary_dim, int pairs, int dtype, void *stream)
{
    return run_heads(MX4_PAGES, k_cache, v_cache, n_pages, page_size, q_out, ldqo, q, ldq, k_out, ldko, k, ldk, v, ldv, T, n_heads, n_kv_heads, head_dim, slot_map,
                     q_weight, k_weight, eps, positions, rotation, n_positions, rotary_dim, pairs, dtype, stream);
}

int preft_kv_fetch_mx(void *k, int64_t ldk, void *v, int64_t ldv, int32_t T, int32_t n_kv_heads, int32_t head_dim, const int64_t *slot_map, const void *k_cache,
                       const void *v_cache, int32_t n_pages, int32_t page_size, int dtype, void *stream)
{
    if (T < 0 || n_pages < 0) return PREFT_EINVAL;
    const int shift = page_shift_of(page_size);
    int rc = check_heads(n_kv_heads, n_kv_heads, head_dim, dtype);
    if (rc != PREFT_OK) return rc;
    if (shift < 0) return PREFT_EUNSUPPORTED;
    if (T == 0) return PREFT_OK;
    if (!slot_map) return PREFT_EINVAL;
    const int64_t width = (int64_t)n_kv_heads * head_dim, e = elem_bytes(dtype);
    if ((rc = check_rows(k, ldk, width, dtype)) != PREFT_OK || (rc = check_rows(v, ldv, width, dtype)) != PREFT_OK) return rc;
    if (rows_meet(k, ldk, width, v, ldv, width, T, dtype)) return PREFT_EINVAL;
    if (n_pages == 0) return PREFT_OK;                 // no slot exists: nothing is written
    if (!k_cache || !v_cache) return PREFT_EINVAL;
    if (((reinterpret_cast<uintptr_t>(k_cache) | reinterpret_cast<uintptr_t>(v_cache)) & 15) != 0) return PREFT_EALIGN;
    const int64_t cache = (int64_t)n_pages * page_size * n_kv_heads * (head_dim / 2 + head_dim / MX4_BLOCK);
    for (const Span &o : {Span{k, ((int64_t)(T - 1) * ldk + width) * e}, Span{v, ((int64_t)(T - 1) * ldv + width) * e}})
        if (o.meets({k_cache, cache}) || o.meets({v_cache, cache})) return PREFT_EINVAL;
    FetchArgs a;
    a.k = (char *)k; a.v = (char *)v; a.k_cache = (const char *)k_cache; a.v_cache = (const char *)v_cache; a.slot_map = slot_map;
    a.ldk = ldk * e; a.ldv = ldv * e; a.n_slots = (int64_t)n_pages * page_size; a.T = T; a.kv_heads = n_kv_heads; a.page_shift = shift;
    const dim3 grid((unsigned)(((int64_t)T + 3) / 4), 2), block = row_threads();
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    if (dtype == PREFT_BF16) {
        if (head_dim == 128) hipLaunchKernelGGL((mx4_fetch_kernel<__bf16, 128>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((mx4_fetch_kernel<__bf16, 64>), grid, block, 0, st, a);
    } else {
        if (head_dim == 128) hipLaunchKernelGGL((mx4_fetch_kernel<float, 128>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((mx4_fetch_kernel<float, 64>), grid, block, 0, st, a);
    }
    return launched();
}

}  // extern "C"
