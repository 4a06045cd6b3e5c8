// Attention of query columns over keys that stand in packed rows or in cache pages, and the join of parts.
//
//   out = sum_j p_j v_j / sum_j p_j,   p_j = 2^(c q.k_j - m),   c = scale log2(e),   m >= the largest exponent - 8
//
// One pass over the keys with a running m and running sums.  Products are taken transposed, S^T = K Q^T and O^T = V^T P^T, in 32x32 matrix
// instructions: a lane then holds 16 keys of ONE query column (the other 16 are in the lane 32 further on), so that the largest of a column
// is 15 comparisons in a lane and one exchange, the sums of the two lanes meet only at the end, and the registers that hold S^T are, rounded, the right operand
// of the second product as they stand: its contraction runs over keys in whatever order, and V^T is read from LDS in the order the lanes hold
// the keys (ds_read_b64_tr_b16 turns 4 keys x 16 dimensions for bf16).
// m is raised only when a tile exceeds it by more than 8: p stays below 2^8, which costs no accuracy in floating point, and the O^T of 64 registers
// is rarely rescaled.  All sums are 32-bit; bf16 P is rounded to nearest even (the matrix cores take no other operand beside bf16 V, and P as head and remainder would be half
// as many products again: outputs are off by 0.18-0.23 % of their norm, 0.15-0.17 % of it their own rounding), the sum of P is taken before that.
//
// Keys that a column may not see: their S is set to -inf whatever it was.  Their V meets P = 0, and 0 * inf is NaN: in the tiles where some column
// does not see some key, rows of V that no column sees are zeroed in LDS, and where a row that some see holds an infinity or a NaN the tile's
// second product is done column by column instead (attend_careful).
#pragma once
#include "attention_schedule.hpp"

namespace preft {

typedef float f32x16_t __attribute__((ext_vector_type(16)));
#define PREFT_LDS __attribute__((address_space(3)))
typedef PREFT_LDS char *lds_t;

struct AttnArgs {
    AttnScheduleArgs s;               // sizes, tables and lists
    const void *q, *k, *v;            // k, v: packed rows, or the cache
    void *out;
    int64_t ldq, ldk, ldv, ldo;       // bytes
    const int32_t *table;
    int64_t ld_table;
    int32_t n_pages, page_shift;
    float scale_log2;
    uint32_t per_head;                // ceil(2^21 / G): x / G = x per_head >> 21 for x < 2048 (G <= 1024)
    int32_t ready;                    // direct calls: the header is there already
};

constexpr float ATTN_LOWEST = -3.0e38f;   // below every score's exponent, and finite: 2^(-inf - it) is 0, not NaN

template <typename E, int D> struct AttnTile {
    static constexpr int ELEM = sizeof(E);
    static constexpr int ROW = D * ELEM;                  // bytes of a key's row
    static constexpr int PIECES = ROW / 16;
    static constexpr int ROWS_PER_COPY = 64 / PIECES;     // rows that one copy of a wavefront (64 x 16 bytes) brings
    static constexpr int STEPS = PIECES / 2;              // products of 16 bytes per lane over a row
    static constexpr int BLOCKS = D / 32;
    static constexpr int TILE = ATTN_KEYS * ROW;
    static constexpr int LDS = 4 * TILE;                  // K and V, two tiles each; or K and V of 32 keys for every wavefront.  (f32 heads of 128: 132 KB, one workgroup a compute unit)
    // Pieces of 16 bytes are exchanged within a row so that what LDS reads in one cycle, 256 bytes, comes from all 64 banks: 16 lanes' 16 bytes of one piece of
    // 16 rows of K; 32 lanes' 8 bytes of four pieces of 4 rows of V (bf16), or 128 bytes each of two rows 4 apart (f32).
    static __device__ __forceinline__ int k_turn(int row) { return PIECES < 16 ? (row >> 1) & 7 : row & 15; }
    static __device__ __forceinline__ int v_turn(int row)
    {
        if constexpr (ELEM == 4) return 8 * ((row >> 2) & 1);
        else return PIECES >= 16 ? 4 * (row & 3) : 4 * ((row >> 1) & 1);
    }
};

__device__ __forceinline__ uint32_t lds_address(lds_t p) { return (uint32_t)(uintptr_t)p; }

// 64 x 16 bytes from base + each lane's offset to LDS, lane after lane.  Written out because the compiler would wait for every copy in flight before any
// read of LDS; the waits are in the loops below.  The copies have no register as output.
__device__ __forceinline__ void copy_to_lds(uint32_t to, const char *base, uint32_t offset)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(offset), "s"(base) : "memory");
}
template <int N> __device__ __forceinline__ void wait_copies() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
__device__ __forceinline__ void wait_lds_reads() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

__device__ __forceinline__ int32_t uniform(int32_t v) { return __builtin_amdgcn_readfirstlane(v); }

__device__ __forceinline__ float other_half_max(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float both_halves_sum(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// ---------------------------------------------------------------------------------------
// where the rows of a key come from
// ---------------------------------------------------------------------------------------
template <typename E, int D, bool PAGED> struct AttnSource {
    using X = AttnTile<E, D>;
    const char *k, *v;                 // of this key/value head
    int64_t ldk, ldv;
    const int32_t *table;
    int32_t last;                      // the last key there is
    int32_t n_pages, page_shift;
    int64_t page_bytes;
    int32_t ids, ids_first;            // 64 page numbers from table[ids_first] on, one a lane

    __device__ __forceinline__ void init(const AttnArgs &a, const AttnUnit &u, int head)
    {
        last = max(u.key1 - 1, 0);
        if constexpr (PAGED) {
            page_shift = a.page_shift;
            n_pages = a.n_pages;
            page_bytes = ((int64_t)a.s.kv_heads * X::ROW) << page_shift;
            k = (const char *)a.k + (((int64_t)head * X::ROW) << page_shift);
            v = (const char *)a.v + (((int64_t)head * X::ROW) << page_shift);
            table = a.table + (int64_t)u.table * a.ld_table;
            ids_first = -64;
        } else {
            k = (const char *)a.k + (int64_t)u.table * a.ldk + head * X::ROW;
            v = (const char *)a.v + (int64_t)u.table * a.ldv + head * X::ROW;
            ldk = a.ldk; ldv = a.ldv;
        }
    }

    // the page of `key` (uniform, not past the last), as the block table names it; outside the pool: its first or last page
    __device__ __forceinline__ int64_t page_of(int32_t key)
    {
        const int32_t i = key >> page_shift;
        if (i - ids_first >= 64 || i < ids_first) {
            ids_first = i;
            ids = table[min(i + (int32_t)(threadIdx.x & 63), last >> page_shift)];
        }
        const uint32_t id = (uint32_t)__builtin_amdgcn_readlane(ids, i - ids_first);
        return min(id, (uint32_t)(n_pages - 1));
    }

    // Copies COPIES x ROWS_PER_COPY rows of K or V, from `key` on, to `to`; `row0`: place of the first in its tile.  ROWS_PER_COPY divides both.
    template <bool V, int COPIES>
    __device__ __forceinline__ void copy(uint32_t to, int32_t key, int row0)
    {
        const int lane = threadIdx.x & 63, r = lane / X::PIECES, c = lane % X::PIECES;
        if constexpr (PAGED) {
            const char *base = nullptr;
#pragma unroll
            for (int i = 0; i < COPIES; ++i) {
                const int32_t at = key + i * X::ROWS_PER_COPY;
                const int turn = V ? X::v_turn(row0 + i * X::ROWS_PER_COPY + r) : X::k_turn(row0 + i * X::ROWS_PER_COPY + r);
                if (i == 0 || (at & ((1 << page_shift) - 1)) == 0) {       // another page; past the last key: the last key's page
                    const int32_t in = at & ((1 << page_shift) - 1);
                    base = (V ? v : k) + page_of(min(at, last)) * page_bytes + in * X::ROW;
                } else {
                    base += X::ROWS_PER_COPY * X::ROW;
                }
                copy_to_lds(to + i * 1024, base, (uint32_t)(r * X::ROW + ((c ^ turn) << 4)));
            }
        } else {
            const int64_t ld = V ? ldv : ldk;
            const int32_t first = min(key, last), most = last - first;     // rows past the last: the last again
            const char *base = (V ? v : k) + first * ld;
#pragma unroll
            for (int i = 0; i < COPIES; ++i) {
                const int row = i * X::ROWS_PER_COPY + r;
                const int turn = V ? X::v_turn(row0 + row) : X::k_turn(row0 + row);
                copy_to_lds(to + i * 1024, base, (uint32_t)(min(row, most) * (int32_t)ld + ((c ^ turn) << 4)));
            }
        }
    }
};

// ---------------------------------------------------------------------------------------
// 32 columns of a wavefront
// ---------------------------------------------------------------------------------------
template <typename E, int D> struct AttnColumns {
    using X = AttnTile<E, D>;
    u32x4_t  q[X::STEPS];
    f32x16_t o[X::BLOCKS];
    float    m, l;                    // l: of this lane's keys
    int32_t  lim;                     // this lane's column sees keys below it
    int32_t  row, head;               // of the query
    bool     valid;

    __device__ __forceinline__ void init(const AttnArgs &a, const AttnUnit &u, int kv_head, int first)
    {
        const int lane = threadIdx.x & 63, half = lane >> 5, col = first + (lane & 31), G = a.s.group;
        valid = col < u.ncols;
        const int32_t x = u.head0 + min(col, u.ncols - 1), i = (int32_t)((uint32_t)x * a.per_head >> 21);
        head = kv_head * G + (x - i * G);
        if (u.row0 >= 0) {
            row = u.row0 + i;
            lim = u.lim0 + i;
        } else {
            const int2 r = a.s.l.group_rows[min(-1 - u.row0 + i, a.s.l.group_row_cap - 1)];
            row = r.x;
            lim = r.y;
        }
        row = max(0, min(row, a.s.T - 1));
        lim = min(lim, u.key1);
        const gcptr_t from = as_global((const char *)a.q + (int64_t)row * a.ldq + head * X::ROW + half * 16);
#pragma unroll
        for (int s = 0; s < X::STEPS; ++s) q[s] = ld16(from + s * 32);
#pragma unroll
        for (int b = 0; b < X::BLOCKS; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[b][r] = 0.0f;
        m = ATTN_LOWEST;
        l = 0.0f;
    }

    // The queries are there: the compiler, which does not know of the copies in flight, would else wait for them in every turn of a loop.
    __device__ __forceinline__ void arrived()
    {
#pragma unroll
        for (int s = 0; s < X::STEPS; ++s) asm volatile("" : "+v"(q[s]));
    }

    // S^T of 32 keys from row `row0` of the K tile on
    __device__ __forceinline__ f32x16_t scores(lds_t tile, int row0) const
    {
        const int lane = threadIdx.x & 63, half = lane >> 5, r = lane & 31;
        const lds_t at = tile + (row0 + r) * X::ROW;
        const int turn = X::k_turn(r);
        f32x16_t s;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.0f;
#pragma unroll
        for (int t = 0; t < X::STEPS; ++t) {
            const u32x4_t k = *(const PREFT_LDS u32x4_t *)(at + (((2 * t + half) ^ turn) << 4));
            if constexpr (sizeof(E) == 2) {
                s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, k), __builtin_bit_cast(bf16x8_t, q[t]), s, 0, 0, 0);
            } else {
                const f32x4_t kf = __builtin_bit_cast(f32x4_t, k), qf = __builtin_bit_cast(f32x4_t, q[t]);
#pragma unroll
                for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[e], qf[e], s, 0, 0, 0);
            }
        }
        return s;
    }

    // the keys of register i of a block of 32: 8 (i / 4) + 4 half + i % 4
    __device__ __forceinline__ void hide(f32x16_t &s, int32_t key, int32_t key0) const
    {
        const int32_t at = key + 4 * ((threadIdx.x & 63) >> 5), n = lim - at;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 8 * (i / 4) + i % 4 < n ? s[i] : -INFINITY;
        if (key < key0) {
            const int32_t from = key0 - at;
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = 8 * (i / 4) + i % 4 >= from ? s[i] : -INFINITY;
        }
    }

    // S^T -> P^T in place, N blocks of 32 keys
    template <int N>
    __device__ __forceinline__ void exponentials(f32x16_t (&s)[N], float c)
    {
        float top = s[0][0];
#pragma unroll
        for (int b = 0; b < N; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, s[b][i]);
        top = other_half_max(top) * c;
        if (__any(top > m + 8.0f)) {
            const float to = fmaxf(m, top), f = __builtin_amdgcn_exp2f(m - to);
            m = to;
            l *= f;
#pragma unroll
            for (int b = 0; b < X::BLOCKS; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[b][r] *= f;
        }
#pragma unroll
        for (int b = 0; b < N; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[b][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][i], c, -m));
                l += s[b][i];
            }
    }

    // O^T += V^T P^T over 32 keys from row `row0` of the V tile on
    __device__ __forceinline__ void add(lds_t tile, int row0, const f32x16_t &p)
    {
        const int lane = threadIdx.x & 63, half = lane >> 5;
        if constexpr (sizeof(E) == 2) {
            const int i = lane & 15, key = 4 * half + (i >> 2), turn = X::v_turn(key);
            const lds_t at = tile + (row0 + key) * X::ROW + (i & 1) * 8;
            const int piece = ((lane >> 4) & 1) * 2 + ((i & 3) >> 1);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                union { uint32_t w[4]; bf16x8_t v; } pb;
#pragma unroll
                for (int w = 0; w < 4; ++w) pb.w[w] = pack_bf16(p[8 * h + 2 * w], p[8 * h + 2 * w + 1]);
#pragma unroll
                for (int b = 0; b < X::BLOCKS; ++b) {
                    const lds_t from = at + 16 * h * X::ROW + (((b * 4 + piece) ^ turn) << 4);
                    const bf16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((PREFT_LDS bf16x4_t *)from);
                    const bf16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((PREFT_LDS bf16x4_t *)(from + 8 * X::ROW));
                    const bf16x8_t v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                    o[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, pb.v, o[b], 0, 0, 0);
                }
            }
        } else {
            const int d = lane & 31;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int key = 8 * (i / 4) + 4 * half + i % 4;
                const lds_t at = tile + (row0 + key) * X::ROW + (d & 3) * 4;
#pragma unroll
                for (int b = 0; b < X::BLOCKS; ++b) {
                    const float v = *(const PREFT_LDS float *)(at + (((b * 8 + (d >> 2)) ^ (8 * half)) << 4));
                    o[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, p[i], o[b], 0, 0, 0);
                }
            }
        }
    }

    // The same, key after key: a key that a column does not see adds nothing to it, whatever its V is.  `scratch`: 32 x 32 values of this wavefront.
    __device__ __forceinline__ void careful(lds_t tile, int row0, const f32x16_t &p, lds_t scratch, int32_t key, int32_t key0)
    {
        const int lane = threadIdx.x & 63, half = lane >> 5;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int at = (8 * (i / 4) + 4 * half + i % 4) * 32 + (lane & 31);
            if constexpr (sizeof(E) == 2) ((PREFT_LDS __bf16 *)scratch)[at] = (__bf16)p[i];
            else ((PREFT_LDS float *)scratch)[at] = p[i];
        }
        wait_lds_reads();
        const int32_t from = max(key0 - key, 0), to = min(lim - key, 32);
#pragma unroll
        for (int b = 0; b < X::BLOCKS; ++b) {
            f32x16_t sum;
#pragma unroll
            for (int i = 0; i < 16; ++i) sum[i] = 0.0f;
            for (int j = 0; j < 32; ++j) {
                if (j < from || j >= to) continue;
                float w;
                if constexpr (sizeof(E) == 2) w = (float)((const PREFT_LDS __bf16 *)scratch)[j * 32 + (lane & 31)];
                else w = ((const PREFT_LDS float *)scratch)[j * 32 + (lane & 31)];
                const int turn = X::v_turn(row0 + j);
#pragma unroll
                for (int i = 0; i < 4; ++i) {                     // dimensions 32 b + 8 i + 4 half ..
                    const int byte = (b * 32 + 8 * i + 4 * half) * X::ELEM;
                    const lds_t at = tile + (row0 + j) * X::ROW + (((byte >> 4) ^ turn) << 4) + (byte & 15);
                    if constexpr (sizeof(E) == 2) {
                        const u32x2_t v = *(const PREFT_LDS u32x2_t *)at;
                        sum[4 * i] += w * bf16_lo(v.x);
                        sum[4 * i + 1] += w * bf16_hi(v.x);
                        sum[4 * i + 2] += w * bf16_lo(v.y);
                        sum[4 * i + 3] += w * bf16_hi(v.y);
                    } else {
                        const f32x4_t v = *(const PREFT_LDS f32x4_t *)at;
#pragma unroll
                        for (int e = 0; e < 4; ++e) sum[4 * i + e] += w * v[e];
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) o[b][i] += sum[i];
        }
    }
};

// 16 bytes of a V row hold an infinity or a NaN: an exponent of ones is the largest there is
typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));
template <typename E> __device__ __forceinline__ bool not_finite(u32x4_t v)
{
    if constexpr (sizeof(E) == 2) {
        u16x2_t top = __builtin_bit_cast(u16x2_t, v[0] & 0x7fff7fffu);
#pragma unroll
        for (int i = 1; i < 4; ++i) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2_t, v[i] & 0x7fff7fffu));
        return max(top.x, top.y) >= 0x7f80;
    } else {
        const uint32_t top = max(max(v[0] & 0x7fffffffu, v[1] & 0x7fffffffu), max(v[2] & 0x7fffffffu, v[3] & 0x7fffffffu));
        return top >= 0x7f800000u;
    }
}

// Rows of a V tile that no column sees become zero; says whether a row that only some see is not finite.  PIECES_EACH pieces of 16 bytes from `tid`
// on, `step` apart.
template <typename E, int D, int PIECES_EACH>
__device__ __forceinline__ bool clean_rows(lds_t tile, int32_t key, int32_t key0, int32_t low, int32_t high, int tid, int step)
{
    using X = AttnTile<E, D>;
    u32x4_t v[PIECES_EACH];
#pragma unroll
    for (int k = 0; k < PIECES_EACH; ++k) v[k] = *(PREFT_LDS u32x4_t *)(tile + (tid + k * step) * 16);
    bool bad = false;
#pragma unroll
    for (int k = 0; k < PIECES_EACH; ++k) {
        const int32_t j = key + (tid + k * step) / X::PIECES;
        if (j < key0 || j >= high) *(PREFT_LDS u32x4_t *)(tile + (tid + k * step) * 16) = u32x4_t{0, 0, 0, 0};
        else if (j >= low) bad = bad || not_finite<E>(v[k]);
    }
    return bad;
}

// four consecutive elements of a result row
template <typename E> __device__ __forceinline__ void store4(gptr_t p, float a, float b, float c, float d)
{
    if constexpr (sizeof(E) == 2) *reinterpret_cast<PREFT_GLOBAL u32x2_t *>(p) = u32x2_t{pack_bf16(a, b), pack_bf16(c, d)};
    else *reinterpret_cast<PREFT_GLOBAL f32x4_t *>(p) = f32x4_t{a, b, c, d};
}
__device__ __forceinline__ float inverse(float l) { return l == 0.0f ? 0.0f : 1.0f / l; }   // a row that sees no key is zero

// The results of a wavefront's 32 columns, or their part.
template <typename E, int D>
__device__ __forceinline__ void write_columns(const AttnArgs &a, const AttnUnit &u, AttnColumns<E, D> &w, int kv_head, int first)
{
    using X = AttnTile<E, D>;
    const int lane = threadIdx.x & 63, half = lane >> 5;
    const float l = both_halves_sum(w.l);
    if (u.slot < 0) {
        const float f = inverse(l);
        const gptr_t to = as_global((char *)a.out + (int64_t)w.row * a.ldo + w.head * X::ROW + half * (X::ELEM == 2 ? 16 : 4 * X::ELEM));
#pragma unroll
        for (int b = 0; b < X::BLOCKS; ++b) {
            if constexpr (X::ELEM == 2) {                         // the two lanes of a column trade halves: 16 bytes each, of consecutive dimensions
#pragma unroll
                for (int r = 0; r < 4; r += 2) {
                    u32x4_t v;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const auto x = __builtin_amdgcn_permlane32_swap(pack_bf16(w.o[b][4 * r + 2 * e] * f, w.o[b][4 * r + 2 * e + 1] * f),
                                                                        pack_bf16(w.o[b][4 * r + 4 + 2 * e] * f, w.o[b][4 * r + 5 + 2 * e] * f), false, false);
                        v[e] = x[0];
                        v[2 + e] = x[1];
                    }
                    if (w.valid) st16(to + (b * 32 + 8 * r) * X::ELEM, v);
                }
            } else {
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (w.valid) store4<E>(to + (b * 32 + 8 * r) * X::ELEM, w.o[b][4 * r] * f, w.o[b][4 * r + 1] * f, w.o[b][4 * r + 2] * f, w.o[b][4 * r + 3] * f);
            }
        }
    } else if (w.valid) {
        const int64_t part = (int64_t)u.slot + kv_head * u.ncols + first + (lane & 31);
        const gptr_t to = as_global((void *)(a.s.l.part_o + part * D + half * 4));
#pragma unroll
        for (int b = 0; b < X::BLOCKS; ++b)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                store4<float>(to + (b * 32 + 8 * r) * 4, w.o[b][4 * r], w.o[b][4 * r + 1], w.o[b][4 * r + 2], w.o[b][4 * r + 3]);
        if (half == 0) a.s.l.part_ml[part] = make_float2(w.m, l);
    }
}

// ---------------------------------------------------------------------------------------
// A unit of more than 32 columns: every wavefront has 32 of them, and all read the tiles of 64 keys that the workgroup brings to LDS, one
// tile ahead.  Two workgroups share a compute unit (registers allow no third): 0.93 us a tile and unit, 1.21 with one.  One prompt of 16 001 rows, 64 heads over 8 of 128:
// 3.83 ms, 1100 TFLOP/s, 90 % of what a large matrix product of the library reaches (power holds the clock of both at about 1.6 GHz).  Prompts of a thousand rows:
// 650 TFLOP/s; 10 us of a workgroup's 28 go into finding its queries and first tile, the tile at the diagonal, and the results.
// ---------------------------------------------------------------------------------------
template <typename E, int D, bool PAGED>
__device__ __forceinline__ void attend_columns(const AttnArgs &a, const AttnUnit &u, int kv_head, lds_t lds, int32_t *votes)
{
    using X = AttnTile<E, D>;
    const int wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63;
    constexpr int COPIES = X::TILE / 1024 / 4, ROWS = COPIES * X::ROWS_PER_COPY;     // of a wavefront
    AttnSource<E, D, PAGED> src;
    src.init(a, u, kv_head);
    const int32_t n = key_tiles(u.key0, u.key1), base = u.key0 / ATTN_KEYS * ATTN_KEYS;
    const uint32_t lds0 = lds_address(lds);
    // Tiles that every column sees whole come first, then those at the end, and a first tile that begins before key0 last.
    const int32_t skip = u.key0 > base ? 1 : 0;
    auto key_of = [&](int32_t i) { return base + (i + skip < n ? i + skip : i + skip - n) * ATTN_KEYS; };
    auto fetch = [&](int32_t i) {
        const uint32_t to = lds0 + (i & 1) * X::TILE + wave * COPIES * 1024;
        const int32_t key = key_of(i) + wave * ROWS;
        src.template copy<false, COPIES>(to, key, wave * ROWS);
        src.template copy<true, COPIES>(to + 2 * X::TILE, key, wave * ROWS);
    };
    AttnColumns<E, D> w;
    w.init(a, u, kv_head, wave * 32);
    if (n > 0) fetch(0);
    w.arrived();
    const int32_t low = min(u.lim0, u.key1), high = u.key1;       // keys that every column sees, and that some column sees
    const float c = a.scale_log2;
    auto arrive = [&](int32_t i) {
        // this wavefront's copies of turn i and its reads of turn i - 1 are done, then everybody's
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (i + 1 < n) fetch(i + 1);
    };
    int32_t i = 0;
    const int32_t full = min(n, max(0, (low - base) / ATTN_KEYS - skip));         // tiles that every column sees whole
    for (; i < full; ++i) {
        arrive(i);
        const lds_t kt = lds + (i & 1) * X::TILE, vt = kt + 2 * X::TILE;
        f32x16_t s[2];
        s[0] = w.scores(kt, 0);
        s[1] = w.scores(kt, 32);
        w.template exponentials<2>(s, c);
        w.add(vt, 0, s[0]);
        w.add(vt, 32, s[1]);
    }
    bool bad = false;
    for (; i < n; ++i) {
        arrive(i);
        const lds_t kt = lds + (i & 1) * X::TILE, vt = kt + 2 * X::TILE;
        const int32_t key = key_of(i);
        const bool mine = __any(clean_rows<E, D, X::TILE / 16 / 256>(vt, key, u.key0, low, high, threadIdx.x, 256));
        if (lane == 0) votes[wave] = mine;
        f32x16_t s[2];
        s[0] = w.scores(kt, 0);
        s[1] = w.scores(kt, 32);
        __syncthreads();
        bad = votes[0] | votes[1] | votes[2] | votes[3];
        if (bad) break;
        w.hide(s[0], key, u.key0);
        w.hide(s[1], key + 32, u.key0);
        w.template exponentials<2>(s, c);
        w.add(vt, 0, s[0]);
        w.add(vt, 32, s[1]);
    }
    for (; i < n; ++i) {                                          // from a tile with infinities or NaN on: a loop of its own, for its registers
        if (!bad) {
            arrive(i);
            clean_rows<E, D, X::TILE / 16 / 256>(lds + (i & 1) * X::TILE + 2 * X::TILE, key_of(i), u.key0, low, high, threadIdx.x, 256);
            __syncthreads();
        }
        bad = false;
        const lds_t kt = lds + (i & 1) * X::TILE, vt = kt + 2 * X::TILE;
        const int32_t key = key_of(i);
        f32x16_t s[2];
        s[0] = w.scores(kt, 0);
        s[1] = w.scores(kt, 32);
        w.hide(s[0], key, u.key0);
        w.hide(s[1], key + 32, u.key0);
        w.template exponentials<2>(s, c);
        __syncthreads();                                          // the K tile becomes scratch
        const lds_t scratch = kt + wave * (X::TILE / 4);
        w.careful(vt, 0, s[0], scratch, key, u.key0);
        w.careful(vt, 32, s[1], scratch, key + 32, u.key0);
    }
    write_columns<E, D>(a, u, w, kv_head, wave * 32);
}

// ---------------------------------------------------------------------------------------
// A unit of up to 32 columns: bound by the bytes of its keys.  The four wavefronts take blocks of 32 keys in turn, each through LDS of its own without a
// barrier -- K of the next block is asked for as soon as this one's is in registers, V likewise -- and join their sums at the end.
// SOLO: the unit is one wavefront's.  Where short units are many this costs the look-ups before the first block once in 12 blocks instead of once in 3, and no join
// (256 rows of 64 heads over shared prefixes of 8192 and up to 700 tokens of their own: 173 us, else 180).
// 224 decode rows over 256..4096 tokens, 32 heads over 8 of 128: 348 us, 5.7 TB/s of keys and values, more than a copy moves on this card (4.9).
// ---------------------------------------------------------------------------------------
template <typename E, int D, bool PAGED, bool SOLO>
__device__ __forceinline__ void attend_keys(const AttnArgs &a, const AttnUnit &u, int kv_head, lds_t lds, float *join)
{
    using X = AttnTile<E, D>;
    constexpr int HALF = X::TILE / 2, COPIES = HALF / 1024;
    constexpr int PITCH = D + 4;                                  // floats between columns when they are joined: spreads the banks
    const int wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63, half = lane >> 5, tid = threadIdx.x;
    AttnSource<E, D, PAGED> src;
    src.init(a, u, kv_head);
    const lds_t kt = lds + wave * 2 * HALF, vt = kt + HALF;
    const uint32_t ka = lds_address(kt), va = ka + HALF;
    // Blocks first, first + STEP, ... of 32 keys; the first one last if it begins before key0.
    constexpr int STEP = SOLO ? 1 : 4;
    const int first = SOLO ? 0 : wave;
    const int32_t base = u.key0 / 32 * 32, blocks = u.key1 > u.key0 ? (u.key1 - 1 - base) / 32 + 1 : 0, n = (blocks - first + STEP - 1) / STEP;
    const int32_t skip = first == 0 && u.key0 > base ? 1 : 0;
    auto key_of = [&](int32_t i) { return base + (first + STEP * (i + skip < n ? i + skip : i + skip - n)) * 32; };
    AttnColumns<E, D> w;
    w.init(a, u, kv_head, 0);                                     // the queries are on their way while the first page is looked up
    if (n > 0) {
        src.template copy<false, COPIES>(ka, key_of(0), 0);
        src.template copy<true, COPIES>(va, key_of(0), 0);
    }
    const float c = a.scale_log2;
    w.arrived();
    const int32_t low = min(u.lim0, u.key1), before = (low - base) / 32 - first;           // blocks from this wavefront's first on that all columns see whole
    const int32_t full = min(n, max(0, (before + STEP - 1) / STEP - skip));
    int32_t i = 0;
    for (; i < full; ++i) {
        const bool more = i + 1 < n;
        wait_copies<COPIES>();                                    // K is there; V may be on its way
        f32x16_t s[1];
        s[0] = w.scores(kt, 0);
        wait_lds_reads();
        if (more) src.template copy<false, COPIES>(ka, key_of(i + 1), 0);
        w.template exponentials<1>(s, c);
        if (more) wait_copies<COPIES>();
        else wait_copies<0>();
        w.add(vt, 0, s[0]);
        wait_lds_reads();
        if (more) src.template copy<true, COPIES>(va, key_of(i + 1), 0);
    }
    bool bad = false;
    for (; i < n; ++i) {
        const int32_t key = key_of(i);
        wait_copies<0>();
        bad = __any(clean_rows<E, D, HALF / 1024>(vt, key, u.key0, low, u.key1, lane, 64));
        if (bad) break;
        f32x16_t s[1];
        s[0] = w.scores(kt, 0);
        w.hide(s[0], key, u.key0);
        w.template exponentials<1>(s, c);
        w.add(vt, 0, s[0]);
        wait_lds_reads();
        if (i + 1 < n) {
            src.template copy<false, COPIES>(ka, key_of(i + 1), 0);
            src.template copy<true, COPIES>(va, key_of(i + 1), 0);
        }
    }
    for (; i < n; ++i) {                                          // as above
        const int32_t key = key_of(i);
        wait_copies<0>();
        if (!bad) clean_rows<E, D, HALF / 1024>(vt, key, u.key0, low, u.key1, lane, 64);
        bad = false;
        f32x16_t s[1];
        s[0] = w.scores(kt, 0);
        w.hide(s[0], key, u.key0);
        w.template exponentials<1>(s, c);
        wait_lds_reads();
        w.careful(vt, 0, s[0], kt, key, u.key0);
        wait_lds_reads();
        if (i + 1 < n) {
            src.template copy<false, COPIES>(ka, key_of(i + 1), 0);
            src.template copy<true, COPIES>(va, key_of(i + 1), 0);
        }
    }
    if constexpr (SOLO) {
        write_columns<E, D>(a, u, w, kv_head, 0);
        return;
    }
    // join: every wavefront's sums at the largest m of all
    const float l = both_halves_sum(w.l);
    if (half == 0) { join[wave * 32 + lane] = w.m; join[128 + wave * 32 + lane] = l; }
    __syncthreads();                                              // and nobody reads K or V any more
    const int col = lane & 31;
    const float top = fmaxf(fmaxf(join[col], join[32 + col]), fmaxf(join[64 + col], join[96 + col]));
    const float f = __builtin_amdgcn_exp2f(w.m - top);
    PREFT_LDS float *o = (PREFT_LDS float *)lds;
    if (col < u.ncols) {
#pragma unroll
        for (int b = 0; b < X::BLOCKS; ++b)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const f32x4_t v = {w.o[b][4 * r] * f, w.o[b][4 * r + 1] * f, w.o[b][4 * r + 2] * f, w.o[b][4 * r + 3] * f};
                *(PREFT_LDS f32x4_t *)(o + (wave * 32 + col) * PITCH + b * 32 + 8 * r + 4 * half) = v;
            }
    }
    __syncthreads();
    for (int i = tid; i < u.ncols * (D / 4); i += 256) {
        const int cc = i / (D / 4), d = i % (D / 4) * 4;
        const float m0 = join[cc], m1 = join[32 + cc], m2 = join[64 + cc], m3 = join[96 + cc];
        const float mm = fmaxf(fmaxf(m0, m1), fmaxf(m2, m3));
        const float ll = join[128 + cc] * __builtin_amdgcn_exp2f(m0 - mm) + join[160 + cc] * __builtin_amdgcn_exp2f(m1 - mm) +
                         join[192 + cc] * __builtin_amdgcn_exp2f(m2 - mm) + join[224 + cc] * __builtin_amdgcn_exp2f(m3 - mm);
        f32x4_t v = *(PREFT_LDS f32x4_t *)(o + cc * PITCH + d);
#pragma unroll
        for (int k = 1; k < 4; ++k) {
            const f32x4_t x = *(PREFT_LDS f32x4_t *)(o + (k * 32 + cc) * PITCH + d);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += x[e];
        }
        if (u.slot < 0) {
            const int32_t x = u.head0 + cc, q = (int32_t)((uint32_t)x * a.per_head >> 21), head = kv_head * a.s.group + (x - q * a.s.group);
            const float inv = inverse(ll);
            const int32_t row = max(0, min(u.row0 + q, a.s.T - 1));   // a group's units always have parts
            store4<E>(as_global((char *)a.out + (int64_t)row * a.ldo + head * X::ROW + d * X::ELEM), v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
        } else {
            const int64_t part = (int64_t)u.slot + kv_head * u.ncols + cc;
            store4<float>(as_global((void *)(a.s.l.part_o + part * D + d)), v[0], v[1], v[2], v[3]);
            if (d == 0) a.s.l.part_ml[part] = make_float2(mm, ll);
        }
    }
}

// false: the call names another batch than the schedule's, and leaves a mark
__device__ __forceinline__ bool attn_schedule_is(const AttnArgs &a, int kind)
{
    const bool same = attn_schedule_fits(a.s);
    if (!same && threadIdx.x == 0 && blockIdx.x + blockIdx.y + blockIdx.z == 0) {
        a.s.l.report[HDR_ALL] = ATTN_REPORT;
        a.s.l.report[ATTN_MARKS + kind] = ATTN_MARK;
    }
    return same;
}

// Consecutive workgroups take the key/value heads of one unit: with 8 heads, or a multiple, every XCD keeps to its own heads' keys in its L2.
// DIRECT: there is no list, every wavefront finds the unit by itself (attn_direct_unit).
template <typename E, int D, bool PAGED, bool DIRECT>
__global__ __launch_bounds__(256, 2) void attention_kernel(AttnArgs a)
{
    using X = AttnTile<E, D>;
    constexpr int JOIN = 4 * 32 * (D + 4) * 4, KIND = PAGED ? 2 : 1;
    __shared__ __align__(1024) char lds[X::LDS > JOIN ? X::LDS : JOIN];
    __shared__ float join[256];
    const int32_t unit = (int32_t)blockIdx.x / a.s.kv_heads, kv_head = (int32_t)blockIdx.x % a.s.kv_heads;
    AttnUnit u;
    if constexpr (DIRECT) {
        if (a.ready && !attn_schedule_is(a, KIND)) return;
        if (!attn_direct_unit(a.s, unit, kv_head, a.ready != 0, u)) return;
    } else {
        if (!attn_schedule_is(a, KIND)) return;
        // short units: one a wavefront, four a workgroup
        const int32_t units = as_const(a.s.l.header)[AH_UNITS], alone = as_const(a.s.l.header)[AH_SHORT];
        const int32_t i = unit < alone ? unit : alone + 4 * (unit - alone) + uniform(threadIdx.x >> 6);
        if (i >= units) return;
        const PREFT_CONST AttnUnit *p = as_const(a.s.l.units) + i;
        u.table = p->table; u.head0 = p->head0; u.ncols = p->ncols; u.key0 = p->key0; u.key1 = p->key1; u.row0 = p->row0; u.lim0 = p->lim0; u.slot = p->slot;
        if (unit >= alone) {
            if (u.ncols > 0) attend_keys<E, D, PAGED, true>(a, u, kv_head, (lds_t)lds, join);
            return;
        }
    }
    if (u.ncols <= 0) return;
    if (u.ncols > ATTN_FEW_COLS) attend_columns<E, D, PAGED>(a, u, kv_head, (lds_t)lds, (int32_t *)join);
    else attend_keys<E, D, PAGED, false>(a, u, kv_head, (lds_t)lds, join);
}

// Joins the parts of a column: M = max m_j, out = sum 2^(m_j - M) o_j / sum 2^(m_j - M) l_j, in the order of the parts.  One wavefront a column.
template <typename E, int D>
__device__ __forceinline__ void join_tile(const AttnArgs &a, const AttnMerge &j, int kv_head)
{
    using X = AttnTile<E, D>;
    const int wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63, G = a.s.group;
    for (int32_t c = blockIdx.z * 4 + wave; c < j.ncols; c += 4 * gridDim.z) {
        const int32_t gc = j.group_col0 + c, tile = gc / ATTN_COLS;
        const int32_t width = min(ATTN_COLS, j.group_cols - tile * ATTN_COLS);
        const int64_t group = (int64_t)j.group_slot + (int64_t)tile * ATTN_COLS * a.s.kv_heads * j.group_parts + kv_head * width + gc % ATTN_COLS;
        const int64_t mine = (int64_t)j.slot + kv_head * j.ncols + c;
        const int32_t parts = j.parts + j.group_parts;           // at least one: see where the entries are made
        auto part = [&](int32_t k) {                               // slots are below 2^31: checked where the workspace is laid out
            const int64_t p = k < j.parts ? mine + (int64_t)k * j.ncols * a.s.kv_heads : group + (int64_t)(k - j.parts) * width * a.s.kv_heads;
            return p < 0 || p >= a.s.l.slot_cap ? 0 : (int32_t)p;
        };
        // A lane has the place and the factor of a part, 64 parts at a time; their rows are then read eight at a time, with nothing to wait for in between.
        int32_t at = part(min(lane, parts - 1));
        float2 ml = a.s.l.part_ml[at];
        float top = ml.x;
        for (int32_t k = lane + 64; k < parts; k += 64) top = fmaxf(top, a.s.l.part_ml[part(k)].x);
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
        float o[D / 64] = {}, l = 0.0f;
        for (int32_t k0 = 0; k0 < parts; k0 += 64) {
            const int32_t n = min(64, parts - k0);
            if (k0 > 0) {
                at = part(min(k0 + lane, parts - 1));
                ml = a.s.l.part_ml[at];
            }
            const float f = __builtin_amdgcn_exp2f(ml.x - top);
            float sum = lane < n ? ml.y * f : 0.0f;
            for (int32_t k = 0; k < n; k += 8) {
                float x[8][D / 64] = {};
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if (k + e >= n) continue;
                    const float *from = a.s.l.part_o + (int64_t)__builtin_amdgcn_readlane(at, k + e) * D + lane;
#pragma unroll
                    for (int d = 0; d < D / 64; ++d) x[e][d] = from[d * 64];
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float w = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), min(k + e, n - 1)));
#pragma unroll
                    for (int d = 0; d < D / 64; ++d) o[d] += x[e][d] * w;
                }
            }
#pragma unroll
            for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
            l += sum;
        }
        const float inv = inverse(l);
        const int32_t q = (j.col0 + c) / G, head = kv_head * G + (j.col0 + c - q * G), row = max(0, min(j.row0 + q, a.s.T - 1));
        E *to = (E *)((char *)a.out + (int64_t)row * a.ldo + head * X::ROW);
#pragma unroll
        for (int d = 0; d < D / 64; ++d) to[d * 64 + lane] = (E)(o[d] * inv);
    }
}

template <typename E, int D>
__global__ __launch_bounds__(256) void attention_merge_kernel(AttnArgs a, int kind)
{
    if (!attn_schedule_is(a, kind)) return;
    const int32_t n = as_const(a.s.l.header)[AH_JOINS];
    for (int32_t i = blockIdx.x; i < n; i += gridDim.x) {
        const AttnMerge j = a.s.l.merges[i];
        if (j.parts + j.group_parts > 0) join_tile<E, D>(a, j, (int)blockIdx.y);
    }
}

}  // namespace preft
