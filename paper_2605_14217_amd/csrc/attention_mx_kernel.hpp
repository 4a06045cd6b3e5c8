// Attention of query columns over keys in pages of 4-bit numbers: attention_kernel.hpp's products, sums and joins, with keys and values that become bf16 numbers
// on the way to the matrix cores.
//
// Every value of such a page is a bf16 number (three bits and a power of two), so nothing is lost there, and the products are those of bf16 pages.  Queries and
// weights in fp32 go to the matrix cores as three bf16 numbers of 8 bits each, cut and not rounded, whose sum they are: products are exact, sums are in fp32, and three
// products of bf16 take a fifth of the time of one in fp32.
//
// K: a lane has half the numbers of one key, two (one) times 16 bytes as they lie in the page, and uses them eight at a time as the left operand of S^T = K Q^T; the
// contraction runs over the head's elements in that order, and the queries are loaded in it.  V goes through LDS as bf16, for O^T = V^T P^T is to have it turned.
//
// Keys that a column may not see: their S is set to -inf whatever it was.  Their V meets P = 0: in the tiles where some column does not see some key, rows of V that
// no column sees, and what is NaN in the others, are zeroed; a column that sees a NaN gets it afterwards (32 elements of a head are NaN together: a mask of keys for each 32).
#pragma once
#include "attention_kernel.hpp"
#include "mx4.hpp"

namespace preft {

template <int D> struct MxTile {
    static constexpr int ROW = 2 * D, PIECES = ROW / 16;           // of a key in LDS, in bf16
    static constexpr int STEPS = PIECES / 2, BLOCKS = D / 32;
    static constexpr int MINE = D / 64;                            // 16-byte pieces of a key, of 32 numbers each, that a lane of 32 keys has
    static constexpr int TILE = ATTN_KEYS * ROW;
    // As in AttnTile; in V also by the row's bits above, so that a lane writes whole pieces of its row without a conflict.
    static __device__ __forceinline__ int k_turn(int row) { return PIECES < 16 ? (row >> 1) & 7 : row & 15; }
    static __device__ __forceinline__ int v_turn(int row) { return (PIECES >= 16 ? 4 * (row & 3) : 4 * ((row >> 1) & 1)) + ((row >> 2) & 3); }
};

// a number as three of 8 bits, its own upper bits first; infinite: the first alone; NaN stays NaN
struct Thirds { float part[3]; };
__device__ __forceinline__ Thirds thirds(float v)
{
    Thirds r;
    r.part[0] = __uint_as_float(__float_as_uint(v) & 0xffff0000u);
    const float rest = v - r.part[0];
    r.part[1] = __uint_as_float(__float_as_uint(rest) & 0xffff0000u);
    r.part[2] = rest - r.part[1];
    return r;
}
// the upper halves of two numbers
__device__ __forceinline__ uint32_t upper_halves(float lo, float hi) { return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u); }

template <typename E, int D> struct MxColumns : AttnColumns<E, D> {
    using X = MxTile<D>;
    using Base = AttnColumns<E, D>;
    using Base::o;
    static constexpr int PARTS = sizeof(E) == 2 ? 1 : 3;
    u32x4_t qp[PARTS][X::STEPS];       // elements D / 2 * half + 8 t .. of the query

    __device__ __forceinline__ void init(const AttnArgs &a, const AttnUnit &u, int kv_head, int first)
    {
        Base::place(a, u, kv_head, first);
        const int half = (threadIdx.x & 63) >> 5;
        const gcptr_t from = as_global((const char *)a.q + (int64_t)this->row * a.ldq + (int64_t)this->head * D * sizeof(E) + half * (D / 2) * (int)sizeof(E));
        if constexpr (PARTS == 1) {
#pragma unroll
            for (int t = 0; t < X::STEPS; ++t) qp[0][t] = ld16(from + t * 16);
        } else {
#pragma unroll
            for (int t = 0; t < X::STEPS; ++t) {
                const u32x4_t lo = ld16(from + t * 32), hi = ld16(from + t * 32 + 16);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const u32x4_t &two = i < 2 ? lo : hi;
                    Thirds x = thirds(__uint_as_float(two[2 * i & 3])), y = thirds(__uint_as_float(two[(2 * i & 3) + 1]));
                    if (!__builtin_isfinite(x.part[0])) x = whole(__uint_as_float(two[2 * i & 3]));
                    if (!__builtin_isfinite(y.part[0])) y = whole(__uint_as_float(two[(2 * i & 3) + 1]));
#pragma unroll
                    for (int p = 0; p < 3; ++p) qp[p][t][i] = upper_halves(x.part[p], y.part[p]);
                }
            }
        }
    }
    static __device__ __forceinline__ Thirds whole(float v) { return Thirds{{__uint_as_float(v != v ? 0x7fc00000u : __float_as_uint(v)), 0.0f, 0.0f}}; }

    __device__ __forceinline__ void arrived()
    {
#pragma unroll
        for (int p = 0; p < PARTS; ++p)
#pragma unroll
            for (int t = 0; t < X::STEPS; ++t) asm volatile("" : "+v"(qp[p][t]));
    }

    __device__ __forceinline__ void score(f32x16_t &s, u32x4_t k, int t) const
    {
#pragma unroll
        for (int p = PARTS - 1; p >= 0; --p)
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, k), __builtin_bit_cast(bf16x8_t, qp[p][t]), s, 0, 0, 0);
    }

    // S^T of 32 keys, a lane's half of its key in registers
    __device__ __forceinline__ f32x16_t scores(const u32x4_t (&k)[X::MINE], uint32_t powers) const
    {
        f32x16_t s;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.0f;
#pragma unroll
        for (int j = 0; j < X::MINE; ++j) {
            const float scale = mx4_scale((powers >> (8 * j)) & 255u);
#pragma unroll
            for (int e = 0; e < 4; ++e) score(s, mx4_bf16(k[j][e], scale), 4 * j + e);
        }
        return s;
    }

    // S^T of 32 keys from row `row0` of a K tile on
    __device__ __forceinline__ f32x16_t scores(lds_t tile, int row0) const
    {
        const int lane = threadIdx.x & 63, half = lane >> 5, r = lane & 31;
        const lds_t at = tile + (row0 + r) * X::ROW;
        const int turn = X::k_turn(r);
        f32x16_t s;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.0f;
#pragma unroll
        for (int t = 0; t < X::STEPS; ++t) score(s, *(const PREFT_LDS u32x4_t *)(at + (((X::STEPS * half + t) ^ turn) << 4)), t);
        return s;
    }

    // O^T += V^T P^T over 32 keys from row `row0` of a V tile on
    __device__ __forceinline__ void add(lds_t tile, int row0, const f32x16_t &p)
    {
        const int lane = threadIdx.x & 63, half = lane >> 5;
        const int i = lane & 15, key = 4 * half + (i >> 2), turn = X::v_turn(key);          // 8 keys further on: the turn's bit 1 changes
        const lds_t at = tile + (row0 + key) * X::ROW + (i & 1) * 8;
        const int piece = ((lane >> 4) & 1) * 2 + ((i & 3) >> 1);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            union { uint32_t w[4]; bf16x8_t v; } pb[PARTS];
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float x = p[8 * h + 2 * w], y = p[8 * h + 2 * w + 1];
                if constexpr (PARTS == 1) {
                    pb[0].w[w] = pack_bf16(x, y);
                } else {
                    const Thirds xs = thirds(x), ys = thirds(y);
#pragma unroll
                    for (int k = 0; k < 3; ++k) pb[k].w[w] = upper_halves(xs.part[k], ys.part[k]);
                }
            }
#pragma unroll
            for (int b = 0; b < X::BLOCKS; ++b) {
                const lds_t from = at + 16 * h * X::ROW;
                const bf16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((PREFT_LDS bf16x4_t *)(from + (((b * 4 + piece) ^ turn) << 4)));
                const bf16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((PREFT_LDS bf16x4_t *)(from + 8 * X::ROW + (((b * 4 + piece) ^ turn ^ 2) << 4)));
                const bf16x8_t v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
                for (int k = PARTS - 1; k >= 0; --k) o[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, pb[k].v, o[b], 0, 0, 0);
            }
        }
    }

    // Of 32 keys from `key` on, those of `bad` are NaN in 32 elements of V: so is a column that sees one, in these.
    __device__ __forceinline__ void spoil(int b, uint32_t bad, int32_t key, int32_t key0)
    {
        const int32_t from = max(key0 - key, 0), to = max(0, min(this->lim - key, 32));
        const uint32_t seen = (to >= 32 ? ~0u : (1u << to) - 1) & (from >= 32 ? 0u : ~0u << from);
        if (bad & seen) {
#pragma unroll
            for (int i = 0; i < 16; ++i) o[b][i] = __uint_as_float(0x7fc00000u);
        }
    }
};

// Where a unit's keys lie.
template <int D> struct MxSource {
    using P = Mx4Page<D>;
    const char *k, *v;                 // of this key/value head
    const int32_t *table;
    int32_t last;                      // the last key there is
    int32_t n_pages, page_shift;
    int64_t page_bytes;

    __device__ __forceinline__ void init(const AttnArgs &a, const AttnUnit &u, int head)
    {
        last = max(u.key1 - 1, 0);
        page_shift = a.page_shift;
        n_pages = a.n_pages;
        page_bytes = P::head_bytes(page_shift) * a.s.kv_heads;
        k = (const char *)a.k + P::head_bytes(page_shift) * head;
        v = (const char *)a.v + P::head_bytes(page_shift) * head;
        table = a.table + (int64_t)u.table * a.ld_table;
    }
    // the page of a lane's key, as the block table names it; outside the pool: its first or last page
    __device__ __forceinline__ uint32_t page_of(int32_t key) const { return (uint32_t)table[min(key, last) >> page_shift]; }
    // where a lane's key begins in its page, and that page (keys past the last: the last)
    __device__ __forceinline__ int64_t page_at(uint32_t page) const { return (int64_t)min(page, (uint32_t)(n_pages - 1)) * page_bytes; }
    __device__ __forceinline__ int32_t in_page(int32_t key) const { return min(key, last) & ((1 << page_shift) - 1); }
};

// What is NaN, or lies in a row that no column sees, becomes zeros; says whether it is NaN in a row that some column sees.
__device__ __forceinline__ bool mx4_clean(u32x4_t &numbers, uint32_t &power, bool seen)
{
    const bool nan = power > 252u;
    if (nan || !seen) { numbers = u32x4_t{0, 0, 0, 0}; power = 127u; }
    return nan && seen;
}

// 32 numbers to four pieces of a row in LDS
__device__ __forceinline__ void mx4_put(lds_t row, int piece, int turn, u32x4_t numbers, uint32_t power)
{
    const float scale = mx4_scale(power);
#pragma unroll
    for (int e = 0; e < 4; ++e) *(PREFT_LDS u32x4_t *)(row + (((piece + e) ^ turn) << 4)) = mx4_bf16(numbers[e], scale);
}

// ---------------------------------------------------------------------------------------
// A unit of more than 32 columns: as in attend_columns, but the tiles of 64 keys come through registers: each thread has 32 numbers of K and 32 of V (heads of 64: of one)
// of the tile after next on their way while this one's products run.
// ---------------------------------------------------------------------------------------
template <typename E, int D>
__device__ __forceinline__ void mx_attend_columns(const AttnArgs &a, const AttnUnit &u, int kv_head, lds_t lds, uint32_t *bad)
{
    using X = MxTile<D>;
    using P = Mx4Page<D>;
    const int wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63;
    MxSource<D> src;
    src.init(a, u, kv_head);
    const int32_t n = key_tiles(u.key0, u.key1), base = u.key0 / ATTN_KEYS * ATTN_KEYS;
    const int32_t skip = u.key0 > base ? 1 : 0;                  // a first tile that begins before key0 comes last
    auto key_of = [&](int32_t i) { return base + (i + skip < n ? i + skip : i + skip - n) * ATTN_KEYS; };
    // this thread's row of the tile, and 32 elements of it; heads of 64: two wavefronts have K and two V
    const int r = (lane & 31) + 32 * (wave & 1), block = D == 128 ? (lane >> 5) + 2 * (wave >> 1) : lane >> 5;
    const bool has_k = D == 128 || wave < 2, has_v = D == 128 || wave >= 2;
    u32x4_t kn = {}, vn = {};
    uint32_t kp = 127, vp = 127, page = 0;
    auto look = [&](int32_t i) { page = src.page_of(key_of(i) + r); };
    auto fetch = [&](int32_t i) {
        const int64_t at = src.page_at(page);
        const int32_t in = src.in_page(key_of(i) + r);
        const int64_t numbers = at + in * P::NUMBERS + block * 16, power = at + ((int64_t)P::NUMBERS << src.page_shift) + in * P::POWERS + block;
        if (has_k) { kn = ld16(as_global((const void *)src.k) + numbers); kp = *(as_global((const void *)src.k) + power) & 255u; }
        if (has_v) { vn = ld16(as_global((const void *)src.v) + numbers); vp = *(as_global((const void *)src.v) + power) & 255u; }
    };
    MxColumns<E, D> w;
    if (n > 0) look(0);
    w.init(a, u, kv_head, wave * 32);
    if (n > 0) fetch(0);
    if (n > 1) look(1);
    w.arrived();
    const int32_t low = min(u.lim0, u.key1);                     // keys that every column sees
    const float c = a.scale_log2;
    const int32_t full = min(n, max(0, (low - base) / ATTN_KEYS - skip));         // tiles that every column sees whole
    // tile i, which is in registers, to LDS; `bad`: for each 32 keys and 32 elements of the tile the keys that are NaN there
    auto put = [&](int32_t i) {
        const lds_t kt = lds + (i & 1) * X::TILE, vt = kt + 2 * X::TILE;
        if (has_k) mx4_put(kt + r * X::ROW, 4 * block, X::k_turn(r), kn, kp);
        if (has_v) {
            if (i >= full) {
                const int32_t key = key_of(i) + r;
                const uint64_t nan = __ballot(mx4_clean(vn, vp, key >= u.key0 && key < u.key1));
                if (lane % 32 == 0) bad[(i & 1) * 8 + (wave & 1) * 4 + block] = (uint32_t)(nan >> lane);
            }
            mx4_put(vt + r * X::ROW, 4 * block, X::v_turn(r), vn, vp);
        }
        if (i + 1 < n) fetch(i + 1);
        if (i + 2 < n) look(i + 2);
    };
    if (n > 0) put(0);
    auto arrive = [&](int32_t i) {
        // this wavefront's share of tile i is in LDS and its reads of tile i - 1 are done, then everybody's
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (i + 1 < n) put(i + 1);
    };
    int32_t i = 0;
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
    for (; i < n; ++i) {
        arrive(i);
        const lds_t kt = lds + (i & 1) * X::TILE, vt = kt + 2 * X::TILE;
        const int32_t key = key_of(i);
        f32x16_t s[2];
        s[0] = w.scores(kt, 0);
        s[1] = w.scores(kt, 32);
        w.hide(s[0], key, u.key0);
        w.hide(s[1], key + 32, u.key0);
        w.template exponentials<2>(s, c);
        w.add(vt, 0, s[0]);
        w.add(vt, 32, s[1]);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int b = 0; b < X::BLOCKS; ++b) w.spoil(b, bad[(i & 1) * 8 + h * 4 + b], key + 32 * h, u.key0);
    }
    write_columns<E, D>(a, u, w, kv_head, wave * 32);
}

// ---------------------------------------------------------------------------------------
// A unit of up to 32 columns: bound by the bytes of its keys.  The four wavefronts take blocks of 32 keys in turn, the next one's on their way in registers, and join their sums at
// the end.  SOLO: the unit is one wavefront's.
// ---------------------------------------------------------------------------------------
template <typename E, int D, bool SOLO>
__device__ __forceinline__ void mx_attend_keys(const AttnArgs &a, const AttnUnit &u, int kv_head, lds_t lds, float *join)
{
    using X = MxTile<D>;
    using P = Mx4Page<D>;
    const int wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63, r = lane & 31, half = lane >> 5;
    MxSource<D> src;
    src.init(a, u, kv_head);
    const lds_t vt = lds + wave * (X::TILE / 2);
    // Blocks first, first + STEP, ... of 32 keys; the first one last if it begins before key0.
    constexpr int STEP = SOLO ? 1 : 4;
    const int first = SOLO ? 0 : wave;
    const int32_t base = u.key0 / 32 * 32, blocks = u.key1 > u.key0 ? (u.key1 - 1 - base) / 32 + 1 : 0, n = (blocks - first + STEP - 1) / STEP;
    const int32_t skip = first == 0 && u.key0 > base ? 1 : 0;
    auto key_of = [&](int32_t i) { return base + (first + STEP * (i + skip < n ? i + skip : i + skip - n)) * 32; };
    u32x4_t kn[X::MINE], vn[X::MINE];
    uint32_t kp = 0, vp = 0, page = 0;
    auto look = [&](int32_t i) { page = src.page_of(key_of(i) + r); };
    auto fetch = [&](int32_t i) {
        const int64_t at = src.page_at(page);
        const int32_t in = src.in_page(key_of(i) + r);
        const int64_t numbers = at + in * P::NUMBERS + half * (16 * X::MINE), powers = at + ((int64_t)P::NUMBERS << src.page_shift) + in * P::POWERS + half * X::MINE;
        const gcptr_t k = as_global((const void *)src.k), v = as_global((const void *)src.v);
#pragma unroll
        for (int j = 0; j < X::MINE; ++j) { kn[j] = ld16(k + numbers + j * 16); vn[j] = ld16(v + numbers + j * 16); }
        if constexpr (X::MINE == 2) {
            kp = *(const PREFT_GLOBAL uint16_t *)(k + powers);
            vp = *(const PREFT_GLOBAL uint16_t *)(v + powers);
        } else {
            kp = *(const PREFT_GLOBAL uint8_t *)(k + powers);
            vp = *(const PREFT_GLOBAL uint8_t *)(v + powers);
        }
    };
    MxColumns<E, D> w;
    if (n > 0) look(0);
    w.init(a, u, kv_head, 0);                                     // the queries are on their way while the first page is looked up
    if (n > 0) fetch(0);
    if (n > 1) look(1);
    const float c = a.scale_log2;
    w.arrived();
    const int32_t low = min(u.lim0, u.key1), before = (low - base) / 32 - first;           // blocks from this wavefront's first on that all columns see whole
    const int32_t full = min(n, max(0, (before + STEP - 1) / STEP - skip));
    for (int32_t i = 0; i < n; ++i) {
        const int32_t key = key_of(i);
        u32x4_t k[X::MINE], v[X::MINE];
        uint32_t powers = kp, vpowers[X::MINE];
#pragma unroll
        for (int j = 0; j < X::MINE; ++j) { k[j] = kn[j]; v[j] = vn[j]; vpowers[j] = (vp >> (8 * j)) & 255u; }
        if (i + 1 < n) fetch(i + 1);
        if (i + 2 < n) look(i + 2);
        uint64_t bad[X::MINE] = {};
        if (i >= full) {
            const int32_t mine = key + r;
#pragma unroll
            for (int j = 0; j < X::MINE; ++j) bad[j] = __ballot(mx4_clean(v[j], vpowers[j], mine >= u.key0 && mine < u.key1));
        }
        f32x16_t s[1];
        s[0] = w.scores(k, powers);
        wait_lds_reads();                                         // of the block before
#pragma unroll
        for (int j = 0; j < X::MINE; ++j) mx4_put(vt + r * X::ROW, 4 * (X::MINE * half + j), X::v_turn(r), v[j], vpowers[j]);
        if (i >= full) w.hide(s[0], key, u.key0);
        w.template exponentials<1>(s, c);
        wait_lds_reads();                                         // written: nobody else's, so without a barrier
        w.add(vt, 0, s[0]);
        if (i >= full) {
#pragma unroll
            for (int j = 0; j < X::MINE; ++j) {
                w.spoil(j, (uint32_t)bad[j], key, u.key0);
                w.spoil(X::MINE + j, (uint32_t)(bad[j] >> 32), key, u.key0);
            }
        }
    }
    if constexpr (SOLO) write_columns<E, D>(a, u, w, kv_head, 0);
    else join_waves<E, D>(a, u, w, kv_head, lds, join);
}

template <typename E, int D, bool DIRECT>
__global__ __launch_bounds__(256, 2) void attention_mx_kernel(AttnArgs a)
{
    using X = MxTile<D>;
    constexpr int JOIN = 4 * 32 * (D + 4) * 4, KIND = 2;
    __shared__ __align__(1024) char lds[4 * X::TILE > JOIN ? 4 * X::TILE : JOIN];
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
            if (u.ncols > 0) mx_attend_keys<E, D, true>(a, u, kv_head, (lds_t)lds, join);
            return;
        }
    }
    if (u.ncols <= 0) return;
    if (u.ncols > ATTN_FEW_COLS) mx_attend_columns<E, D>(a, u, kv_head, (lds_t)lds, (uint32_t *)join);
    else mx_attend_keys<E, D, false>(a, u, kv_head, (lds_t)lds, join);
}

}  // namespace preft
