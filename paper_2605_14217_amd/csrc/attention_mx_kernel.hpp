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
    // Rows in LDS are further apart than they are long, so that what is read in one cycle comes from all banks: of K, 16 lanes' 16 bytes of as many rows; of V, 64 bytes each
    // of 4 rows.  (Turning the pieces of a row does it too, but takes a register for every address: with 16-byte pieces at constant distances one is enough.  So nothing spills, but in the kernels of f32
    // heads of 128, whose three parts of a query are 96 registers: 15 spilled, 44 bytes a lane.)
    static constexpr int K_PITCH = ROW + 16;
    static __device__ __forceinline__ constexpr int v_row(int row) { return row * (ROW + 64) + (row >> 2) * 16; }       // (and what is written, 16 bytes of 16 rows)
    static constexpr int K_TILE = ATTN_KEYS * K_PITCH, V_TILE = ATTN_KEYS * (ROW + 68), LDS = 2 * (K_TILE + V_TILE);
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

// eight elements of a query, as they go to the matrix cores
template <typename E, int PARTS, int STEPS> __device__ __forceinline__ void mx_query(gcptr_t from, u32x4_t (&q)[PARTS][STEPS], int t)
{
    if constexpr (sizeof(E) == 2) {
        q[0][t] = ld16(from);
    } else {
        const u32x4_t lo = ld16(from), hi = ld16(from + 16);
        auto cut = [](uint32_t bits) {
            const float v = __uint_as_float(bits);
            if (__builtin_isfinite(v)) return thirds(v);
            return Thirds{{__uint_as_float(v != v ? 0x7fc00000u : bits), 0.0f, 0.0f}};
        };
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const u32x4_t &two = i < 2 ? lo : hi;
            const Thirds x = cut(two[2 * i & 3]), y = cut(two[(2 * i & 3) + 1]);
#pragma unroll
            for (int p = 0; p < 3; ++p) q[p][t][i] = upper_halves(x.part[p], y.part[p]);
        }
    }
}
// Two weights likewise: put(part, both).  Those of bf16 rows are rounded to bf16, each off by up to 2^-8 of itself, as over bf16 pages: a row's result is as near whatever its pages hold and however wide
// its unit is.  With a remainder beside them outputs would be off by 0.17 % of their norm, their own rounding, instead of 0.23 %; wide units, which the matrix cores bound, have no time for half as many products again.
template <int PARTS, typename Put> __device__ __forceinline__ void mx_weights(float x, float y, Put put)
{
    if constexpr (PARTS == 1) {
        put(0, pack_bf16(x, y));
    } else {
        const Thirds xs = thirds(x), ys = thirds(y);
#pragma unroll
        for (int k = 0; k < 3; ++k) put(k, upper_halves(xs.part[k], ys.part[k]));
    }
}
// the power that begins at bit `bits` of four
__device__ __forceinline__ uint32_t mx4_power_of(uint32_t four, int bits) { return (four >> bits) & 255u; }
// of 32 keys from `key` on, those that a column sees
__device__ __forceinline__ uint32_t seen_keys(int32_t lim, int32_t key, int32_t key0)
{
    const int32_t from = max(key0 - key, 0), to = max(0, min(lim - key, 32));
    return (to >= 32 ? ~0u : (1u << to) - 1) & (from >= 32 ? 0u : ~0u << from);
}

constexpr int MX_FEW_COLS = 16;        // up to here a unit's columns are one tile of 16

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
#pragma unroll
        for (int t = 0; t < X::STEPS; ++t) mx_query<E>(from + t * 8 * (int)sizeof(E), qp, t);
    }

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
    struct Scores { f32x16_t s[1]; };
    __device__ __forceinline__ void scores(Scores &r, const uint32_t (&k)[4 * X::MINE], const uint32_t (&powers)[2], int bits) const
    {
#pragma unroll
        for (int i = 0; i < 16; ++i) r.s[0][i] = 0.0f;
#pragma unroll
        for (int j = 0; j < X::MINE; ++j) {
            const float scale = mx4_scale(mx4_power_of(powers[0], bits + 8 * j));
#pragma unroll
            for (int e = 0; e < 4; ++e) score(r.s[0], mx4_bf16(k[4 * j + e], scale), 4 * j + e);
        }
    }
    __device__ __forceinline__ void hide_all(Scores &r, int32_t key, int32_t key0) const { this->hide(r.s[0], key, key0); }
    using Base::exponentials;
    __device__ __forceinline__ void exponentials(Scores &r, float c) { Base::template exponentials<1>(r.s, c); }
    __device__ __forceinline__ void add_all(lds_t tile, const Scores &r) { add(tile, 0, r.s[0]); }
    __device__ __forceinline__ void write(const AttnArgs &a, const AttnUnit &u, int kv_head) { write_columns<E, D>(a, u, *this, kv_head, 0); }
    static constexpr int V_BLOCK = X::V_TILE / 2;
    static __device__ __forceinline__ int v_row(int row) { return X::v_row(row); }

    // S^T of 32 keys from row `row0` of a K tile on
    __device__ __forceinline__ f32x16_t scores(lds_t tile, int row0) const
    {
        const int lane = threadIdx.x & 63, half = lane >> 5, r = lane & 31;
        const lds_t at = tile + r * X::K_PITCH + half * (X::ROW / 2);
        f32x16_t s;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.0f;
#pragma unroll
        for (int t = 0; t < X::STEPS; ++t) score(s, *(const PREFT_LDS u32x4_t *)(at + row0 * X::K_PITCH + 16 * t), t);
        return s;
    }

    // S^T -> P^T by the m there is, without the largest S, a tenth of a tile's vector instructions: true where a weight may pass 2^8, S^T is then to be taken anew, and `exponentials` to look at the largest S.  It
    // raises m where that is more than 2^8 above; where many are 2^4 to 2^8 above and none is further, m stays, and the next tile is taken twice again.  (Sums that are NaN stay: so is the result.)
    __device__ __forceinline__ bool try_exponentials(f32x16_t (&s)[2], float c)
    {
        float sum = 0.0f;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[b][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][i], c, -this->m));
                sum += s[b][i];
            }
        if (__any(sum > 256.0f)) return true;
        this->l += sum;
        return false;
    }

    // O^T += V^T P^T over 32 keys from row `row0` of a V tile on
    __device__ __forceinline__ void add(lds_t tile, int row0, const f32x16_t &p)
    {
        const int lane = threadIdx.x & 63, half = lane >> 5;
        const int i = lane & 15;
        const lds_t at = tile + X::v_row(4 * half + (i >> 2)) + ((lane >> 4) & 1) * 32 + (i & 3) * 8;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            union { uint32_t w[4]; bf16x8_t v; } pb[PARTS];
#pragma unroll
            for (int w = 0; w < 4; ++w) mx_weights<PARTS>(p[8 * h + 2 * w], p[8 * h + 2 * w + 1], [&](int k, uint32_t two) { pb[k].w[w] = two; });
#pragma unroll
            for (int b = 0; b < X::BLOCKS; ++b) {
                const lds_t from = at + X::v_row(row0 + 16 * h) + 64 * b;
                const bf16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((PREFT_LDS bf16x4_t *)from);
                const bf16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((PREFT_LDS bf16x4_t *)(from + X::v_row(8)));
                const bf16x8_t v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
                for (int k = PARTS - 1; k >= 0; --k) o[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, pb[k].v, o[b], 0, 0, 0);
            }
        }
    }

    // How the reads of LDS and the products of 64 keys stand: reads several products ahead (the compiler keeps two in flight).
    static __device__ __forceinline__ void order_scores()
    {
        __builtin_amdgcn_sched_group_barrier(0x100, X::STEPS, 0);
#pragma unroll
        for (int t = 0; t < X::STEPS; ++t) {
            __builtin_amdgcn_sched_group_barrier(0x008, PARTS, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, X::STEPS * PARTS, 0);
    }
    static __device__ __forceinline__ void order_sums()
    {
        constexpr int READS = 8 * X::BLOCKS, FIRST = 8;           // of 8 bytes
        __builtin_amdgcn_sched_group_barrier(0x100, FIRST, 1);
#pragma unroll
        for (int t = 0; t < (READS - FIRST) / 2; ++t) {
            __builtin_amdgcn_sched_group_barrier(0x008, PARTS, 1);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 1);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, FIRST / 2 * PARTS, 1);
    }

    // Of 32 keys from `key` on, those of `bad` are NaN in 32 elements of V: so is a column that sees one, in these.
    __device__ __forceinline__ void spoil(int b, uint32_t bad, int32_t key, int32_t key0)
    {
        if (bad & seen_keys(this->lim, key, key0)) {
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
    // Powers are loaded four at a time, a key's (heads of 64: those of two): bytes of the four from the first, of key `in` of a page; and the bits before its first.  (Loaded as bytes they are
    // 8-bit values to the compiler, which copies such registers at the end of a loop, and waits there for all that is on its way.)
    static __device__ __forceinline__ int32_t powers_at(int32_t in) { return D == 128 ? in * 4 : (in & ~1) * 2; }
    static __device__ __forceinline__ int32_t power_bits(int32_t in) { return D == 128 ? 0 : (in & 1) * 16; }
};

// Pages of 32 tokens and more: 32 keys that begin at a multiple of 32 are in one.  It is looked up when they are asked for, among 64 entries of the table that the lanes hold, and the
// loads are buffer loads: a page's address and the keys' place in it are scalar, the lanes' offsets constant, and what is asked for past the last block is a load of no bytes.  So no
// vector instruction makes an address, no branch need stand between the loads of a stream, and the compiler waits for those that it needs and not for all.
template <int D> struct MxOnePage {
    using P = Mx4Page<D>;
    int32_t ids, ids_first;            // 64 page numbers from table[ids_first] on, one a lane
    struct Keys { __amdgpu_buffer_rsrc_t k, v; int numbers, powers; };     // of a block: the page's K and V, and where its numbers and powers begin there

    __device__ __forceinline__ void init(const MxSource<D> &src, int32_t key) { reload(src, min(key, src.last) >> src.page_shift); }
    __device__ __forceinline__ void reload(const MxSource<D> &src, int32_t i)
    {
        ids_first = i;
        ids = src.table[min(i + (int32_t)(threadIdx.x & 63), src.last >> src.page_shift)];
        asm volatile("" : "+v"(ids));                             // waited for here, and not wherever it is read
    }
    __device__ __forceinline__ Keys at(const MxSource<D> &src, int32_t key, bool there)
    {
        const int32_t i = min(key, src.last) >> src.page_shift, in = key & ((1 << src.page_shift) - 1);
        if (there && (i - ids_first >= 64 || i < ids_first)) reload(src, i);
        const int64_t from = src.page_at((uint32_t)__builtin_amdgcn_readlane(ids, there ? i - ids_first : 0));
        const int bytes = there ? (int)P::head_bytes(src.page_shift) : 0;
        return Keys{__builtin_amdgcn_make_buffer_rsrc((void *)(src.k + from), 0, bytes, 0x00027000),
                    __builtin_amdgcn_make_buffer_rsrc((void *)(src.v + from), 0, bytes, 0x00027000), in * P::NUMBERS, (P::NUMBERS << src.page_shift) + in * P::POWERS};
    }
};

// Blocks of 32 keys on their way to a wavefront's registers.  What a lane has of K: FEW, quarter lane / 16 of keys lane % 16 and 16 + lane % 16; else half lane / 32 of key lane % 32, as
// always of V.
//
// ONE: MxOnePage.  Else each lane looks its keys' pages up, a block earlier, and past the last block asks for that again.
template <int D, bool FEW, bool ONE> struct MxStream {
    using P = Mx4Page<D>;
    static constexpr int MINE = D / 64, WORDS = D / 16;           // 16-byte pieces of V, and words of K
    struct Block { uint32_t k[WORDS], kp[2], vp, page[2]; u32x4_t v[MINE]; };
    MxSource<D> src;
    int32_t n, base, first, step, skip;
    MxOnePage<D> one;
    int32_t k_at, kp_at, v_at, vp_at;  // ONE: bytes of the lane's share in a block's numbers, and of the powers of its keys
    int32_t k_bits, v_bits;            // where the powers of its share are among four.  (Keys past the last are the last's in other places: nobody sees them.)

    __device__ __forceinline__ void init(const AttnArgs &a, const AttnUnit &u, int kv_head, int first_, int step_)
    {
        src.init(a, u, kv_head);
        first = first_;
        step = step_;
        // Blocks first, first + step, ... of 32 keys; the first one last if it begins before key0.
        base = u.key0 / 32 * 32;
        const int32_t blocks = u.key1 > u.key0 ? (u.key1 - 1 - base) / 32 + 1 : 0;
        n = (blocks - first + step - 1) / step;
        skip = first == 0 && u.key0 > base ? 1 : 0;
        const int lane = threadIdx.x & 63, g = lane >> 4, half = lane >> 5, r = lane & 31;
        v_at = r * P::NUMBERS + half * (16 * MINE);
        vp_at = src.powers_at(r);
        v_bits = src.power_bits(r) + 8 * half * MINE;
        k_at = FEW ? (lane & 15) * P::NUMBERS + g * (D / 8) : v_at;
        kp_at = FEW ? src.powers_at(lane & 15) : vp_at;
        k_bits = FEW ? src.power_bits(lane & 15) + 8 * (g * P::POWERS / 4) : v_bits;
        if (ONE && n > 0) one.init(src, key_of(0));                // no key: the table may have no entry
    }
    __device__ __forceinline__ int32_t key_of(int32_t i) const { return base + (first + step * (i + skip < n ? i + skip : i + skip - n)) * 32; }
    // blocks that come before any that some column does not see whole; low: keys that every column sees
    __device__ __forceinline__ int32_t whole(int32_t low) const { return min(n, max(0, ((low - base) / 32 - first + step - 1) / step - skip)); }

    __device__ __forceinline__ void look(Block &b, int32_t i) const
    {
        if constexpr (!ONE) {
            const int lane = threadIdx.x & 63;
            const int32_t key = key_of(min(i, n - 1));
            b.page[0] = src.page_of(key + (FEW ? lane & 15 : lane & 31));
            if constexpr (FEW) b.page[1] = src.page_of(key + 16 + (lane & 15));
        }
    }
    __device__ __forceinline__ void fetch(Block &b, int32_t i)
    {
        const int lane = threadIdx.x & 63;
        if constexpr (ONE) {
            const bool there = i < n;
            const auto [k, v, numbers, powers] = one.at(src, key_of(there ? i : 0), there);
            if constexpr (!FEW) {
#pragma unroll
                for (int j = 0; j < MINE; ++j) words(b, 4 * j, __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(k, k_at + 16 * j, numbers, 0)));
                b.kp[0] = __builtin_amdgcn_raw_buffer_load_b32(k, kp_at, powers, 0);
            } else {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if constexpr (D == 128) words(b, 4 * h, __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(k, k_at + 16 * h * P::NUMBERS, numbers, 0)));
                    else two_words(b, 2 * h, __builtin_bit_cast(u32x2_t, __builtin_amdgcn_raw_buffer_load_b64(k, k_at + 16 * h * P::NUMBERS, numbers, 0)));
                    b.kp[h] = __builtin_amdgcn_raw_buffer_load_b32(k, kp_at + 16 * h * P::POWERS, powers, 0);
                }
            }
#pragma unroll
            for (int j = 0; j < MINE; ++j) b.v[j] = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(v, v_at + 16 * j, numbers, 0));
            b.vp = __builtin_amdgcn_raw_buffer_load_b32(v, vp_at, powers, 0);
        } else {
            const int g = lane >> 4, half = lane >> 5;
            const int32_t key = key_of(min(i, n - 1));
            const gcptr_t k = as_global((const void *)src.k), v = as_global((const void *)src.v);
            const int64_t powers = (int64_t)P::NUMBERS << src.page_shift;
            int64_t from[2];
            int32_t in[2];
#pragma unroll
            for (int h = 0; h < (FEW ? 2 : 1); ++h) {
                from[h] = src.page_at(b.page[h]);
                in[h] = src.in_page(key + 16 * h + (FEW ? lane & 15 : lane & 31));
                const gcptr_t row = k + from[h] + in[h] * P::NUMBERS, power = k + from[h] + powers + src.powers_at(in[h]);
                if constexpr (FEW) {
                    if constexpr (D == 128) words(b, 4 * h, ld16(row + g * 16));
                    else two_words(b, 2 * h, ld8(row + g * 8));
                    b.kp[h] = ld4(power);
                } else {
#pragma unroll
                    for (int j = 0; j < MINE; ++j) words(b, 4 * j, ld16(row + half * (16 * MINE) + 16 * j));
                    b.kp[0] = ld4(power);
                }
            }
            const bool second = FEW && (lane & 16);
            const int64_t page = second ? from[1] : from[0];
            const int32_t at = second ? in[1] : in[0];
#pragma unroll
            for (int j = 0; j < MINE; ++j) b.v[j] = ld16(v + page + at * P::NUMBERS + half * (16 * MINE) + 16 * j);
            b.vp = ld4(v + page + powers + src.powers_at(at));
        }
    }
    static __device__ __forceinline__ void words(Block &b, int at, u32x4_t x)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) b.k[at + i] = x[i];
    }
    static __device__ __forceinline__ void two_words(Block &b, int at, u32x2_t x) { b.k[at] = x[0]; b.k[at + 1] = x[1]; }
};

// What is NaN, or lies in a row that no column sees, becomes zeros; says whether it is NaN in a row that some column sees.
__device__ __forceinline__ bool mx4_clean(u32x4_t &numbers, uint32_t &power, bool seen)
{
    const bool nan = power > 252u;
    if (nan || !seen) { numbers = u32x4_t{0, 0, 0, 0}; power = 127u; }
    return nan && seen;
}

// 32 numbers to their place in a row in LDS
__device__ __forceinline__ void mx4_put(lds_t to, u32x4_t numbers, uint32_t power)
{
    const float scale = mx4_scale(power);
#pragma unroll
    for (int e = 0; e < 4; ++e) *(PREFT_LDS u32x4_t *)(to + 16 * e) = mx4_bf16(numbers[e], scale);
}

// ---------------------------------------------------------------------------------------
// A unit of more than 32 columns: as in attend_columns, but the tiles of 64 keys come through registers: each thread has 32 numbers of K and 32 of V (heads of 64: of one)
// of the tile after next on their way while this one's products run.  Four requests' further chunks, 6000 rows over 5000..17 000 tokens, 32 heads over 8 of 128: 867-895 us with schedule and join, by the card, 1110-1150 TFLOP/s,
// 92-95 % of a large matrix product's 1200 (keys that all score 2^4 to 2^8 above those of the first tile, so that each tile is taken twice: 1175, all alike 755); before the wavefronts' priorities and the weights without a look for the largest score 999, with them 958, with scalar addresses 900, with reads ordered ahead of the
// products and rows at a pitch 867 (half of the products of a tile stood waiting for LDS; a K tile further ahead, its products beside the exponentials, took 1040).
// ---------------------------------------------------------------------------------------
template <typename E, int D, bool ONE>
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
    const int r = (lane & 31) + 32 * (wave & 1), block = D == 128 ? 2 * (lane >> 5) + (wave >> 1) : lane >> 5;
    const bool has_k = D == 128 || wave < 2, has_v = D == 128 || wave >= 2;
    const int bits = src.power_bits(r) + 8 * block;              // of its power among four
    u32x4_t kn = {}, vn = {};
    uint32_t kp = 0, vp = 0, page = 0;
    MxOnePage<D> one;
    if (ONE && n > 0) one.init(src, key_of(0) + 32 * (wave & 1));
    auto look = [&](int32_t i) {
        if constexpr (!ONE) page = src.page_of(key_of(min(i, n - 1)) + r);
    };
    auto fetch = [&](int32_t i) {
        if constexpr (ONE) {
            const bool there = i < n;
            const auto [k, v, numbers, powers] = one.at(src, key_of(there ? i : 0) + 32 * (wave & 1), there);
            const int at = (lane & 31) * P::NUMBERS + block * 16, power_at = src.powers_at(lane & 31);
            if (has_k) {
                kn = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(k, at, numbers, 0));
                kp = __builtin_amdgcn_raw_buffer_load_b32(k, power_at, powers, 0);
            }
            if (has_v) {
                vn = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(v, at, numbers, 0));
                vp = __builtin_amdgcn_raw_buffer_load_b32(v, power_at, powers, 0);
            }
        } else {
            const int64_t at = src.page_at(page);
            const int32_t in = src.in_page(key_of(min(i, n - 1)) + r);
            const int64_t numbers = at + in * P::NUMBERS + block * 16, power = at + ((int64_t)P::NUMBERS << src.page_shift) + src.powers_at(in);
            if (has_k) { kn = ld16(as_global((const void *)src.k) + numbers); kp = ld4(as_global((const void *)src.k) + power); }
            if (has_v) { vn = ld16(as_global((const void *)src.v) + numbers); vp = ld4(as_global((const void *)src.v) + power); }
        }
    };
    MxColumns<E, D> w;
    if (n > 0) look(0);
    w.init(a, u, kv_head, wave * 32);
    if (n > 0) {
        fetch(0);
        look(1);
    }
    w.arrived();
    const int32_t low = min(u.lim0, u.key1);                     // keys that every column sees
    const float c = a.scale_log2;
    const int32_t full = min(n, max(0, (low - base) / ATTN_KEYS - skip));         // tiles that every column sees whole
    auto k_tile = [&](int32_t i) { return lds + (i & 1) * X::K_TILE; };
    auto v_tile = [&](int32_t i) { return lds + 2 * X::K_TILE + (i & 1) * X::V_TILE; };
    // tile i, which is in registers, to LDS; `bad`: for each 32 keys and 32 elements of the tile the keys that are NaN there
    auto put = [&](int32_t i) {
        if (has_k) mx4_put(k_tile(i) + r * X::K_PITCH + 64 * block, kn, mx4_power_of(kp, bits));
        if (has_v) {
            uint32_t power = mx4_power_of(vp, bits);
            if (i >= full) {
                const int32_t key = key_of(i) + r;
                const uint64_t nan = __ballot(mx4_clean(vn, power, key >= u.key0 && key < u.key1));
                if (lane % 32 == 0) bad[(i & 1) * 8 + (wave & 1) * 4 + block] = (uint32_t)(nan >> lane);
            }
            mx4_put(v_tile(i) + X::v_row(r) + 64 * block, vn, power);
        }
        if (i + 1 < n) fetch(i + 1);
        if (i + 2 < n) look(i + 2);
        __builtin_amdgcn_sched_barrier(0);                        // else it all stands among the products and takes their registers
    };
    if (n > 0) put(0);
    auto arrive = [&](int32_t i) {
        // this wavefront's share of tile i is in LDS and its reads of tile i - 1 are done, then everybody's
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (i + 1 < n) put(i + 1);
    };
    int32_t i = 0;
    if (__builtin_expect(wave * 32 >= u.ncols, 0)) {              // no columns: its share of the tiles only (100 requests of 10 rows over 1000..5000 tokens: 147 us, 170 with their products)
        for (; i < n; ++i) arrive(i);
        return;
    }
    for (; i < full; ++i) {
        arrive(i);
        const lds_t kt = k_tile(i), vt = v_tile(i);
        f32x16_t s[2];
        __builtin_amdgcn_s_setprio(1);                            // to the matrix cores first: the other wavefront of the unit has its exponentials in between
        s[0] = w.scores(kt, 0);
        s[1] = w.scores(kt, 32);
        w.order_scores();
        __builtin_amdgcn_s_setprio(0);
        if (i == 0 || __any(w.try_exponentials(s, c))) {          // (__any: a branch for all lanes, in the compiler's eyes too)
            if (i > 0) {
                s[0] = w.scores(kt, 0);
                s[1] = w.scores(kt, 32);
            }
            w.template exponentials<2>(s, c);
        }
        __builtin_amdgcn_s_setprio(1);
        w.add(vt, 0, s[0]);
        w.add(vt, 32, s[1]);
        w.order_sums();
        __builtin_amdgcn_s_setprio(0);
    }
    for (; i < n; ++i) {
        arrive(i);
        const lds_t kt = k_tile(i), vt = v_tile(i);
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
// 16 columns of a wavefront: decode rows of up to 16 query heads to a key/value head.  Products of 16x16x32: a lane has a quarter of one key's numbers, and 4 keys of 16 of one column
// of S^T.  As the right operand of the second product its keys of 32 are 4 g .. 4 g + 3 and 16 + 4 g .. (g = lane / 16), and V^T is read so.
// ---------------------------------------------------------------------------------------
template <typename E, int D> struct MxFewColumns {
    static constexpr int COLS = 16, PARTS = sizeof(E) == 2 ? 1 : 3;
    static constexpr int ROW = 2 * D, STEPS = D / 32, BLOCKS = D / 16, EACH = D / 4;      // EACH: elements of a key that a lane has
    u32x4_t qp[PARTS][STEPS];
    f32x4_t o[BLOCKS];
    float   m, l;
    int32_t lim, row, head;
    bool    valid;
    static __device__ __forceinline__ constexpr int v_row(int row) { return row * (ROW + 32) + (row >> 3) * 16; }       // as in MxTile: 32 bytes each of 8 rows are read
    static constexpr int V_BLOCK = 32 * (ROW + 34);

    __device__ __forceinline__ void init(const AttnArgs &a, const AttnUnit &u, int kv_head, int first)
    {
        const int lane = threadIdx.x & 63, g = lane >> 4;
        const AttnQuery r = attn_query(a, u, kv_head, first + (lane & 15));
        row = r.row; head = r.head; lim = r.lim; valid = r.valid;
        const gcptr_t from = as_global((const char *)a.q + (int64_t)row * a.ldq + ((int64_t)head * D + g * EACH) * (int)sizeof(E));
#pragma unroll
        for (int t = 0; t < STEPS; ++t) mx_query<E>(from + t * 8 * (int)sizeof(E), qp, t);
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) o[b] = f32x4_t{0, 0, 0, 0};
        m = ATTN_LOWEST;
        l = 0.0f;
    }
    __device__ __forceinline__ void arrived()
    {
#pragma unroll
        for (int p = 0; p < PARTS; ++p)
#pragma unroll
            for (int t = 0; t < STEPS; ++t) asm volatile("" : "+v"(qp[p][t]));
    }
    // the largest, and the sum, of a column's four lanes
    static __device__ __forceinline__ float most(float v)
    {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        return other_half_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
    }
    __device__ __forceinline__ float total() const
    {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(l), __float_as_uint(l), false, false);
        return both_halves_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
    }

    // S^T of 16 keys twice: a lane's quarter of its two keys
    struct Scores { f32x4_t s[2]; };
    __device__ __forceinline__ void scores(Scores &r, const uint32_t (&k)[2 * STEPS], const uint32_t (&powers)[2], int bits) const
    {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float scale = mx4_scale(mx4_power_of(powers[h], bits));
            r.s[h] = f32x4_t{0, 0, 0, 0};
#pragma unroll
            for (int t = 0; t < STEPS; ++t) {
                const bf16x8_t kt = __builtin_bit_cast(bf16x8_t, mx4_bf16(k[STEPS * h + t], scale));
#pragma unroll
                for (int p = PARTS - 1; p >= 0; --p) r.s[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kt, __builtin_bit_cast(bf16x8_t, qp[p][t]), r.s[h], 0, 0, 0);
            }
        }
    }
    __device__ __forceinline__ void hide_all(Scores &r, int32_t key, int32_t key0) const
    {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int32_t at = key + 16 * h + 4 * ((threadIdx.x & 63) >> 4) + i;
                r.s[h][i] = at < lim && at >= key0 ? r.s[h][i] : -INFINITY;
            }
    }
    __device__ __forceinline__ void exponentials(Scores &r, float c)
    {
        f32x4_t (&s)[2] = r.s;
        float top = s[0][0];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) top = fmaxf(top, s[h][i]);
        top = most(top) * c;
        if (__any(top > m + 8.0f)) {
            const float to = fmaxf(m, top), f = __builtin_amdgcn_exp2f(m - to);
            m = to;
            l *= f;
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[b][i] *= f;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[h][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[h][i], c, -m));
                l += s[h][i];
            }
    }
    // O^T += V^T P^T over the 32 keys of the V tile
    __device__ __forceinline__ void add_all(lds_t tile, const Scores &r)
    {
        const f32x4_t (&p)[2] = r.s;
        const int lane = threadIdx.x & 63, i = lane & 15;
        const lds_t at = tile + v_row(4 * (lane >> 4) + (i >> 2)) + (i & 3) * 8;
        union { uint32_t w[4]; bf16x8_t v; } pb[PARTS];
#pragma unroll
        for (int w = 0; w < 4; ++w) mx_weights<PARTS>(p[w >> 1][2 * w & 3], p[w >> 1][(2 * w & 3) + 1], [&](int k, uint32_t two) { pb[k].w[w] = two; });
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) {
            const lds_t from = at + 32 * b;
            const bf16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((PREFT_LDS bf16x4_t *)from);
            const bf16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((PREFT_LDS bf16x4_t *)(from + v_row(16)));
            const bf16x8_t v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
            for (int k = PARTS - 1; k >= 0; --k) o[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pb[k].v, o[b], 0, 0, 0);
        }
    }
    // as in MxColumns; b: 32 elements
    __device__ __forceinline__ void spoil(int b, uint32_t bad, int32_t key, int32_t key0)
    {
        if (bad & seen_keys(lim, key, key0)) {
#pragma unroll
            for (int i = 0; i < 4; ++i) o[2 * b][i] = o[2 * b + 1][i] = __uint_as_float(0x7fc00000u);
        }
    }
    // this lane's share of its column's sums, times f
    __device__ __forceinline__ void put(PREFT_LDS float *to, float f) const
    {
        const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) *(PREFT_LDS f32x4_t *)(to + b * 16 + 4 * g) = f32x4_t{o[b][0] * f, o[b][1] * f, o[b][2] * f, o[b][3] * f};
    }
    // the columns' results, or their part
    __device__ __forceinline__ void write(const AttnArgs &a, const AttnUnit &u, int kv_head) const
    {
        const int lane = threadIdx.x & 63, g = lane >> 4;
        const float sum = total();
        if (!valid) return;
        if (u.slot < 0) {
            const float f = inverse(sum);
            const gptr_t to = as_global((char *)a.out + (int64_t)row * a.ldo + ((int64_t)head * D + 4 * g) * (int)sizeof(E));
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) store4<E>(to + b * 16 * (int)sizeof(E), o[b][0] * f, o[b][1] * f, o[b][2] * f, o[b][3] * f);
        } else {
            const int64_t part = (int64_t)u.slot + kv_head * u.ncols + (lane & 15);
            const gptr_t to = as_global((void *)(a.s.l.part_o + part * D + 4 * g));
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) store4<float>(to + b * 64, o[b][0], o[b][1], o[b][2], o[b][3]);
            if (g == 0) a.s.l.part_ml[part] = make_float2(m, sum);
        }
    }
};

// ---------------------------------------------------------------------------------------
// A unit of up to 32 columns (C: MxColumns), or up to 16 (MxFewColumns): bound by the bytes of its keys.  The four wavefronts take blocks of 32 keys in turn, AHEAD of them on their way in
// registers, V through LDS of their own without a barrier, and join their sums at the end.  SOLO: the unit is one wavefront's.
// 512 rows over 4000 tokens, 32 heads over 8 of 128: 396 us, 5.65 TB/s; 224 rows over 256..4096 tokens 110 us with their schedule and join, 101-104 of them in the kernel under the profiler, 5.1-5.3 TB/s.
// Units of 32 columns on 32x32x16 products alone 117.7; powers loaded as bytes, after which a loop waits at its end for all loads, 114.  Four blocks ahead: 129 in pages of 16 (heads of 64: 48 us, two
// ahead 40, where their bytes would take 14: more loads on their way do not help, and what the time goes to is not known).
// ---------------------------------------------------------------------------------------
template <typename E, int D, typename C, int AHEAD, bool SOLO, bool ONE>
__device__ __forceinline__ void mx_attend_keys(const AttnArgs &a, const AttnUnit &u, int kv_head, lds_t lds, float *join)
{
    using X = MxTile<D>;
    using Stream = MxStream<D, C::COLS == 16, ONE>;
    const int wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63, r = lane & 31, half = lane >> 5;
    const lds_t vt = lds + wave * C::V_BLOCK;
    Stream st;
    st.init(a, u, kv_head, SOLO ? 0 : wave, SOLO ? 1 : 4);
    const int32_t n = st.n;
    typename Stream::Block on_way[AHEAD];
    C w;
    w.init(a, u, kv_head, 0);
    const float c = a.scale_log2;
    const int32_t full = st.whole(min(u.lim0, u.key1));
    if (n > 0) {
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) st.look(on_way[j], j);
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            st.fetch(on_way[j], j);
            st.look(on_way[j], j + AHEAD);
        }
    }
    w.arrived();
    auto block = [&](auto &b, int32_t i, bool more) {
        const int32_t key = st.key_of(i);
        typename C::Scores s;
        w.scores(s, b.k, b.kp, st.k_bits);
        u32x4_t v[X::MINE];
        uint32_t vp[X::MINE];
#pragma unroll
        for (int j = 0; j < X::MINE; ++j) { v[j] = b.v[j]; vp[j] = mx4_power_of(b.vp, st.v_bits + 8 * j); }
        uint64_t bad[X::MINE] = {};
        if (i >= full) {
            const int32_t mine = key + r;
#pragma unroll
            for (int j = 0; j < X::MINE; ++j) bad[j] = __ballot(mx4_clean(v[j], vp[j], mine >= u.key0 && mine < u.key1));
        }
        wait_lds_reads();                                         // of the block before
#pragma unroll
        for (int j = 0; j < X::MINE; ++j) mx4_put(vt + C::v_row(r) + 64 * (X::MINE * half + j), v[j], vp[j]);
        if (more) {
            st.fetch(b, i + AHEAD);
            st.look(b, i + 2 * AHEAD);
        }
        if (i >= full) w.hide_all(s, key, u.key0);
        w.exponentials(s, c);
        wait_lds_reads();                                         // written: nobody else's, so without a barrier
        w.add_all(vt, s);
        if (i >= full) {
#pragma unroll
            for (int j = 0; j < X::MINE; ++j) {
                w.spoil(j, (uint32_t)bad[j], key, u.key0);
                w.spoil(X::MINE + j, (uint32_t)(bad[j] >> 32), key, u.key0);
            }
        }
    };
    int32_t i = 0;
    for (; i + AHEAD <= n; i += AHEAD) {
#pragma unroll
        for (int q = 0; q < AHEAD; ++q) block(on_way[q], i + q, true);
    }
#pragma unroll
    for (int q = 0; q < AHEAD - 1; ++q)                           // a loop with a way out in its middle would be one that waits for all
        if (i + q < n) block(on_way[q], i + q, false);
    if constexpr (SOLO) w.write(a, u, kv_head);
    else join_waves<E, D>(a, u, w, kv_head, lds, join);
}

template <typename E, int D, bool SOLO>
__device__ __forceinline__ void mx_attend_narrow(const AttnArgs &a, const AttnUnit &u, int kv_head, lds_t lds, float *join)
{
    constexpr int AHEAD = 2, AHEAD_WIDE = sizeof(E) == 2 ? 2 : 1;             // as many as registers allow
    const bool one = a.page_shift >= 5;
    if (u.ncols <= MX_FEW_COLS) {
        if (one) mx_attend_keys<E, D, MxFewColumns<E, D>, AHEAD, SOLO, true>(a, u, kv_head, lds, join);
        else mx_attend_keys<E, D, MxFewColumns<E, D>, AHEAD, SOLO, false>(a, u, kv_head, lds, join);
    } else {
        if (one) mx_attend_keys<E, D, MxColumns<E, D>, AHEAD_WIDE, SOLO, true>(a, u, kv_head, lds, join);
        else mx_attend_keys<E, D, MxColumns<E, D>, AHEAD_WIDE, SOLO, false>(a, u, kv_head, lds, join);
    }
}

template <typename E, int D, bool DIRECT>
__global__ __launch_bounds__(256, 2) void attention_mx_kernel(AttnArgs a)
{
    using X = MxTile<D>;
    constexpr int JOIN = 4 * 32 * (D + 4) * 4, KIND = 2;
    __shared__ __align__(1024) char lds[X::LDS > JOIN ? X::LDS : JOIN];
    __shared__ float join[256];
    const int32_t unit = (DIRECT ? 0 : a.first) + (int32_t)blockIdx.x / a.s.kv_heads, kv_head = (int32_t)blockIdx.x % a.s.kv_heads;
    AttnUnit u;
    if constexpr (DIRECT) {
        if (a.ready && !attn_schedule_is(a, KIND)) return;
        if (!attn_direct_unit(a.s, unit, kv_head, a.ready != 0, u)) return;
        u.table = uniform(u.table); u.key0 = uniform(u.key0); u.key1 = uniform(u.key1); u.lim0 = uniform(u.lim0); u.ncols = uniform(u.ncols);
    } else {
        if (!attn_schedule_is(a, KIND)) return;
        // short units: one a wavefront, four a workgroup
        const int32_t units = as_const(a.s.l.header)[AH_UNITS], alone = as_const(a.s.l.header)[AH_SHORT];
        const uint32_t i = unit < alone ? (uint32_t)unit : (uint32_t)alone + 4u * (uint32_t)(unit - alone) + (uint32_t)uniform(threadIdx.x >> 6);     // units: fewer than 2^30
        if (i >= (uint32_t)units) return;
        const PREFT_CONST AttnUnit *p = as_const(a.s.l.units) + i;
        u.table = p->table; u.head0 = p->head0; u.ncols = p->ncols; u.key0 = p->key0; u.key1 = p->key1; u.row0 = p->row0; u.lim0 = p->lim0; u.slot = p->slot;
        if (unit >= alone) {
            if (u.ncols > 0) mx_attend_narrow<E, D, true>(a, u, kv_head, (lds_t)lds, join);
            return;
        }
    }
    if (u.ncols <= 0) return;
    if (u.ncols > ATTN_FEW_COLS) {
        if (a.page_shift >= 5) mx_attend_columns<E, D, true>(a, u, kv_head, (lds_t)lds, (uint32_t *)join);
        else mx_attend_columns<E, D, false>(a, u, kv_head, (lds_t)lds, (uint32_t *)join);
    }
    else mx_attend_narrow<E, D, false>(a, u, kv_head, (lds_t)lds, join);
}

}  // namespace preft
