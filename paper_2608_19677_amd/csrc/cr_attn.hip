// Attention of a destination: whole prompts (packed, causal, grouped heads) and requests that share a
// cached prefix in pages.
//
// Mathematics: scores s_j = scale q.k_j, running maximum m and sum l of exp(s_j - m) over the keys
// in one pass, o = sum_j exp(s_j - m) v_j / l, lse = m + ln l. Results over disjoint sets of keys
// are joined by lse = ln sum exp(lse_p), o = sum exp(lse_p - lse) o_p. Exponentials are taken base
// 2 with log2(e) folded into the scale.
//
// The weights exp(s_j - m) are rounded to 16 bits for the second product. l for the lse is summed
// before that; what o is divided by is the sum of the rounded weights, so that a row that leans on
// few keys keeps their values exactly (divided by l, the rounding of one large weight would scale the
// whole row, up to 2^-8).
#include "cr_kv.h"

#include <type_traits>

// Code of the tile loops is inlined whatever its size: its arrays live in registers only so.
#define CR_INLINE __attribute__((always_inline))

namespace cr {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr uint32_t kWaves = 4;
constexpr uint32_t kThreads = kWaves * kWave;
constexpr uint32_t kKeys = 64;           // keys per tile
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kNoMax = -3.0e38f;       // running maximum before the first key
constexpr float kSlack = 8.f;            // weights may reach 2^kSlack before the maximum is moved

struct Bf16 {
    static constexpr float kLift = 0.f;
    static constexpr uint32_t kInf = 0x7F80u;
    static __device__ __forceinline__ float wide(uint32_t x) { return __uint_as_float(x << 16); }  // of 16 bits
    static __device__ __forceinline__ f32x16 mfma(s16x8 a, s16x8 b, f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint32_t pack(float x, float y)
    {
        return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x, y}), bf16x2));
    }
    static __device__ __forceinline__ float add(uint32_t two, float sum)  // sum + both elements
    {
        return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, two), __builtin_bit_cast(bf16x2, 0x3F803F80u), sum, false);
    }
};

// The largest weight lies between 2^kLift and 2^(kLift + kSlack), so that 16 bits hold weights down to 2^-30
// of it at least; around 1 those below 2^-24 would be lost, and many of them may add up.
struct F16 {
    static constexpr float kLift = 6.f;
    static constexpr uint32_t kInf = 0x7C00u;
    static __device__ __forceinline__ float wide(uint32_t x) { return (float)__builtin_bit_cast(_Float16, (uint16_t)x); }
    static __device__ __forceinline__ f32x16 mfma(s16x8 a, s16x8 b, f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint32_t pack(float x, float y)
    {
        return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x, y}), f16x2));
    }
    static __device__ __forceinline__ float add(uint32_t two, float sum)
    {
        return __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, two), __builtin_bit_cast(f16x2, 0x3C003C00u), sum, false);
    }
};

// The stretches of keys a call works on.
enum Kind : uint32_t {
    kPrompt,  // a sequence's keys
    kGroup,   // a group's prefix, for all rows of its requests
    kOwn,     // a request's own tokens
    kWhole,   // a request's prefix and own tokens, one after the other
};

struct Attn {
    cr_rows q, k, v, out;  // k, v: prompt only
    float* lse;
    KvPages pg;            // shared only, k and v at the call's layer
    const uint32_t* q_off;
    const uint32_t* k_off;         // prompt
    const uint32_t* group_off;     // shared
    const uint32_t* prefix_table;
    const uint32_t* prefix_len;
    const uint32_t* own_table;
    const uint32_t* own_len;
    uint32_t prefix_width, own_width;
    uint32_t heads_q, heads_kv, group, batch, groups, total_q, total_k, causal;
    float c;               // scale * log2(e)
    // A sequence's keys are cut into chunks of at least `chunk` and at most as many as there are slots;
    // chunk i's results go to slot i, of the own parts of a call that joins them with prefixes to slot
    // `slots` + i.
    uint32_t chunk, slots, own_chunk, own_slots;
    uint32_t least_share;  // narrow kernel: tiles a block takes at least, so that no sequence needs more slots
    float* part_o;         // f32 [slots + own_slots][total_q * heads_q][dim], NULL: results are final
    float* part_lse;       // f32 [slots + own_slots][total_q * heads_q], base 2
    uint32_t* err;
};

// A stretch of keys with the rows that see it. Row m is query token tok0 + m / group and sees keys
// below max(least, first_lim + m / group) (causal) or all n. In pages, keys 0 .. len0 are the first
// table's and keys gap_end .. n the second's; gap_end is len0 rounded up to whole tiles, so that a
// tile has keys of one table, and the keys between are seen by no row.
struct Seq {
    uint32_t tok0, nq, n;
    int32_t first_lim, least;
    uint32_t causal;
    uint32_t key0;             // prompt: first key row
    uint32_t len0, gap_end;
    const uint32_t* table0;
    const uint32_t* table1;
};

__device__ __forceinline__ bool bad_seq(const Attn& a)
{
    if (threadIdx.x == 0) atomicOr(a.err, CR_ERR_SEQ);
    return false;
}

template <bool kPaged>
__device__ __forceinline__ bool get_seq(const Attn& a, uint32_t kind, uint32_t x, Seq* s)
{
    uint32_t r0 = x, r1 = x + 1u;
    if (kPaged && kind == kGroup) {
        r0 = a.group_off[x];
        r1 = a.group_off[x + 1u];
        if (r0 > r1 || r1 > a.batch) return bad_seq(a);
        if ((x == 0u && r0 != 0u) || (x + 1u == a.groups && r1 != a.batch)) bad_seq(a);  // requests without a group
    }
    const uint32_t t0 = a.q_off[r0], t1 = a.q_off[r1];
    if (t0 > t1 || t1 > a.total_q) return bad_seq(a);
    if ((r0 == 0u && t0 != 0u) || (r1 == a.batch && t1 != a.total_q)) bad_seq(a);  // rows without a sequence
    s->tok0 = t0;
    s->nq = t1 - t0;
    s->least = 0;
    if (!kPaged) {
        const uint32_t k0 = a.k_off[x], k1 = a.k_off[x + 1u];
        if (k0 > k1 || k1 > a.total_k) return bad_seq(a);
        s->n = k1 - k0;
        s->key0 = k0;
        s->causal = a.causal;
    } else {
        uint32_t pre = 0, own = 0;
        if (kind != kOwn) {
            const uint32_t g = kind == kGroup ? x : wave_find(a.groups, x, [&](uint32_t i) { return a.group_off[i]; });
            if (kind != kGroup && (a.group_off[g] > x || a.group_off[g + 1u] <= x)) return bad_seq(a);
            pre = a.prefix_len[g];
            if (pages_of(pre, a.pg.log_tokens) > a.prefix_width) return bad_seq(a);
            s->table0 = a.prefix_table + (uint64_t)g * a.prefix_width;
        }
        if (kind != kGroup) {
            own = a.own_len[x];
            if (pages_of(own, a.pg.log_tokens) > a.own_width) return bad_seq(a);
            s->table1 = a.own_table + (uint64_t)x * a.own_width;
        }
        s->len0 = pre;
        s->gap_end = (pre + kKeys - 1u) / kKeys * kKeys;
        s->n = kind == kGroup ? pre : s->gap_end + own;
        s->causal = kind != kGroup;
        s->least = (int32_t)s->gap_end;
    }
    s->first_lim = s->causal ? (int32_t)s->n - (int32_t)s->nq + 1 : (int32_t)s->n;
    return true;
}

// Keys that row m of a sequence sees.
__device__ __forceinline__ uint32_t row_limit(const Attn& a, const Seq& s, uint32_t m)
{
    return s.causal ? (uint32_t)max(s.least, s.first_lim + (int32_t)(m / a.group)) : s.n;
}

// Keys per chunk of a sequence of n keys, and the number of its chunks.
constexpr uint32_t kChunkUnit = 128;
__device__ __forceinline__ uint32_t chunk_of(uint32_t n, uint32_t chunk, uint32_t slots)
{
    return max(chunk, ((n + slots - 1u) / slots + kChunkUnit - 1u) / kChunkUnit * kChunkUnit);
}

__device__ __forceinline__ uint32_t chunks_of(uint32_t n, uint32_t chunk, uint32_t slots)
{
    const uint32_t c = chunk_of(n, chunk, slots);
    return (n + c - 1u) / c;
}

// Tiles in LDS, in elements. Keys: pieces of 16 bytes, all rows of one piece together (a lane reads a
// row's piece, so 16 lanes read 256 contiguous bytes). Values: 32 elements, all rows of them together
// (a transposed read takes 4 rows of 64 bytes by 32 lanes, 256 contiguous bytes). Each run is
// shifted against the one before, so that the pieces of one row, which lie next to each other
// in memory and are written together, fall on different banks. All reads of a tile are one lane
// address and constants.
constexpr uint32_t key_run(uint32_t keys) { return keys * 8u + 8u; }
constexpr uint32_t val_run(uint32_t keys) { return keys * 32u + 32u; }
constexpr uint32_t key_tile(uint32_t keys, uint32_t dim) { return dim / 8u * key_run(keys); }
constexpr uint32_t val_tile(uint32_t keys, uint32_t dim) { return dim / 32u * val_run(keys); }

__device__ __forceinline__ s16x4 read_tr(const uint16_t* p)
{
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (__attribute__((address_space(3))) s16x4*)(__attribute__((address_space(3))) void*)const_cast<uint16_t*>(p));
}

// Keeps the computation of x here: the compiler would move it past the next branch, to its first use.
template <typename T>
__device__ __forceinline__ void stay(T& x)
{
    asm volatile("" : "+v"(x));
}

// The larger of a column's values in the two half-waves, and their sum.
__device__ __forceinline__ float both_max(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __builtin_elementwise_maximum(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

__device__ __forceinline__ float both_sum(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Tiles of kTile keys and values on their way from memory to LDS, moved by kMovers threads: each
// moves one 16-byte piece of every kStep-th row.
template <int kDim, bool kPaged, uint32_t kTile, uint32_t kMovers>
struct Loader {
    static constexpr uint32_t kPieces = kDim / 8, kStep = kMovers / kPieces, kPer = kTile / kStep;
    static constexpr uint32_t kWaveRows = kWave / kPieces;  // rows that a wavefront moves at once
    // Longest stride whose lane offsets, up to kWaveRows - 1 rows and a piece, stay in 32 bits.
    static constexpr uint32_t kLaneStride = (0xFFFFFFFFu - kDim) / (kWaveRows - 1u);
    const uint16_t *kb, *vb;  // of the key head (prompt: at the sequence's first key)
    uint32_t row, piece, end, lane_k, lane_v, bad;
    uint32_t page[kPer];      // of the next tile's rows
    u32x4 rk[kPer], rv[kPer];

    __device__ __forceinline__ void init(const Attn& a, const Seq& s, uint32_t head_kv, uint32_t last, uint32_t mover)
    {
        piece = mover % kPieces;
        row = mover / kPieces;
        end = last;
        if (kPaged) {
            kb = a.pg.k + (int64_t)head_kv * a.pg.head_stride;
            vb = a.pg.v + (int64_t)head_kv * a.pg.head_stride;
            lane_k = lane_v = row % kWaveRows * (uint32_t)a.pg.token_stride + piece * 8u;
        } else {
            kb = (const uint16_t*)a.k.p + (int64_t)head_kv * a.k.head_stride + (int64_t)s.key0 * a.k.token_stride;
            vb = (const uint16_t*)a.v.p + (int64_t)head_kv * a.v.head_stride + (int64_t)s.key0 * a.v.token_stride;
            lane_k = row % kWaveRows * (uint32_t)a.k.token_stride + piece * 8u;
            lane_v = row % kWaveRows * (uint32_t)a.v.token_stride + piece * 8u;
        }
    }
    // The table of the tile at k0, its first key there, and the end of the keys in it (keys end at `stop`).
    static __device__ __forceinline__ const uint32_t* place(const Seq& s, uint32_t k0, uint32_t stop, uint32_t* first, uint32_t* last)
    {
        const bool second = k0 >= s.gap_end && stop > s.gap_end;
        *first = second ? k0 - s.gap_end : k0;
        *last = second ? stop - s.gap_end : min(stop, s.len0);
        return second ? s.table1 : s.table0;
    }
    static __device__ __forceinline__ void pages_of_tile(const Attn& a, const Seq& s, uint32_t k0, uint32_t stop, uint32_t row,
                                                         uint32_t (&to)[kPer])
    {
        if (!kPaged) return;
        uint32_t first, last;
        const uint32_t* table = place(s, k0, stop, &first, &last);
#pragma unroll
        for (uint32_t p = 0; p < kPer; ++p) to[p] = table[min(first + p * kStep + row, last - 1u) >> a.pg.log_tokens];
    }
    __device__ __forceinline__ void pages(const Attn& a, const Seq& s, uint32_t k0) { pages_of_tile(a, s, k0, end, row, page); }
    // Whole tiles whose rows of one wavefront and pass lie in one page and not too far apart: scalar addresses.
    // Otherwise an address per lane; rows behind the last key repeat it: their weights are 0, and nothing foreign is
    // read.
    __device__ __forceinline__ void load(const Attn& a, const Seq& s, uint32_t k0)
    {
        const uint32_t mask = (1u << a.pg.log_tokens) - 1u;
        uint32_t first = k0, last = end;
        if (kPaged) place(s, k0, end, &first, &last);
        const bool near = kPaged ? mask >= kWaveRows - 1u && (uint32_t)a.pg.token_stride <= kLaneStride
                                 : max((uint32_t)a.k.token_stride, (uint32_t)a.v.token_stride) <= kLaneStride;
        if (first + kTile <= last && near) {
            const uint32_t r0 = __builtin_amdgcn_readfirstlane(row);
#pragma unroll
            for (uint32_t p = 0; p < kPer; ++p) {
                const uint32_t j = first + p * kStep + r0;
                int64_t ak, av;
                if (kPaged) {
                    uint32_t g = __builtin_amdgcn_readfirstlane(page[p]);
                    bad |= g >= a.pg.num_pages;
                    g = min(g, a.pg.num_pages - 1u);
                    ak = av = (int64_t)((uint64_t)g * (uint32_t)a.pg.page_stride + (uint64_t)(j & mask) * (uint32_t)a.pg.token_stride);
                } else {
                    ak = (int64_t)((uint64_t)j * (uint32_t)a.k.token_stride);
                    av = (int64_t)((uint64_t)j * (uint32_t)a.v.token_stride);
                }
                rk[p] = *reinterpret_cast<const u32x4*>(kb + ak + lane_k);
                rv[p] = *reinterpret_cast<const u32x4*>(vb + av + lane_v);
            }
        } else {
#pragma unroll
            for (uint32_t p = 0; p < kPer; ++p) {
                const uint32_t j = min(first + p * kStep + row, last - 1u);
                int64_t ak, av;
                if (kPaged) {
                    uint32_t g = page[p];
                    bad |= g >= a.pg.num_pages;
                    g = min(g, a.pg.num_pages - 1u);
                    ak = av = (int64_t)((uint64_t)g * (uint32_t)a.pg.page_stride + (uint64_t)(j & mask) * (uint32_t)a.pg.token_stride);
                } else {
                    ak = (int64_t)((uint64_t)j * (uint32_t)a.k.token_stride);
                    av = (int64_t)((uint64_t)j * (uint32_t)a.v.token_stride);
                }
                rk[p] = *reinterpret_cast<const u32x4*>(kb + ak + piece * 8u);
                rv[p] = *reinterpret_cast<const u32x4*>(vb + av + piece * 8u);
            }
        }
    }
    __device__ __forceinline__ void report(const Attn& a) const
    {
        if (kPaged && bad) atomicOr(a.err, CR_ERR_PAGE);
    }
    __device__ __forceinline__ void store(uint16_t* lk, uint16_t* lv) const
    {
#pragma unroll
        for (uint32_t p = 0; p < kPer; ++p) {
            const uint32_t r = p * kStep + row;
            *reinterpret_cast<u32x4*>(lk + piece * key_run(kTile) + r * 8u) = rk[p];
            *reinterpret_cast<u32x4*>(lv + (piece >> 2) * val_run(kTile) + r * 32u + (piece & 3u) * 8u) = rv[p];
        }
    }
};

// Values that are not finite. A weight of 0 times such a value is not 0, so the products of a half tile that some
// rows see in part carry it to rows that do not see it. Sums that are not finite show that it may have happened; the wave
// then looks at the values from its first row's end on, and if there is one among them does its products once more,
// straight from memory, with 0 in its place, and adds it to the rows that see it. Where all is finite that is the look at
// the sums and a few registers: 24 prompts of about 300 tokens 39.9 -> 40.5 us, a decode step behind one prefix 35.1 -> 35.7,
// long prompts within 0.5 %. (Checked on their way to LDS, the values of such tiles took 10 % of the short prompts.)
template <int kDim>
__device__ __forceinline__ bool all_finite(const f32x16 (&o)[kDim / 32])
{
    float top = 0.f;
#pragma unroll
    for (int d = 0; d < kDim / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 2)
            top = __builtin_elementwise_maximum(__builtin_elementwise_maximum(top, __builtin_fabsf(o[d][i])), __builtin_fabsf(o[d][i + 1]));
    return ballot(!(top < INFINITY)) == 0;
}

// The wave's rows are row .. last_row (repeated) of the sequence, its half tiles at first, first + step, ... below stop;
// keys are read up to key_end, and all of its rows see `full` of them. The running maximum moves as it did in the first run,
// so that all other sums come out the same, bit for bit.
template <typename E, int kDim, bool kPaged>
__device__ CR_INLINE void only_seen(const Attn& a, const Seq& it, uint32_t head_kv, uint32_t row, uint32_t last_row, uint32_t first, uint32_t step,
                                    uint32_t stop, uint32_t key_end, uint32_t full, f32x16 (&o)[kDim / 32])
{
    uint32_t lane = lane_id();
    stay(lane);  // what follows from it is computed again, not kept over the loop before
    const uint32_t half = lane >> 5, col = lane & 31u, m = min(row + col, last_row);
    const int32_t lim = (int32_t)min(row_limit(a, it, m), key_end);
    const uint16_t* qp = (const uint16_t*)a.q.p + (int64_t)(it.tok0 + m / a.group) * a.q.token_stride +
                         (int64_t)(head_kv * a.group + m % a.group) * a.q.head_stride;
    // Row r of the half tile at k0, the last one repeated: its place in k or v.
    auto at = [&](const uint16_t* k_or_v, const cr_rows& rows, uint32_t k0, uint32_t r) CR_INLINE {
        uint32_t j = k0, last = key_end;
        if (kPaged) {
            const uint32_t* table = Loader<kDim, true, 32, kWave>::place(it, k0, key_end, &j, &last);
            j = min(j + r, last - 1u);
            const uint32_t g = min(table[j >> a.pg.log_tokens], a.pg.num_pages - 1u), mask = (1u << a.pg.log_tokens) - 1u;
            return k_or_v + (int64_t)head_kv * a.pg.head_stride + (int64_t)g * a.pg.page_stride + (int64_t)(j & mask) * a.pg.token_stride;
        }
        return (const uint16_t*)rows.p + (int64_t)head_kv * rows.head_stride + ((int64_t)it.key0 + min(j + r, last - 1u)) * rows.token_stride;
    };
    auto not_finite = [&](uint32_t x) CR_INLINE { return (x & 0x7FFFu) >= E::kInf; };
    const uint32_t part = first + (full >= first + 32u ? (full - first - 32u) / step + 1u : 0u) * step;  // the first half tile seen in part
    bool any = false;
    for (uint32_t k0 = part; k0 < key_end; k0 += step) {
        const uint16_t* v = at(a.pg.v, a.v, k0, col);
        for (uint32_t e = half * 8u; e < kDim; e += 16u) {
            const u32x4 x = *reinterpret_cast<const u32x4*>(v + e);
#pragma unroll
            for (int y = 0; y < 4; ++y) any |= not_finite(x[y]) || not_finite(x[y] >> 16);
        }
    }
    if (__builtin_expect(!ballot(any), 1)) return;

    float mc = kNoMax;
#pragma unroll
    for (int d = 0; d < kDim / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
    for (uint32_t k0 = first; k0 < stop; k0 += step) {
        f32x16 s;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.f;
        const uint16_t* k = at(a.pg.k, a.k, k0, col);
#pragma unroll
        for (int d = 0; d < kDim / 16; ++d)
            s = E::mfma(*reinterpret_cast<const s16x8*>(k + d * 16 + half * 8u), *reinterpret_cast<const s16x8*>(qp + d * 16 + half * 8u), s);
        const int32_t l = kPaged && k0 < it.gap_end ? min(lim, (int32_t)it.len0) : lim;
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if ((int32_t)(k0 + 8u * (i / 4) + 4u * half + (i & 3)) >= l) s[i] = -INFINITY;
            top = __builtin_elementwise_maximum(top, s[i]);
        }
        top = both_max(top) * a.c;
        if (ballot(top > mc + (kSlack + E::kLift))) {
            const float up = fmaxf(mc, top - E::kLift), f = __builtin_amdgcn_exp2f(mc - up);
            mc = up;
#pragma unroll
            for (int d = 0; d < kDim / 32; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= f;
        }
        uint32_t pk[8];
#pragma unroll
        for (int i = 0; i < 16; i += 2)
            pk[i / 2] = E::pack(__builtin_amdgcn_exp2f(__builtin_fmaf(s[i], a.c, -mc)), __builtin_amdgcn_exp2f(__builtin_fmaf(s[i + 1], a.c, -mc)));
        const bool in_part = k0 >= part;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            const u32x4 w = {pk[ks * 4], pk[ks * 4 + 1], pk[ks * 4 + 2], pk[ks * 4 + 3]};
            s16x8 vf[kDim / 32];
#pragma unroll
            for (int y = 0; y < 8; ++y) {
                const uint16_t* v = at(a.pg.v, a.v, k0, ks * 16u + (y / 4) * 8u + half * 4u + (y & 3)) + col;
#pragma unroll
                for (int d = 0; d < kDim / 32; ++d) {
                    const uint16_t x = v[d * 32];
                    vf[d][y] = (short)(in_part && not_finite(x) ? 0u : x);
                }
            }
#pragma unroll
            for (int d = 0; d < kDim / 32; ++d) o[d] = E::mfma(vf[d], __builtin_bit_cast(s16x8, w), o[d]);
        }
    }
    for (uint32_t k0 = part; k0 < stop; k0 += step)
        for (uint32_t r = 0; r < 32u && (int32_t)(k0 + r) < lim; ++r) {
            const uint16_t* v = at(a.pg.v, a.v, k0, r);
#pragma unroll
            for (int d = 0; d < kDim / 32; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const uint32_t x = v[d * 32 + 8 * (i / 4) + 4u * half + (i & 3)];
                    if (not_finite(x)) o[d][i] += E::wide(x);
                }
        }
}

// A wavefront keeps 32 rows, each in one column: S^T = K Q^T gives a lane its row's scores of 16 of 32
// keys (the other half-wave has the other 16), so the row's maximum needs one exchange, and the
// weights are the second operand of O^T = V^T P^T as they lie: the order of keys inside a
// product is the same on both sides, 4 + 4 of 16 per half-wave, which is what two transposed LDS
// reads of the values give.
//
// The wave works on half tiles of 32 keys, three of them at a time: the scores of the next and the
// values of the last on the matrix unit, and between these products the weights of the one between
// and the maximum of the next on the vector unit. The maximum is moved, and what is summed rescaled,
// only when a score passes it by 2^kSlack.
//
// kW wavefronts share the tiles. Eight (256 rows) read a tile from memory for twice the rows that four
// do; four are for sequences of fewer rows. Values have three buffers where a block has a compute
// unit to itself (one barrier per tile), else two and a barrier more.
//
// Bound by the matrix and vector units: one prompt of 16,384 tokens (64 heads of 128 on 8 key heads) runs at 990 to
// 1,050 TFLOP/s on different cards, matrix units 48 % busy, no LDS conflicts; a tile of 64 keys takes 256 rows
// 2.1 us, a block's start and end about 6 us: eight prompts of 1,000 to 4,100 tokens 830 to 850 TFLOP/s.
struct Part {
    uint32_t kind, tiles, blocks;  // blocks: tiles x slots x key heads
    uint32_t sorted;               // sequences in the order of their keys, the longest first
};

// The tile of a rank where sequences follow each other by falling numbers of keys, each with its last tile
// first: a call of several rounds of blocks then ends with short ones. For up to 64 sequences, one a lane;
// what does not fit has no tiles. false: no such tile. Calls of one round of blocks gain nothing and keep the
// order of the sequences; suffixes of hits behind prefixes of 1,000 to 9,000 tokens take 407 us so, 430 without.
constexpr uint32_t kSortSeqs = 64;

template <bool kPaged, uint32_t kRows>
__device__ __forceinline__ bool longest_first(const Attn& a, uint32_t kind, uint32_t rank, uint32_t* x, uint32_t* row0)
{
    const uint32_t lane = lane_id(), seqs = kPaged && kind == kGroup ? a.groups : a.batch, y = min(lane, seqs - 1u);
    uint32_t r0 = y, r1 = y + 1u, n;
    bool ok = true, covers = true;
    if (kPaged) {
        const uint32_t g = min(lane, a.groups - 1u), g0 = a.group_off[g], g1 = a.group_off[g + 1u], prefix = a.prefix_len[g];
        covers = (g != 0u || g0 == 0u) && (g + 1u != a.groups || g1 == a.batch);
        if (kind == kGroup) {
            r0 = g0;
            r1 = g1;
            ok = r0 <= r1 && r1 <= a.batch;
            n = prefix;
        } else {
            n = a.own_len[y];
            if (kind == kWhole) {
                uint32_t of = 0;
                for (uint32_t j = 1; j < a.groups; ++j) of = (uint32_t)__builtin_amdgcn_readlane((int)g0, (int)j) <= y ? j : of;
                n += (uint32_t)__shfl((int)prefix, (int)of);
            }
        }
    } else {
        const uint32_t k0 = a.k_off[y], k1 = a.k_off[y + 1u];
        covers = k0 <= k1 && k1 <= a.total_k;
        n = k1 - k0;
    }
    uint32_t t0 = 0, t1 = 0;
    if (ok) {
        t0 = a.q_off[r0];
        t1 = a.q_off[r1];
        ok = t0 <= t1 && t1 <= a.total_q;
        covers = covers && (r0 != 0u || t0 == 0u) && (r1 != a.batch || t1 == a.total_q);
    }
    if (!ok || !covers) atomicOr(a.err, CR_ERR_SEQ);
    const uint32_t tiles = ok && lane < seqs ? ((t1 - t0) * a.group + kRows - 1u) / kRows : 0u;
    uint32_t before = 0;  // tiles of longer sequences
    for (uint32_t j = 0; j < seqs; ++j) {
        const uint32_t nj = (uint32_t)__builtin_amdgcn_readlane((int)n, (int)j), tj = (uint32_t)__builtin_amdgcn_readlane((int)tiles, (int)j);
        before += nj > n || (nj == n && j < lane) ? tj : 0u;
    }
    const uint64_t mine = ballot(before <= rank && rank - before < tiles);
    if (!mine) return false;
    const uint32_t l = (uint32_t)__builtin_ctzll(mine);
    *x = l;
    *row0 = ((uint32_t)__builtin_amdgcn_readlane((int)tiles, (int)l) - 1u - (rank - (uint32_t)__builtin_amdgcn_readlane((int)before, (int)l))) * kRows;
    return true;
}

constexpr uint32_t val_bufs(uint32_t waves) { return waves == 8u ? 3u : 2u; }
constexpr uint32_t wide_lds(uint32_t waves, uint32_t dim)  // elements
{
    return 2u * key_tile(kKeys, dim) + val_bufs(waves) * val_tile(kKeys, dim);
}

template <typename E, int kDim, bool kPaged, uint32_t kW>
__device__ CR_INLINE void wide_block(const Attn& a, const Part& part_of, uint32_t block, uint16_t* lds)
{
    constexpr uint32_t kRows = kW * 32u;  // of the block
    constexpr uint32_t kKeyRun = key_run(kKeys), kValRun = val_run(kKeys), kValBufs = val_bufs(kW);
    auto lds_k = [&](uint32_t i) CR_INLINE { return lds + i * key_tile(kKeys, kDim); };
    auto lds_v = [&](uint32_t i) CR_INLINE { return lds + 2u * key_tile(kKeys, kDim) + i * val_tile(kKeys, kDim); };
    const uint32_t kind = part_of.kind, tiles = part_of.tiles;

    // Tiles of sequence x start at floor(first row / kRows) + x: steps of at least ceil(rows / kRows),
    // so the tiles of all sequences fit into floor(all rows / kRows) + sequences without a pass that
    // counts them; some are empty. The last rows of causal sequences, the longest, come first. Where the
    // blocks are more than one round of few sequences, the longest sequences do too.
    const uint32_t head_kv = block % a.heads_kv, id = block / a.heads_kv;
    const uint32_t slots = kind == kOwn ? a.own_slots : a.slots;
    const uint32_t split = id / tiles, tile = tiles - 1u - id % tiles;  // tiles that read the same keys side by side
    auto start = [&](uint32_t x) {
        return a.q_off[kPaged && kind == kGroup ? min(a.group_off[x], a.batch) : x] * a.group / kRows + x;
    };
    uint32_t x, row0;
    if (part_of.sorted) {
        if (!longest_first<kPaged, kRows>(a, kind, id % tiles, &x, &row0)) return;
    } else {
        x = wave_find(kPaged && kind == kGroup ? a.groups : a.batch, tile, start);
        row0 = (tile - min(start(x), tile)) * kRows;
    }
    Seq it;
    if (!get_seq<kPaged>(a, kind, x, &it)) return;
    const uint32_t seq_rows = it.nq * a.group;
    if (row0 >= seq_rows) return;
    const uint32_t rows = min(kRows, seq_rows - row0);
    const uint32_t chunk = chunk_of(it.n, kind == kOwn ? a.own_chunk : a.chunk, slots), key_begin = split * chunk;
    const uint32_t key_end = min(row_limit(a, it, row0 + rows - 1u), key_begin + chunk);

    const uint32_t lane = lane_id(), wv = wave_in_block(), half = lane >> 5, col = lane & 31u;
    const uint32_t wrow = wv * 32u;  // the wave's first row
    const uint32_t m = row0 + min(wrow + col, rows - 1u);
    const uint32_t tok = it.tok0 + m / a.group, head = head_kv * a.group + m % a.group;
    const int32_t lim = (int32_t)min(row_limit(a, it, m), key_end);
    // keys that the wave's last and first rows see
    uint32_t w_end = 0, w_full = key_end;
    if (wrow < rows) {
        w_end = min(row_limit(a, it, row0 + min(wrow + 32u, rows) - 1u), key_end);
        w_full = min(row_limit(a, it, row0 + wrow), key_end);
    }

    f32x16 o[kDim / 32];
    float mc = kNoMax, sum = 0.f, rounded = 0.f;  // sums of the weights and of the rounded ones
#pragma unroll
    for (int d = 0; d < kDim / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.f;

    if (key_begin < key_end) {
        Loader<kDim, kPaged, kKeys, kW * kWave> ld;
        ld.bad = 0;
        ld.init(a, it, head_kv, key_end, threadIdx.x);
        ld.pages(a, it, key_begin);
        ld.load(a, it, key_begin);
        ld.pages(a, it, key_begin + kKeys);
        constexpr int kSteps = kDim / 16;  // products of a half tile's scores, and of its values
        s16x8 qf[kSteps];
        const uint16_t* qp = (const uint16_t*)a.q.p + (int64_t)tok * a.q.token_stride + (int64_t)head * a.q.head_stride;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) qf[s] = *reinterpret_cast<const s16x8*>(qp + s * 16 + half * 8u);

        f32x16 s[2];            // scores of the two halves of a tile
        uint32_t pk[2][8];      // their weights
        float top, part[2], part_rounded;
        float late = 1.f;       // factor that o lacks: its values come a half tile after their weights
        bool is_late = false;
        const uint32_t k_lane = half * kKeyRun + col * 8u;
        const uint32_t v_lane = (half * 4u + (lane & 15u) / 4u) * 32u + ((lane >> 4) & 1u) * 16u + (lane & 3u) * 4u;

        // Fragment d of half tile h of the keys in lk; fragment n of the values in lv: 16 keys
        // n / (kDim / 32) by 32 elements n % (kDim / 32).
        auto key_frag = [&](const uint16_t* lk, int h, int d) CR_INLINE {
            return *reinterpret_cast<const s16x8*>(lk + k_lane + d * 2u * kKeyRun + h * 32u * 8u);
        };
        auto val_frag = [&](const uint16_t* lv, int h, int n) CR_INLINE {
            const uint16_t* p = lv + v_lane + n % (kDim / 32) * kValRun + (h * 32u + n / (kDim / 32) * 16u) * 32u;
            const s16x4 x = read_tr(p), y = read_tr(p + 8u * 32u);
            return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
        };
        auto mask = [&](uint32_t k0, int h) CR_INLINE {
            const int32_t l = kPaged && k0 < it.gap_end ? min(lim, (int32_t)it.len0) : lim;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if ((int32_t)(k0 + h * 32u + 8u * (i / 4) + 4u * half + (i & 3)) >= l) s[h][i] = -INFINITY;
        };
        // Whether every row of the wave sees the second half of the tile at k0 and the first of the next.
        auto whole = [&](uint32_t k0) CR_INLINE {
            bool w = k0 + kKeys + 32u <= w_full;
            if (kPaged) w = w && (k0 + kKeys + 32u <= it.len0 || k0 >= it.gap_end);
            return w;
        };
        auto maximum = [&](int h, int i) CR_INLINE {  // over scores i and i + 1
            top = __builtin_elementwise_maximum(__builtin_elementwise_maximum(i ? top : s[h][i], s[h][i]), s[h][i + 1]);
        };
        auto scale_o = [&](float f) CR_INLINE {
#pragma unroll
            for (int d = 0; d < kDim / 32; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= f;
        };
        auto move_maximum = [&]() CR_INLINE {
            top = both_max(top) * a.c;
            stay(top);
            if (is_late) {
                scale_o(late);
                is_late = false;
            }
            if (ballot(top > mc + (kSlack + E::kLift))) {
                const float up = fmaxf(mc, top - E::kLift);
                late = __builtin_amdgcn_exp2f(mc - up);
                is_late = true;
                sum *= late;
                rounded *= late;
                mc = up;
            }
        };
        auto weight = [&](int h, int i) CR_INLINE {  // of scores i and i + 1
            const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[h][i], a.c, -mc));
            const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(s[h][i + 1], a.c, -mc));
            part[0] = i ? part[0] + x : x;
            part[1] = i ? part[1] + y : y;
            if (i) part_rounded = E::add(pk[h][i / 2 - 1], i > 2 ? part_rounded : 0.f);  // of the pair before: packed some cycles ago
            pk[h][i / 2] = E::pack(x, y);
            stay(pk[h][i / 2]);
        };
        auto value = [&](s16x8 vf, int h, int n) CR_INLINE {
            const int ks = n / (kDim / 32), d = n % (kDim / 32);
            const u32x4 w = {pk[h][ks * 4], pk[h][ks * 4 + 1], pk[h][ks * 4 + 2], pk[h][ks * 4 + 3]};
            o[d] = E::mfma(vf, __builtin_bit_cast(s16x8, w), o[d]);
        };
        // Scores of half h of the keys in lk (of the tile at k0), weights of the other half, values (in lv) of
        // half h before that. The order stands as written: fragments are read two products ahead, 5 of the 8
        // pairs of weights lie between the products of scores, 3 and the maximum between those of values.
        auto half_tile = [&](const uint16_t* lk, const uint16_t* lv, int h, uint32_t k0, auto masked, auto has_last) CR_INLINE {
            constexpr int kEarly = 5;
            s16x8 kf[kSteps + 2], vf[kSteps + 2];
            kf[0] = key_frag(lk, h, 0);
            kf[1] = key_frag(lk, h, 1);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int d = 0; d < kSteps; ++d) {
                if (d + 2 < kSteps) kf[d + 2] = key_frag(lk, h, d + 2);
                else if (has_last) vf[d + 2 - kSteps] = val_frag(lv, h, d + 2 - kSteps);
                if (d == 0) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[h][i] = 0.f;
                }
                s[h] = E::mfma(kf[d], qf[d], s[h]);
#pragma unroll
                for (int i = d * kEarly / kSteps; i < (d + 1) * kEarly / kSteps; ++i) weight(h ^ 1, 2 * i);
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int n = 0; n < kSteps; ++n) {
                if (has_last) {
                    if (n + 2 < kSteps) vf[n + 2] = val_frag(lv, h, n + 2);
                    value(vf[n], h, n);
                }
                if (n == 1 && masked) mask(k0, h);
                if (n < kSteps / 2) {
#pragma unroll
                    for (int i = kEarly + n * (8 - kEarly) * 2 / kSteps; i < kEarly + (n + 1) * (8 - kEarly) * 2 / kSteps; ++i) weight(h ^ 1, 2 * i);
                } else {
#pragma unroll
                    for (int i = (n - kSteps / 2) * 16 / kSteps; i < (n - kSteps / 2 + 1) * 16 / kSteps; ++i) maximum(h, 2 * i);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            sum += part[0] + part[1];
            rounded += E::add(pk[h ^ 1][7], part_rounded);
            stay(sum);
            stay(rounded);
            move_maximum();
        };

        ld.store(lds_k(0), lds_v(0));
        ld.load(a, it, key_begin + kKeys);
        ld.pages(a, it, key_begin + 2u * kKeys);
        __syncthreads();
        uint32_t kbuf = 0, vbuf = 0, k0 = key_begin;
        const uint16_t* lv_last = lds_v(0);
        // The next tile into LDS, the one behind it into registers. The keys' buffer was last read before
        // the last barrier, the values' one barrier and a half tile earlier.
        auto stage = [&]() CR_INLINE {
            kbuf ^= 1u;
            vbuf = vbuf + 1u == kValBufs ? 0u : vbuf + 1u;
            if (kValBufs == 2u) __syncthreads();
            if (k0 + kKeys < key_end) ld.store(lds_k(kbuf), lds_v(vbuf));
            ld.load(a, it, k0 + 2u * kKeys);
            ld.pages(a, it, k0 + 3u * kKeys);
            __syncthreads();
        };
        auto tile_of = [&](auto masked, auto has_last) CR_INLINE {
            const uint16_t* lv = lds_v(vbuf);
            half_tile(lds_k(kbuf), lv_last, 1, k0, masked, has_last);
            stage();
            half_tile(lds_k(kbuf), lv, 0, k0 + kKeys, masked, std::true_type{});  // behind the last tile: of what lies there, masked
            lv_last = lv;
            k0 += kKeys;
        };
        if (k0 < w_end) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[0][i] = 0.f;
#pragma unroll
            for (int d = 0; d < kSteps; ++d) s[0] = E::mfma(key_frag(lds_k(0), 0, d), qf[d], s[0]);
            mask(k0, 0);
#pragma unroll
            for (int i = 0; i < 16; i += 2) maximum(0, i);
            move_maximum();
            tile_of(std::true_type{}, std::false_type{});
            if (kPaged) {
                while (k0 < w_end) {
                    while (whole(k0)) tile_of(std::false_type{}, std::true_type{});
                    tile_of(std::true_type{}, std::true_type{});
                }
            } else {
                while (whole(k0)) tile_of(std::false_type{}, std::true_type{});
                while (k0 < w_end) tile_of(std::true_type{}, std::true_type{});
            }
#pragma unroll
            for (int n = 0; n < kSteps; ++n) value(val_frag(lv_last, 1, n), 1, n);
            if (is_late) scale_o(late);
        }
        for (; k0 < key_end; k0 += kKeys) stage();  // keys that only other waves' rows see
        ld.report(a);
    }

    if (__builtin_expect(w_full < key_end && !all_finite<kDim>(o), 0))
        only_seen<E, kDim, kPaged>(a, it, head_kv, row0 + wrow, row0 + rows - 1u, key_begin, 32u, w_end, key_end, w_full, o);
    const float total = both_sum(sum), total_rounded = both_sum(rounded);
    if (wrow + col >= rows) return;
    const bool none = total == 0.f;  // the largest weight of a row that sees a key is 2^kLift or more
    const float inv = none ? 0.f : 1.f / total_rounded;
    const float lse2 = none ? -INFINITY : mc + log2f(total);
    const uint64_t orow = (uint64_t)tok * a.heads_q + head;
    if (a.part_o) {
        const uint64_t at = (uint64_t)(split + (kind == kOwn ? a.slots : 0u)) * a.total_q * a.heads_q + orow;
        if (half == 0) a.part_lse[at] = lse2;
        if (none) return;
#pragma unroll
        for (int d = 0; d < kDim / 32; ++d)
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                *reinterpret_cast<f32x4*>(a.part_o + at * kDim + d * 32 + 2 * i + half * 4u) =
                    f32x4{o[d][i] * inv, o[d][i + 1] * inv, o[d][i + 2] * inv, o[d][i + 3] * inv};
        return;
    }
    if (a.lse && half == 0) a.lse[orow] = lse2 * kLn2;
    uint16_t* op = (uint16_t*)a.out.p + (int64_t)tok * a.out.token_stride + (int64_t)head * a.out.head_stride;
#pragma unroll
    for (int d = 0; d < kDim / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
            *reinterpret_cast<uint2*>(op + d * 32 + 2 * i + half * 4u) =
                uint2{E::pack(o[d][i] * inv, o[d][i + 1] * inv), E::pack(o[d][i + 2] * inv, o[d][i + 3] * inv)};
}

template <typename E, int kDim, bool kPaged>
__global__ __launch_bounds__(8 * kWave, 2) void k_attn_wide(const Attn a, const Part p)
{
    __shared__ __align__(16) uint16_t lds[wide_lds(8, kDim)];
    wide_block<E, kDim, kPaged, 8>(a, p, blockIdx.x, lds);
}

// Few rows: up to 64 at a time. The block's wavefronts take tiles of 32 keys in turn, each with tiles of
// its own in LDS and no barrier, and join their results at the end of a stretch. Where a sequence
// has more than 32 rows, two wavefronts work on each 32 of them and the pairs read the same keys side
// by side, so that memory is read once for 64 rows.
//
// The work of a key head is one line of units: for every sequence of up to two lists (prefixes of groups
// or prompts, own tokens of requests) and every 64 rows of it, kStart units for the start and one
// (more than 32 rows: two) for each tile of keys. A block takes an equal share of the line, whatever lengths fall into it;
// where a share ends inside a sequence's tiles, the parts go to different slots. Lists of one slot are
// not cut: a sequence is worked on where its first unit lies.
//
// Bound by memory where keys are long: 256 requests on 2,000 tokens of their own each, pages of 128, 5.6 TB/s with
// heads of 128 and 5.2 with 64 (4.2 with pages of 32 in token order: pieces of 128 bytes); by the starts where they
// are short: 256 requests and 48 prefixes of about 2,000 tokens, 417 MB in 114 us. Three blocks of a compute unit
// instead of two (heads of 64) were 3 % slower.
constexpr uint32_t kNarrowRows = 64, kNarrowKeys = 32;
constexpr uint32_t kStart = 12; // tiles that a stretch's start and join cost

template <int kDim>
constexpr uint32_t narrow_lds()  // elements per wavefront: tiles, then its sums [32][dim + 4] f32
{
    const uint32_t tiles = key_tile(kNarrowKeys, kDim) + val_tile(kNarrowKeys, kDim), sums = 32u * (kDim + 4u) * 2u;
    return tiles > sums ? tiles : sums;
}

// What a block keeps of 256 sequences at a time, and its wavefronts' maxima and sums.
struct NarrowLds {
    uint32_t at[kThreads];  // units before the sequence, from the first of the 256
    uint32_t sums[16];
    uint32_t tok0[kThreads], nq[kThreads], n[kThreads], key0[kThreads];
    uint32_t disorder[kWaves];
    float row_max[kWaves][32], row_sum[kWaves][32], row_rounded[kWaves][32];
};

template <typename E, int kDim, bool kPaged>
__device__ CR_INLINE void narrow_block(const Attn& a, uint32_t lists, uint32_t block, uint32_t blocks, uint16_t* lds, NarrowLds& sh)
{
    constexpr uint32_t kKeyRun = key_run(kNarrowKeys), kValRun = val_run(kNarrowKeys), kSumRow = kDim + 4u;

    const uint32_t lane = lane_id(), wv = wave_in_block(), half = lane >> 5, col = lane & 31u;
    const uint32_t head_kv = block % a.heads_kv;
    uint16_t* lk = lds + wv * narrow_lds<kDim>();
    uint16_t* lv = lk + key_tile(kNarrowKeys, kDim);
    float* sums = reinterpret_cast<float*>(lk);

    // Sequences 0 .. first_n of the first list, then those of the second.
    const uint32_t first_n = (lists & 1u) ? (kPaged ? a.groups : a.batch) : 0u;
    const uint32_t all_n = first_n + ((lists & 2u) ? a.batch : 0u);
    // Units of sequence x; what does not fit has none. Where offsets of rows or groups are out of order
    // sequences may overlap, and the sum of their units passes what the host allowed for: no list is worked on.
    bool disorder = false;
    auto units = [&](uint32_t x, uint32_t* tok0, uint32_t* nq, uint32_t* n, uint32_t* key0) CR_INLINE -> uint32_t {
        if (x >= all_n) return 0u;
        const bool own = x >= first_n;
        const uint32_t y = own ? x - first_n : x;
        uint32_t r0 = y, r1 = y + 1u;
        if (kPaged && !own) {
            r0 = a.group_off[y];
            r1 = a.group_off[y + 1u];
        }
        const bool in_order = r0 <= r1 && r1 <= a.batch;
        bool ok = in_order;
        if (kPaged && !own && ((y == 0u && r0 != 0u) || (y + 1u == a.groups && r1 != a.batch))) atomicOr(a.err, CR_ERR_SEQ);
        if (kPaged) {
            *n = own ? a.own_len[y] : a.prefix_len[y];
            ok = ok && pages_of(*n, a.pg.log_tokens) <= (own ? a.own_width : a.prefix_width);
        } else {
            const uint32_t k0 = a.k_off[y], k1 = a.k_off[y + 1u];
            *key0 = k0;
            *n = k1 - k0;
            ok = ok && k0 <= k1 && k1 <= a.total_k;
        }
        disorder |= !in_order;
        if (in_order) {  // looked at whatever the keys are: the other sequences' sum depends on it
            const uint32_t t0 = a.q_off[r0], t1 = a.q_off[r1];
            const bool fits = t0 <= t1 && t1 <= a.total_q;
            disorder |= !fits;
            ok = ok && fits;
            *tok0 = t0;
            *nq = t1 - t0;
            if ((r0 == 0u && t0 != 0u) || (r1 == a.batch && t1 != a.total_q)) atomicOr(a.err, CR_ERR_SEQ);
        }
        if (!ok) {
            atomicOr(a.err, CR_ERR_SEQ);
            return 0u;
        }
        const uint32_t rows = *nq * a.group;
        return (rows + kNarrowRows - 1u) / kNarrowRows *
               ((*n + kNarrowKeys - 1u) / kNarrowKeys * (rows > 32u ? 2u : 1u) + kStart);
    };
    uint32_t here = 0;  // units of the 256 sequences in LDS
    auto window = [&](uint32_t x0) CR_INLINE {
        uint32_t tok0 = 0, nq = 0, n = 0, key0 = 0;
        const uint32_t v = units(x0 + threadIdx.x, &tok0, &nq, &n, &key0);
        const uint64_t wrong = ballot(disorder);
        if (lane == 0) sh.disorder[wv] = wrong != 0;
        const uint32_t at = block_exscan_u32(v, sh.sums, &here);
        here = __builtin_amdgcn_readfirstlane(here);
        sh.at[threadIdx.x] = at;
        sh.tok0[threadIdx.x] = tok0;
        sh.nq[threadIdx.x] = nq;
        sh.n[threadIdx.x] = n;
        sh.key0[threadIdx.x] = key0;
        __syncthreads();
    };
    window(0);
    uint32_t all = here;
    for (uint32_t x0 = kThreads; x0 < all_n; x0 += kThreads) {
        uint32_t t0, t1, t2, t3, sum;
        const uint32_t v = units(x0 + threadIdx.x, &t0, &t1, &t2, &t3);
        const uint64_t wrong = ballot(disorder);
        if (lane == 0) sh.disorder[wv] = wrong != 0;
        block_exscan_u32(v, sh.sums, &sum);
        all += __builtin_amdgcn_readfirstlane(sum);
    }
    for (uint32_t w = 0; w < kWaves; ++w)
        if (sh.disorder[w]) return;
    const uint32_t index = block / a.heads_kv, of = blocks / a.heads_kv;
    const uint32_t share = max(all / of + 1u, a.least_share);
    if ((uint64_t)index * share >= all) return;
    uint32_t u = index * share, base = 0, x0 = 0;
    const uint32_t u_end = min(all - u, share) + u;

    // A stretch: up to 64 rows of a sequence over the tiles of it that fall into the block's share.
    struct Stretch {
        Seq it;
        uint32_t row0, rows, key_begin, key_end, slot;
        bool own, pairs, ends, valid;
    };
    auto next = [&]() CR_INLINE {
        Stretch st;
        st.valid = false;
        while (u < u_end && !st.valid) {
            while (u >= base + here) {  // all > u: there is a window behind
                base += here;
                x0 += kThreads;
                window(x0);
            }
            uint32_t i = 0;  // the sequence of unit u
#pragma unroll
            for (uint32_t y = 0; y < kThreads; y += 64u) i += (uint32_t)__popcll(ballot(sh.at[y + lane] <= u - base));
            i = __builtin_amdgcn_readfirstlane(i - 1u);
            const uint32_t x = x0 + i;
            Seq& it = st.it;
            st.own = x >= first_n;
            it.tok0 = __builtin_amdgcn_readfirstlane(sh.tok0[i]);
            it.nq = __builtin_amdgcn_readfirstlane(sh.nq[i]);
            it.n = __builtin_amdgcn_readfirstlane(sh.n[i]);
            it.least = 0;
            it.gap_end = 0;
            it.len0 = 0;
            if (kPaged) {
                it.causal = st.own;
                if (!st.own) it.len0 = it.gap_end = it.n;
                it.table0 = a.prefix_table + (uint64_t)x * a.prefix_width;
                it.table1 = a.own_table + (uint64_t)(x - first_n) * a.own_width;
            } else {
                it.causal = a.causal;
                it.key0 = __builtin_amdgcn_readfirstlane(sh.key0[i]);
            }
            it.first_lim = it.causal ? (int32_t)it.n - (int32_t)it.nq + 1 : (int32_t)it.n;
            const uint32_t tiles = (it.n + kNarrowKeys - 1u) / kNarrowKeys;
            st.pairs = it.nq * a.group > 32u;
            const uint32_t per_tile = st.pairs ? 2u : 1u;  // units
            const uint32_t from = base + __builtin_amdgcn_readfirstlane(sh.at[i]), step = tiles * per_tile + kStart;
            const uint32_t row_tile = __builtin_amdgcn_readfirstlane((u - from) / step);
            const uint32_t first = from + row_tile * step, keys = first + kStart, last = first + step;  // the rows' units
            uint32_t t0 = 0, t1 = tiles;
            st.slot = 0;
            st.ends = true;
            st.valid = u == first;
            if ((st.own ? a.own_slots : a.slots) > 1u && tiles != 0u) {
                // every block whose share has a unit of the keys has a slot, though it may come without a tile
                st.valid = u_end > keys;
                t0 = u > keys ? (u - keys) / per_tile : 0u;
                t1 = u_end < last ? (st.valid ? (u_end - keys) / per_tile : 0u) : tiles;
                st.slot = index - __builtin_amdgcn_readfirstlane(keys / share);
                st.ends = last <= u_end;
            }
            u = last;
            st.row0 = row_tile * kNarrowRows;
            st.rows = min(kNarrowRows, it.nq * a.group - st.row0);
            st.key_begin = t0 * kNarrowKeys;
            st.key_end = min(row_limit(a, it, st.row0 + st.rows - 1u), t1 * kNarrowKeys);
        }
        return st;
    };
    for (Stretch st = next(); st.valid; st = next()) {
        const Seq& it = st.it;
        const bool own = st.own, pairs = st.pairs;
        const uint32_t slots = own ? a.own_slots : a.slots, row0 = st.row0, rows = st.rows, key_end = st.key_end;
        const uint32_t wave_row = pairs ? (wv & 1u) * 32u : 0u;      // of the 64
        const uint32_t full = min(row_limit(a, it, row0 + min(wave_row, rows - 1u)), key_end);  // keys that every row of the wave sees
        const uint32_t key_step = (pairs ? 2u : kWaves) * kNarrowKeys;
        const uint32_t m = row0 + min(wave_row + col, rows - 1u);
        const uint32_t tok = it.tok0 + m / a.group, head = head_kv * a.group + m % a.group;
        const int32_t lim = (int32_t)min(row_limit(a, it, m), key_end);

        f32x16 o[kDim / 32];
#pragma unroll
        for (int d = 0; d < kDim / 32; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
        float mc = kNoMax, sum = 0.f, rounded = 0.f;
        const uint32_t first_key = st.key_begin + (pairs ? wv >> 1 : wv) * kNarrowKeys;
        uint32_t k0 = first_key;
        if (k0 < key_end && wave_row < rows) {
            Loader<kDim, kPaged, kNarrowKeys, kWave> ld;
            ld.bad = 0;
            ld.init(a, it, head_kv, key_end, lane);
            ld.pages(a, it, k0);
            ld.load(a, it, k0);
            ld.pages(a, it, k0 + key_step);
            s16x8 qf[kDim / 16];
            const uint16_t* qp = (const uint16_t*)a.q.p + (int64_t)tok * a.q.token_stride + (int64_t)head * a.q.head_stride;
#pragma unroll
            for (int s = 0; s < kDim / 16; ++s) qf[s] = *reinterpret_cast<const s16x8*>(qp + s * 16 + half * 8u);
            const uint32_t k_lane = half * kKeyRun + col * 8u;
            const uint32_t v_lane = (half * 4u + (lane & 15u) / 4u) * 32u + ((lane >> 4) & 1u) * 16u + (lane & 3u) * 4u;
            for (; k0 < key_end; k0 += key_step) {
                ld.store(lk, lv);
                wave_lds_fence();
                ld.load(a, it, k0 + key_step);
                ld.pages(a, it, k0 + 2u * key_step);
                f32x16 s;
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
                for (int d = 0; d < kDim / 16; ++d)
                    s = E::mfma(*reinterpret_cast<const s16x8*>(lk + k_lane + d * 2u * kKeyRun), qf[d], s);
                if (k0 + kNarrowKeys > full) {
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if ((int32_t)(k0 + 8u * (i / 4) + 4u * half + (i & 3)) >= lim) s[i] = -INFINITY;
                }
                float top = __builtin_elementwise_maximum(s[0], s[1]);
#pragma unroll
                for (int i = 2; i < 16; i += 2)
                    top = __builtin_elementwise_maximum(__builtin_elementwise_maximum(top, s[i]), s[i + 1]);
                top = both_max(top) * a.c;
                if (ballot(top > mc + (kSlack + E::kLift))) {
                    const float up = fmaxf(mc, top - E::kLift), f = __builtin_amdgcn_exp2f(mc - up);
                    mc = up;
                    sum *= f;
                    rounded *= f;
#pragma unroll
                    for (int d = 0; d < kDim / 32; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[d][i] *= f;
                }
                uint32_t pk[8];
                float t[4], part_rounded = 0.f;
#pragma unroll
                for (int i = 0; i < 16; i += 2) {
                    const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], a.c, -mc));
                    const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i + 1], a.c, -mc));
                    t[i & 3] = i < 4 ? x : t[i & 3] + x;
                    t[(i & 3) + 1] = i < 4 ? y : t[(i & 3) + 1] + y;
                    pk[i / 2] = E::pack(x, y);
                    part_rounded = E::add(pk[i / 2], part_rounded);
                }
                sum += (t[0] + t[1]) + (t[2] + t[3]);
                rounded += part_rounded;
#pragma unroll
                for (int ks = 0; ks < 2; ++ks) {
                    const u32x4 w = {pk[ks * 4], pk[ks * 4 + 1], pk[ks * 4 + 2], pk[ks * 4 + 3]};
#pragma unroll
                    for (int d = 0; d < kDim / 32; ++d) {
                        s16x4 vf[2];
#pragma unroll
                        for (int y = 0; y < 2; ++y) vf[y] = read_tr(lv + v_lane + d * kValRun + (ks * 16u + y * 8u) * 32u);
                        o[d] = E::mfma(__builtin_shufflevector(vf[0], vf[1], 0, 1, 2, 3, 4, 5, 6, 7), __builtin_bit_cast(s16x8, w), o[d]);
                    }
                }
                wave_lds_fence();
            }
            ld.report(a);
        }
        if (__builtin_expect(full < key_end && !all_finite<kDim>(o), 0))
            only_seen<E, kDim, kPaged>(a, it, head_kv, row0 + wave_row, row0 + rows - 1u, first_key, key_step, key_end, key_end, full, o);
        sum = both_sum(sum);
        rounded = both_sum(rounded);
        if (half == 0) {
            sh.row_max[wv][col] = mc;
            sh.row_sum[wv][col] = sum;
            sh.row_rounded[wv][col] = rounded;
        }
#pragma unroll
        for (int d = 0; d < kDim / 32; ++d)
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                *reinterpret_cast<f32x4*>(sums + col * kSumRow + d * 32 + 2 * i + half * 4u) = f32x4{o[d][i], o[d][i + 1], o[d][i + 2], o[d][i + 3]};
        __syncthreads();
        // 4 elements of a row per thread
        for (uint32_t y = threadIdx.x; y < rows * (kDim / 4u); y += kThreads) {
            const uint32_t row = y / (kDim / 4u), r = row & 31u, e = y % (kDim / 4u) * 4u, mm = row0 + row;
            const uint32_t w0 = row >> 5, w_step = pairs ? 2u : 1u;  // the wavefronts that worked on the row
            float mx = sh.row_max[w0][r], total = 0.f, total_rounded = 0.f;
            for (uint32_t w = w0 + w_step; w < kWaves; w += w_step) mx = fmaxf(mx, sh.row_max[w][r]);
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
            for (uint32_t w = w0; w < kWaves; w += w_step) {
                const float f = __builtin_amdgcn_exp2f(sh.row_max[w][r] - mx);
                const f32x4 v = *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(lds + w * narrow_lds<kDim>()) + r * kSumRow + e);
                total = __builtin_fmaf(f, sh.row_sum[w][r], total);
                total_rounded = __builtin_fmaf(f, sh.row_rounded[w][r], total_rounded);
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[i] = __builtin_fmaf(f, v[i], acc[i]);
            }
            const bool none = total == 0.f;
            const float inv = none ? 0.f : 1.f / total_rounded, lse2 = none ? -INFINITY : mx + log2f(total);
            const uint32_t ot = it.tok0 + mm / a.group, oh = head_kv * a.group + mm % a.group;
            const uint64_t orow = (uint64_t)ot * a.heads_q + oh;
            if (a.part_o) {
                const uint64_t at = (uint64_t)(st.slot + (own ? a.slots : 0u)) * a.total_q * a.heads_q + orow;
                if (e == 0) {
                    a.part_lse[at] = lse2;
                    if (st.ends)  // slots that are left
                        for (uint32_t z = st.slot + 1u; z < slots; ++z) a.part_lse[at + (uint64_t)(z - st.slot) * a.total_q * a.heads_q] = -INFINITY;
                }
                *reinterpret_cast<f32x4*>(a.part_o + at * kDim + e) = acc * inv;
            } else {
                if (a.lse && e == 0) a.lse[orow] = lse2 * kLn2;
                *reinterpret_cast<uint2*>((uint16_t*)a.out.p + (int64_t)ot * a.out.token_stride + (int64_t)oh * a.out.head_stride + e) =
                    uint2{E::pack(acc[0] * inv, acc[1] * inv), E::pack(acc[2] * inv, acc[3] * inv)};
            }
        }
        __syncthreads();
    }
}

// One launch of what is not wide: tiles of 128 rows (up to two parts) and the narrow lists' blocks,
// so that neither waits for the other's last.
constexpr uint32_t kMixedPerCu = 2;  // blocks that share a compute unit

template <typename E, int kDim, bool kPaged>
__global__ __launch_bounds__(kThreads, kMixedPerCu) void k_attn_mixed(const Attn a, const Part p0, const Part p1, uint32_t lists)
{
    constexpr uint32_t kWide = wide_lds(kWaves, kDim), kNarrow = kWaves * narrow_lds<kDim>();
    __shared__ __align__(16) uint16_t lds[kWide > kNarrow ? kWide : kNarrow];
    __shared__ NarrowLds sh;
    const uint32_t wides = p0.blocks + p1.blocks;
    if (blockIdx.x < wides) {
        const bool second = blockIdx.x >= p0.blocks;
        wide_block<E, kDim, kPaged, kWaves>(a, second ? p1 : p0, second ? blockIdx.x - p0.blocks : blockIdx.x, lds);
    } else {
        narrow_block<E, kDim, kPaged>(a, lists, blockIdx.x - wides, gridDim.x - wides, lds, sh);
    }
}

// Joins the partial results of a token's rows: 4 elements of a row per thread, kPar threads share the
// slots of a row's elements (eight where there are more than eight slots). Bound by memory and the launch: two
// slots of 3 tokens 4 us, 11 slots of 128 tokens' 64 heads (46 MB) 16.
template <typename E, int kDim, uint32_t kPar>
__global__ __launch_bounds__(kThreads) void k_attn_join(const Attn a)
{
    constexpr uint32_t kPer = kDim / 4, kGroup4 = kThreads / kPar;
    __shared__ float sh[kPar > 1 ? kPar : 1][kPar > 1 ? kGroup4 : 1][6];
    const uint32_t tok = blockIdx.x, slots = a.slots + a.own_slots;
    const uint32_t x = blockIdx.y * kGroup4 + threadIdx.x % kGroup4, part = threadIdx.x / kGroup4;
    const uint32_t head = x / kPer, e = x % kPer * 4u;
    const bool ok = head < a.heads_q;
    const uint64_t rows = (uint64_t)a.total_q * a.heads_q, row = (uint64_t)tok * a.heads_q + (ok ? head : 0u);
    float mx = -INFINITY, sum = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (uint32_t i = part; i < slots; i += kPar) {
        const uint64_t at = i * rows + row;
        const float l = a.part_lse[at];
        if (l == -INFINITY) continue;  // its elements may be unwritten
        const f32x4 v = *reinterpret_cast<const f32x4*>(a.part_o + at * kDim + e);
        const float up = l > mx || l != l ? l : mx;
        const float f = __builtin_amdgcn_exp2f(mx - up), w = __builtin_amdgcn_exp2f(l - up);
        mx = up;
        sum = __builtin_fmaf(sum, f, w);
#pragma unroll
        for (int y = 0; y < 4; ++y) acc[y] = __builtin_fmaf(acc[y], f, w * v[y]);
    }
    if (kPar > 1) {
        float* mine = sh[part][threadIdx.x % kGroup4];
        mine[0] = mx;
        mine[1] = sum;
#pragma unroll
        for (int y = 0; y < 4; ++y) mine[2 + y] = acc[y];
        __syncthreads();
        if (part != 0) return;
        for (uint32_t p = 1; p < kPar; ++p) {
            const float* his = sh[p][threadIdx.x % kGroup4];
            const float l = his[0];
            if (l == -INFINITY) continue;
            const float up = l > mx || l != l ? l : mx;
            const float f = __builtin_amdgcn_exp2f(mx - up), w = __builtin_amdgcn_exp2f(l - up);
            mx = up;
            sum = __builtin_fmaf(sum, f, w * his[1]);
#pragma unroll
            for (int y = 0; y < 4; ++y) acc[y] = __builtin_fmaf(acc[y], f, w * his[2 + y]);
        }
    }
    if (!ok) return;
    const bool none = mx == -INFINITY;
    const float inv = none ? 0.f : 1.f / sum;
    uint16_t* op = (uint16_t*)a.out.p + (int64_t)tok * a.out.token_stride + (int64_t)head * a.out.head_stride + e;
    *reinterpret_cast<uint2*>(op) = uint2{E::pack(acc[0] * inv, acc[1] * inv), E::pack(acc[2] * inv, acc[3] * inv)};
    if (a.lse && e == 0) a.lse[row] = none ? -INFINITY : (mx + log2f(sum)) * kLn2;
}

// How a call is cut: the wide kernels' launches, the lists of the narrow one, chunks and slots.
struct Wide {
    uint32_t kind, rows;  // rows per block
};
struct Shape {
    Wide wide[2];
    uint32_t wides, lists;  // lists of the narrow launch: 1 the first kind's, 2 own tokens
    uint32_t chunk, slots, own_chunk, own_slots;
    uint32_t least;                                        // share of a narrow block, in tiles
    uint64_t blocks;                                       // of the narrow launch, per key head
    bool join;
};

constexpr uint32_t kFewRows = 64;        // mean rows of a sequence up to which the narrow kernel takes it
constexpr uint32_t kWholeRows = 128;     // mean rows of a request from which its prefix is read again, not joined
constexpr uint32_t kSplitKeys = 384;     // keys a workgroup should have at least where a call is split
constexpr uint32_t kSplitMax = 32;
constexpr uint32_t kLongKeys = 1024;     // mean keys from which blocks of 256 rows pay
constexpr uint32_t kNarrowParts = 63;    // shares a sequence's keys may fall into
constexpr uint32_t kShareLeast = 8;      // tiles a narrow block should have

inline uint32_t up_to(uint64_t x, uint32_t m) { return (uint32_t)((x + m - 1u) / m * m); }

// Tiles that a call's rows make, about: whole ones, and one for each sequence's rest.
inline uint64_t tiles_of(uint64_t rows, uint32_t per, uint32_t seqs)
{
    return seqs == 1u ? (rows + per - 1u) / per : rows / per + (rows < (uint64_t)seqs * per ? seqs : seqs / 2u);
}

// Rows per block, and the chunks of sequences of about `keys` keys. Blocks of 256 rows have a compute
// unit each, two of 128 share one. More chunks fill the last round of blocks better and cost a start each
// (about four tiles) and a join (a row's 8 dim bytes written and read again, about as long as 500
// bytes take a tile's time per block); the number with the least estimated time is taken.
inline Wide wide_shape(uint32_t kind, uint64_t rows, uint32_t seqs, uint32_t heads_kv, uint64_t keys, uint32_t dim, uint32_t* chunk,
                       uint32_t* slots)
{
    uint64_t most = keys / kSplitKeys;
    most = most < 1 ? 1 : (most < kSplitMax ? most : kSplitMax);
    Wide w{kind, 128u};
    if (keys >= kLongKeys && rows >= 192ull * seqs && tiles_of(rows, 256, seqs) * heads_kv * most >= 256u) w.rows = 256u;
    const uint64_t blocks = tiles_of(rows, w.rows, seqs) * heads_kv, room = w.rows == 256u ? 256u : 512u;
    const double tile_us = dim == 128 ? 2.0 : 1.2;
    double least = 0;
    for (uint64_t s = 1; s <= most; ++s) {
        const double rounds = (double)((blocks * s + room - 1u) / room), tiles = (double)((keys + kKeys * s - 1u) / (kKeys * s));
        const double us = rounds * (tiles + 4.0) * tile_us + (s > 1 ? 4.0 + (double)(s * rows * heads_kv * dim) * 8.0 / 4.0e6 : 0.0);
        if (s == 1 || us < least) {
            least = us;
            *slots = (uint32_t)s;
        }
    }
    *chunk = up_to(keys / *slots + 1u, kChunkUnit);
    return w;
}

// Slots of a narrow list of sequences of up to `keys` keys, where a block's share of the work is about
// `share` tiles; *least: the share from which no sequence passes its slots.
inline uint32_t narrow_slots(uint64_t keys, uint64_t share, uint32_t* least)
{
    const uint64_t tiles = (keys + kNarrowKeys - 1u) / kNarrowKeys * 2u;  // units, where there are more than 32 rows
    if (tiles * 2u <= share) return 1u;  // cutting would not level the shares by much
    uint64_t parts = (tiles + share - 1u) / share;
    parts = parts < kNarrowParts ? parts : kNarrowParts;
    const uint32_t need = (uint32_t)((tiles + parts - 1u) / parts);
    *least = need > *least ? need : *least;
    return (uint32_t)parts + 1u;
}

// Units of a list per key head, its sequences half as long as they may be.
inline uint64_t narrow_units(uint64_t rows, uint32_t seqs, uint64_t keys)
{
    return tiles_of(rows, kNarrowRows, seqs) * (keys / (2u * kNarrowKeys) * (rows > 32ull * seqs ? 2u : 1u) + kStart);
}

// Most units that a list can have per key head.
inline uint64_t narrow_most(uint64_t rows, uint32_t seqs, uint64_t keys)
{
    return (rows / kNarrowRows + seqs) * (keys / (kNarrowKeys / 2u) + 2u + kStart);
}

// Whether the list's units stay in 32 bits whatever the lengths.
inline bool narrow_fits(uint64_t rows, uint32_t seqs, uint64_t keys)
{
    return narrow_most(rows, seqs, keys) < (1ull << 31);
}

// Whether every sequence can have a block to itself: shares of kStart units hold one sequence's first
// unit at most, so with whole sequences (one slot) and as many blocks none works on two. For short ones:
// a block's wavefronts take four tiles at a time.
constexpr uint32_t kAloneKeys = 512;
inline bool narrow_alone(uint64_t most, uint64_t keys, uint64_t blocks) { return keys <= kAloneKeys && most <= blocks * kStart; }

// Blocks per key head: what the wide parts of the launch leave of the GPU, at least half of it.
inline uint64_t narrow_blocks(uint32_t heads_kv, uint64_t wides)
{
    const uint64_t room = kMixedPerCu * (uint64_t)device_cus();
    return ((wides < room / 2u ? room - wides : room / 2u) + heads_kv - 1u) / heads_kv;
}

inline bool good_scale(float s) { return s > 0.f && s <= 3.0e38f; }

inline bool good_heads(uint32_t hq, uint32_t hkv) { return hkv >= 1 && hq >= hkv && hq <= CR_MAX_HEADS && hq % hkv == 0; }

inline bool good_prompt_sizes(const cr_attn_prompt_args* p)
{
    return p && p->dtype <= CR_F16 && good_heads(p->heads_q, p->heads_kv) && (p->dim == 64 || p->dim == 128) &&
           p->causal <= 1 && good_scale(p->scale) && (uint64_t)p->total_q * p->heads_q < (1ull << 31) &&
           p->total_k < CR_MAX_KEYS && p->batch <= (1u << 24) && (p->batch > 0 || p->total_q == 0);
}

inline bool good_shared_sizes(const cr_kv_cache* c, const cr_attn_shared_args* p)
{
    return good_cache_sizes(c) && p && good_heads(p->heads_q, c->heads) && p->layer < c->layers && good_scale(p->scale) &&
           (uint64_t)p->total_q * p->heads_q < (1ull << 31) && p->batch <= (1u << 24) && p->groups <= p->batch &&
           (p->total_q == 0 || p->groups > 0) &&
           ((uint64_t)p->prefix_width + p->own_width) * c->page_tokens < CR_MAX_KEYS;
}

// Lengths are on the device: the mean stands for them, and a sequence's chunks grow where it is longer.
inline Shape prompt_shape(const cr_attn_prompt_args* p)
{
    Shape s{};
    const uint64_t rows = (uint64_t)p->total_q * (p->heads_q / p->heads_kv), keys = p->total_k / p->batch;
    if (rows <= (uint64_t)kFewRows * p->batch && narrow_fits(rows, p->batch, p->total_k)) {
        s.lists = 1;
        s.blocks = narrow_blocks(p->heads_kv, 0);
        s.least = kShareLeast;
        const uint64_t units = narrow_units(rows, p->batch, 2u * keys), equal = units / s.blocks;
        s.slots = narrow_slots(p->batch > 1 ? 2u * keys : keys, equal > kShareLeast ? equal : kShareLeast, &s.least);
        if (s.slots > 1 && p->batch > 1) {  // a sequence may be longer than twice the mean
            const uint32_t need = (2u * (p->total_k / kNarrowKeys + 1u) + s.slots - 2u) / (s.slots - 1u);
            s.least = need > s.least ? need : s.least;
        }
        const uint64_t most = (2u * units + s.least - 1u) / s.least;  // more blocks would have no share
        const uint64_t all = narrow_most(rows, p->batch, p->total_k);
        if (narrow_alone(all, p->total_k, s.blocks)) {
            s.slots = s.least = 1u;
            s.blocks = (all + kStart - 1u) / kStart;
        } else if (most < s.blocks) {
            s.blocks = most ? most : 1u;
        }
    } else {
        s.wide[s.wides++] = wide_shape(kPrompt, rows, p->batch, p->heads_kv, keys, p->dim, &s.chunk, &s.slots);
    }
    s.join = s.slots > 1;
    return s;
}

// Here the tables' widths stand for the lengths.
inline Shape shared_shape(const cr_kv_cache* c, const cr_attn_shared_args* p)
{
    Shape s{};
    const uint64_t rows = (uint64_t)p->total_q * (p->heads_q / c->heads);
    const uint64_t prefix = (uint64_t)p->prefix_width * c->page_tokens, own = (uint64_t)p->own_width * c->page_tokens;
    if (rows >= (uint64_t)kWholeRows * p->batch) {
        s.wide[s.wides++] = wide_shape(kWhole, rows, p->batch, c->heads, prefix + own, c->dim, &s.chunk, &s.slots);
        s.join = s.slots > 1;
        return s;
    }
    s.join = true;
    uint64_t units = 0, wides = 0;
    if (rows <= (uint64_t)kFewRows * p->groups && narrow_fits(rows, p->groups, prefix)) {
        s.lists |= 1u;
        units += narrow_units(rows, p->groups, prefix);
    } else {
        const Wide w = wide_shape(kGroup, rows, p->groups, c->heads, prefix, c->dim, &s.chunk, &s.slots);
        if (w.rows == 128u) wides += tiles_of(rows, w.rows, p->groups) * s.slots * c->heads;
        s.wide[s.wides++] = w;
    }
    if (rows <= (uint64_t)kFewRows * p->batch && narrow_fits(rows, p->batch, own)) {
        s.lists |= 2u;
        units += narrow_units(rows, p->batch, own);
    } else {
        s.wide[s.wides++] = wide_shape(kOwn, rows, p->batch, c->heads, own, c->dim, &s.own_chunk, &s.own_slots);
    }
    if (s.lists) {
        s.blocks = narrow_blocks(c->heads, wides);
        s.least = kShareLeast;
        const uint64_t equal = units / s.blocks, share = equal > kShareLeast ? equal : kShareLeast;
        if (s.lists & 1u) s.slots = narrow_slots(prefix, share, &s.least);
        if (s.lists & 2u) s.own_slots = narrow_slots(own, share, &s.least);
        const uint64_t most = (2u * units + s.least - 1u) / s.least;  // more blocks would have no share
        const uint64_t all = ((s.lists & 1u) ? narrow_most(rows, p->groups, prefix) : 0u) + ((s.lists & 2u) ? narrow_most(rows, p->batch, own) : 0u);
        if (narrow_alone(all, (s.lists & 1u) && prefix > own ? prefix : own, s.blocks)) {
            if (s.lists & 1u) s.slots = 1u;
            if (s.lists & 2u) s.own_slots = 1u;
            s.least = 1u;
            s.blocks = (all + kStart - 1u) / kStart;
        } else if (most < s.blocks) {
            s.blocks = most ? most : 1u;
        }
    }
    return s;
}

inline size_t part_bytes(const Shape& s, uint64_t rows, uint32_t dim)
{
    return s.join ? ((uint64_t)s.slots + s.own_slots) * rows * (dim + 1u) * sizeof(float) : 0;
}

template <typename E, int kDim, bool kPaged>
void launch(const Attn& a, const Shape& s, hipStream_t st)
{
    const uint64_t rows = (uint64_t)a.total_q * a.group;
    Part few[2] = {};
    uint32_t fews = 0;
    for (uint32_t i = 0; i < s.wides; ++i) {
        const Wide& w = s.wide[i];
        const uint32_t seqs = w.kind == kGroup ? a.groups : a.batch;
        Part p{w.kind, (uint32_t)(rows / w.rows) + seqs, 0, 0};
        p.blocks = p.tiles * (w.kind == kOwn ? a.own_slots : a.slots) * a.heads_kv;
        p.sorted = seqs > 1u && seqs <= kSortSeqs && p.blocks > (w.rows == 256u ? 1u : kMixedPerCu) * (uint32_t)device_cus();
        if (w.rows == 256u) hipLaunchKernelGGL((k_attn_wide<E, kDim, kPaged>), dim3(p.blocks), dim3(8 * kWave), 0, st, a, p);
        else few[fews++] = p;
    }
    uint32_t blocks = few[0].blocks + few[1].blocks;
    if (s.lists) blocks += (uint32_t)s.blocks * a.heads_kv;
    if (blocks) hipLaunchKernelGGL((k_attn_mixed<E, kDim, kPaged>), dim3(blocks), dim3(kThreads), 0, st, a, few[0], few[1], s.lists);
    if (s.join) {
        constexpr uint32_t kPer = kDim / 4;
        if (s.slots + s.own_slots > 8u)
            hipLaunchKernelGGL((k_attn_join<E, kDim, 8>), dim3(a.total_q, (a.heads_q * kPer + 31u) / 32u), dim3(kThreads), 0, st, a);
        else
            hipLaunchKernelGGL((k_attn_join<E, kDim, 1>), dim3(a.total_q, (a.heads_q * kPer + 255u) / 256u), dim3(kThreads), 0, st, a);
    }
}

template <bool kPaged>
cr_status dispatch(Attn& a, const Shape& s, void* ws, uint32_t dtype, uint32_t dim, void* stream)
{
    const hipStream_t st = as_stream(stream);
    const uint64_t rows = (uint64_t)a.total_q * a.group;
    // Threads of a launch: two parts' tiles of 128 rows, or one's and the few-row blocks, stay below 2^32 with these.
    for (uint32_t i = 0; i < s.wides; ++i)
        if ((rows / s.wide[i].rows + a.batch) * (s.wide[i].kind == kOwn ? s.own_slots : s.slots) * a.heads_kv >= (1ull << 32) / (8u * kWave))
            return CR_EINVAL;
    if (s.join && a.total_q >= (1ull << 32) / kThreads) return CR_EINVAL;  // a block of the join per token
    a.chunk = s.chunk;
    a.slots = s.slots;
    a.own_chunk = s.own_chunk;
    a.own_slots = s.own_slots;
    a.least_share = s.least;
    if (s.join) {
        a.part_o = (float*)ws;
        a.part_lse = a.part_o + ((uint64_t)s.slots + s.own_slots) * a.total_q * a.heads_q * dim;
    }
    (void)hipGetLastError();
    if (dtype == CR_BF16 && dim == 128) launch<Bf16, 128, kPaged>(a, s, st);
    else if (dtype == CR_BF16) launch<Bf16, 64, kPaged>(a, s, st);
    else if (dim == 128) launch<F16, 128, kPaged>(a, s, st);
    else launch<F16, 64, kPaged>(a, s, st);
    return hipGetLastError() == hipSuccess ? CR_OK : CR_EHIP;
}

}  // namespace
}  // namespace cr

extern "C" size_t cr_attn_prompt_workspace_bytes(const cr_attn_prompt_args* p)
{
    using namespace cr;
    if (!good_prompt_sizes(p) || p->total_q == 0) return 0;
    return part_bytes(prompt_shape(p), (uint64_t)p->total_q * p->heads_q, p->dim);
}

extern "C" cr_status cr_attn_prompt(const cr_attn_prompt_args* p, void* ws, size_t ws_bytes, uint32_t* err, void* stream)
{
    using namespace cr;
    if (!good_prompt_sizes(p) || !err) return CR_EINVAL;
    if (p->total_q == 0) return CR_OK;
    if (!good_rows(p->q) || !good_rows(p->out) || !p->q_off || !p->k_off ||
        (p->total_k > 0 && (!good_rows(p->k) || !good_rows(p->v))) || (p->lse && !aligned4(p->lse)))
        return CR_EINVAL;
    const Shape s = prompt_shape(p);
    const size_t need = part_bytes(s, (uint64_t)p->total_q * p->heads_q, p->dim);
    if (need && (!ws || !aligned16(ws))) return CR_EINVAL;
    if (ws_bytes < need) return CR_ESIZE;
    Attn a{};
    a.q = p->q;
    a.k = p->k;
    a.v = p->v;
    a.out = p->out;
    a.lse = p->lse;
    a.q_off = p->q_off;
    a.k_off = p->k_off;
    a.heads_q = p->heads_q;
    a.heads_kv = p->heads_kv;
    a.group = p->heads_q / p->heads_kv;
    a.batch = p->batch;
    a.total_q = p->total_q;
    a.total_k = p->total_k;
    a.causal = p->causal;
    a.c = p->scale * kLog2e;
    a.err = err;
    return dispatch<false>(a, s, ws, p->dtype, p->dim, stream);
}

extern "C" size_t cr_attn_shared_workspace_bytes(const cr_kv_cache* c, const cr_attn_shared_args* p)
{
    using namespace cr;
    if (!good_shared_sizes(c, p) || p->total_q == 0) return 0;
    return part_bytes(shared_shape(c, p), (uint64_t)p->total_q * p->heads_q, c->dim);
}

extern "C" cr_status cr_attn_shared(const cr_kv_cache* c, const cr_attn_shared_args* p, void* ws, size_t ws_bytes,
                                    uint32_t* err, void* stream)
{
    using namespace cr;
    if (!good_cache(c) || !good_shared_sizes(c, p) || !err) return CR_EINVAL;
    if (p->total_q == 0) return CR_OK;
    if (!good_rows(p->q) || !good_rows(p->out) || !p->q_off || !p->group_off || !p->prefix_len || !p->own_len ||
        (p->prefix_width && !p->prefix_table) || (p->own_width && !p->own_table) || (p->lse && !aligned4(p->lse)))
        return CR_EINVAL;
    const Shape s = shared_shape(c, p);
    const size_t need = part_bytes(s, (uint64_t)p->total_q * p->heads_q, c->dim);
    if (need && (!ws || !aligned16(ws))) return CR_EINVAL;
    if (ws_bytes < need) return CR_ESIZE;
    Attn a{};
    a.q = p->q;
    a.out = p->out;
    a.lse = p->lse;
    a.pg = kv_pages(c);
    a.pg.k += (int64_t)p->layer * c->layer_stride;
    a.pg.v += (int64_t)p->layer * c->layer_stride;
    a.q_off = p->q_off;
    a.group_off = p->group_off;
    a.prefix_table = p->prefix_table;
    a.prefix_len = p->prefix_len;
    a.own_table = p->own_table;
    a.own_len = p->own_len;
    a.prefix_width = p->prefix_width;
    a.own_width = p->own_width;
    a.heads_q = p->heads_q;
    a.heads_kv = c->heads;
    a.group = p->heads_q / c->heads;
    a.batch = p->batch;
    a.groups = p->groups;
    a.total_q = p->total_q;
    a.c = p->scale * kLog2e;
    a.err = err;
    return dispatch<true>(a, s, ws, c->dtype, c->dim, stream);
}
