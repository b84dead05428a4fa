// Attention of a destination: whole prompts (packed, causal, grouped heads) and requests that share a
// cached prefix in pages.
//
// Mathematics: scores s_j = scale q.k_j, running maximum m and sum l of exp(s_j - m) over the keys
// in one pass, o = sum_j exp(s_j - m) v_j / l, lse = m + ln l. Results over disjoint sets of keys
// are joined by lse = ln sum exp(lse_p), o = sum exp(lse_p - lse) o_p. Exponentials are taken base
// 2 with log2(e) folded into the scale.
#include "cr_kv.h"

#include <type_traits>

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
    static __device__ __forceinline__ f32x16 mfma(s16x8 a, s16x8 b, f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint32_t pack(float x, float y)
    {
        return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x, y}), bf16x2));
    }
};

struct F16 {
    static __device__ __forceinline__ f32x16 mfma(s16x8 a, s16x8 b, f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint32_t pack(float x, float y)
    {
        return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x, y}), f16x2));
    }
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
    uint32_t rows;                   // query rows (token, head of the group) per block
    uint32_t tiles, splits;          // prompt: over sequences; shared: over groups
    uint32_t own_tiles, own_splits;  // shared: over requests
    float* part_o;         // f32 [splits + own_splits][total_q * heads_q][dim], NULL: results are final
    float* part_lse;       // f32 [splits + own_splits][total_q * heads_q], base 2
    uint32_t* err;
};

// What a block works on: rows row0 .. row0 + rows of a sequence's (token, head of the group) rows,
// over keys begin .. end. Row m is query token tok0 + m / group and sees keys below
// first_lim + m / group (causal) or all n.
struct Item {
    uint32_t row0, rows, tok0, begin, end, slot;
    int32_t first_lim;
    uint32_t causal;
    uint32_t key0;                // prompt: first key row
    const uint32_t* table;        // shared: the sequence's pages
};

__device__ __forceinline__ bool bad_seq(const Attn& a, uint32_t bit)
{
    if (threadIdx.x == 0) atomicOr(a.err, bit);
    return false;
}

// Tile t of sequence x starts at floor(first row / rows per block) + x: steps of at least
// ceil(rows / rows per block), so that the tiles of all sequences fit into floor(all rows / rows per block) +
// sequences without a pass that counts them; some are empty.
template <bool kPaged>
__device__ __forceinline__ bool find_item(const Attn& a, uint32_t id, Item* it)
{
    uint32_t tile, split, splits, x, t0, t1, n;
    if (kPaged && id < a.tiles * a.splits) {
        split = id % a.splits;
        tile = id / a.splits;
        splits = a.splits;
        it->slot = split;
        auto start = [&](uint32_t g) { return a.q_off[min(a.group_off[g], a.batch)] * a.group / a.rows + g; };
        x = wave_find(a.groups, tile, start);
        const uint32_t r0 = a.group_off[x], r1 = a.group_off[x + 1];
        if (r0 > r1 || r1 > a.batch) return bad_seq(a, CR_ERR_SEQ);
        t0 = a.q_off[r0];
        t1 = a.q_off[r1];
        n = a.prefix_len[x];
        if (pages_of(n, a.pg.log_tokens) > a.prefix_width) return bad_seq(a, CR_ERR_SEQ);
        it->table = a.prefix_table + (uint64_t)x * a.prefix_width;
        it->causal = 0;
        tile -= min(start(x), tile);
    } else {
        if (kPaged) {
            id -= a.tiles * a.splits;
            splits = a.own_splits;
            tile = id / splits;
        } else {
            splits = a.splits;
            tile = a.tiles - 1u - id / splits;  // a causal sequence's last rows, the longest, first
        }
        split = id % splits;
        it->slot = (kPaged ? a.splits : 0u) + split;
        auto start = [&](uint32_t r) { return a.q_off[r] * a.group / a.rows + r; };
        x = wave_find(a.batch, tile, start);
        t0 = a.q_off[x];
        t1 = a.q_off[x + 1];
        if (kPaged) {
            n = a.own_len[x];
            if (pages_of(n, a.pg.log_tokens) > a.own_width) return bad_seq(a, CR_ERR_SEQ);
            it->table = a.own_table + (uint64_t)x * a.own_width;
            it->causal = 1;
        } else {
            const uint32_t k0 = a.k_off[x], k1 = a.k_off[x + 1];
            if (k0 > k1 || k1 > a.total_k) return bad_seq(a, CR_ERR_SEQ);
            n = k1 - k0;
            it->key0 = k0;
            it->causal = a.causal;
        }
        tile -= min(start(x), tile);
    }
    if (t0 > t1 || t1 > a.total_q) return bad_seq(a, CR_ERR_SEQ);
    const uint32_t nq = t1 - t0, rows = nq * a.group;
    it->row0 = tile * a.rows;
    if (it->row0 >= rows) return false;
    it->rows = min(a.rows, rows - it->row0);
    it->tok0 = t0;
    it->first_lim = it->causal ? (int32_t)n - (int32_t)nq + 1 : (int32_t)n;
    uint32_t top = n;  // keys that the last row sees
    if (it->causal) top = (uint32_t)max(0, it->first_lim + (int32_t)((it->row0 + it->rows - 1u) / a.group));
    const uint32_t per = ((top + splits - 1u) / splits + kKeys - 1u) / kKeys * kKeys;
    it->begin = min(top, split * per);
    it->end = min(top, it->begin + per);
    return true;
}

// Tiles in LDS, in elements. Keys: pieces of 16 bytes, all rows of one piece together (a lane reads a
// row's piece, so 16 lanes read 256 contiguous bytes). Values: 32 elements, all rows of them together
// (a transposed read takes 4 rows of 64 bytes by 32 lanes, 256 contiguous bytes). Each run is
// shifted against the one before, so that the pieces of one row, which lie next to each other
// in memory and are written together, fall on different banks. All reads of a tile are one lane
// address and constants.
constexpr uint32_t kKeyRun = kKeys * 8u + 8u;
constexpr uint32_t kValRun = kKeys * 32u + 32u;
template <int kDim>
constexpr uint32_t kKeyTile = kDim / 8 * kKeyRun;
template <int kDim>
constexpr uint32_t kValTile = kDim / 32 * kValRun;

__device__ __forceinline__ s16x4 read_tr(const uint16_t* p)
{
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (__attribute__((address_space(3))) s16x4*)(__attribute__((address_space(3))) void*)const_cast<uint16_t*>(p));
}

// The larger of a column's values in the two half-waves, and their sum.
__device__ __forceinline__ float both_max(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

__device__ __forceinline__ float both_sum(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Tiles of keys and values on their way from memory to LDS: a thread moves one 16-byte piece of every
// kStep-th row.
template <int kDim, bool kPaged>
struct Loader {
    static constexpr uint32_t kPieces = kDim / 8, kStep = kThreads / kPieces, kPer = kKeys / kStep;
    const uint16_t *kb, *vb;
    uint32_t row, piece, end;
    uint32_t page[kPer];  // of the next tile's rows
    u32x4 rk[kPer], rv[kPer];

    __device__ __forceinline__ void init(const Attn& a, const Item& it, uint32_t head_kv)
    {
        piece = threadIdx.x % kPieces;
        row = threadIdx.x / kPieces;
        end = it.end;
        if (kPaged) {
            kb = a.pg.k + (int64_t)head_kv * a.pg.head_stride + piece * 8u;
            vb = a.pg.v + (int64_t)head_kv * a.pg.head_stride + piece * 8u;
        } else {
            kb = (const uint16_t*)a.k.p + (int64_t)head_kv * a.k.head_stride + (int64_t)it.key0 * a.k.token_stride + piece * 8u;
            vb = (const uint16_t*)a.v.p + (int64_t)head_kv * a.v.head_stride + (int64_t)it.key0 * a.v.token_stride + piece * 8u;
        }
    }
    // Rows behind the last key repeat it: their weights are 0, and nothing foreign is read.
    __device__ __forceinline__ uint32_t key(uint32_t k0, uint32_t p) const { return min(k0 + p * kStep + row, end - 1u); }

    __device__ __forceinline__ void pages(const Attn& a, const Item& it, uint32_t k0)
    {
        if (!kPaged) return;
#pragma unroll
        for (uint32_t p = 0; p < kPer; ++p) page[p] = it.table[key(k0, p) >> a.pg.log_tokens];
    }
    __device__ __forceinline__ void load(const Attn& a, uint32_t k0)
    {
#pragma unroll
        for (uint32_t p = 0; p < kPer; ++p) {
            const uint32_t j = key(k0, p);
            int64_t ak, av;
            if (kPaged) {
                uint32_t g = page[p];
                if (g >= a.pg.num_pages) {
                    atomicOr(a.err, CR_ERR_PAGE);
                    g = 0;
                }
                ak = (int64_t)((uint64_t)g * (uint32_t)a.pg.page_stride) +
                     (int64_t)((uint64_t)(j & ((1u << a.pg.log_tokens) - 1u)) * (uint32_t)a.pg.token_stride);
                av = ak;
            } else {
                ak = (int64_t)((uint64_t)j * (uint32_t)a.k.token_stride);
                av = (int64_t)((uint64_t)j * (uint32_t)a.v.token_stride);
            }
            rk[p] = *reinterpret_cast<const u32x4*>(kb + ak);
            rv[p] = *reinterpret_cast<const u32x4*>(vb + av);
        }
    }
    __device__ __forceinline__ void store(uint16_t* lk, uint16_t* lv) const
    {
#pragma unroll
        for (uint32_t p = 0; p < kPer; ++p) {
            const uint32_t r = p * kStep + row;
            *reinterpret_cast<u32x4*>(lk + piece * kKeyRun + r * 8u) = rk[p];
            *reinterpret_cast<u32x4*>(lv + (piece >> 2) * kValRun + r * 32u + (piece & 3u) * 8u) = rv[p];
        }
    }
};

// A wavefront keeps 32 kBlk rows, each in one column: S^T = K Q^T gives a lane its row's scores of 16
// of 32 keys (the other half-wave has the other 16), so the row's maximum needs one exchange, and
// the weights are the second operand of O^T = V^T P^T as they lie: the order of keys inside a
// product is the same on both sides, 4 + 4 of 16 per half-wave, which is what two transposed LDS
// reads of the values give.
//
// The wave works on half tiles of 32 keys: the weights of one (vector unit) beside the scores of the
// next (matrix unit), then the values of the first beside the maximum of the next. The maximum is
// moved, and what is summed rescaled, only when a score passes it by 2^kSlack.
template <typename E, int kDim, bool kPaged, int kBlk>
__global__ __launch_bounds__(kThreads, (kDim == 128 && kBlk == 2) ? 1 : 2) void k_attn(const Attn a)
{
    __shared__ __align__(16) uint16_t lds_k[2][kKeyTile<kDim>];
    __shared__ __align__(16) uint16_t lds_v[3][kValTile<kDim>];

    const uint32_t head_kv = blockIdx.x % a.heads_kv;
    Item it;
    if (!find_item<kPaged>(a, blockIdx.x / a.heads_kv, &it)) return;

    const uint32_t lane = lane_id(), wv = wave_in_block(), half = lane >> 5, col = lane & 31u;
    const uint32_t wrow = wv * 32u * kBlk;  // the wave's first row
    uint32_t tok[kBlk], head[kBlk];
    int32_t lim[kBlk];
#pragma unroll
    for (int b = 0; b < kBlk; ++b) {
        const uint32_t m = it.row0 + min(wrow + b * 32u + col, it.rows - 1u);
        tok[b] = it.tok0 + m / a.group;
        head[b] = head_kv * a.group + m % a.group;
        lim[b] = it.causal ? min(it.first_lim + (int32_t)(m / a.group), (int32_t)it.end) : (int32_t)it.end;
    }
    // keys that the wave's last and first rows see
    uint32_t w_end = 0, w_full = it.end;
    if (wrow < it.rows) {
        w_end = it.end;
        if (it.causal) {
            const uint32_t last = it.row0 + min(wrow + 32u * kBlk, it.rows) - 1u;
            w_end = (uint32_t)min((int32_t)it.end, max(0, it.first_lim + (int32_t)(last / a.group)));
            w_full = (uint32_t)min((int32_t)it.end, max(0, it.first_lim + (int32_t)((it.row0 + wrow) / a.group)));
        }
    }

    f32x16 o[kBlk][kDim / 32];
    float mc[kBlk], sum[kBlk];
#pragma unroll
    for (int b = 0; b < kBlk; ++b) {
        mc[b] = kNoMax;
        sum[b] = 0.f;
#pragma unroll
        for (int d = 0; d < kDim / 32; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[b][d][i] = 0.f;
    }

    if (it.begin < it.end) {
        Loader<kDim, kPaged> ld;
        ld.init(a, it, head_kv);
        ld.pages(a, it, it.begin);
        ld.load(a, it.begin);
        ld.pages(a, it, it.begin + kKeys);
        s16x8 qf[kBlk][kDim / 16];
#pragma unroll
        for (int b = 0; b < kBlk; ++b) {
            const uint16_t* qp = (const uint16_t*)a.q.p + (int64_t)tok[b] * a.q.token_stride + (int64_t)head[b] * a.q.head_stride;
#pragma unroll
            for (int s = 0; s < kDim / 16; ++s) qf[b][s] = *reinterpret_cast<const s16x8*>(qp + s * 16 + half * 8u);
        }
        f32x16 s[2][kBlk];

        // scores of half tile h (keys 32 h ..) of the tile in lk, into s[h]
        const uint32_t k_lane = half * kKeyRun + col * 8u, v_lane = (half * 4u + (lane & 15u) / 4u) * 32u + ((lane >> 4) & 1u) * 16u + (lane & 3u) * 4u;
        auto scores = [&](const uint16_t* lk, int h) {
#pragma unroll
            for (int b = 0; b < kBlk; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[h][b][i] = 0.f;
#pragma unroll
            for (int d = 0; d < kDim / 16; ++d) {
                const s16x8 kf = *reinterpret_cast<const s16x8*>(lk + k_lane + d * 2u * kKeyRun + h * 32u * 8u);
#pragma unroll
                for (int b = 0; b < kBlk; ++b) s[h][b] = E::mfma(kf, qf[b][d], s[h][b]);
            }
        };
        auto mask = [&](uint32_t k0, int h) {
#pragma unroll
            for (int b = 0; b < kBlk; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if ((int32_t)(k0 + h * 32u + 8u * (i / 4) + 4u * half + (i & 3)) >= lim[b]) s[h][b][i] = -INFINITY;
        };
        float top[kBlk];
        auto maxima = [&](int h) {
#pragma unroll
            for (int b = 0; b < kBlk; ++b) {
                float t = __builtin_elementwise_maximum(s[h][b][0], s[h][b][1]);
#pragma unroll
                for (int i = 2; i < 16; i += 2)
                    t = __builtin_elementwise_maximum(__builtin_elementwise_maximum(t, s[h][b][i]), s[h][b][i + 1]);
                top[b] = both_max(t) * a.c;
            }
        };
        auto rescale = [&]() {
            bool up = false;
#pragma unroll
            for (int b = 0; b < kBlk; ++b) up |= top[b] > mc[b] + kSlack;
            if (!ballot(up)) return;
#pragma unroll
            for (int b = 0; b < kBlk; ++b) {
                const float m = fmaxf(mc[b], top[b]), f = __builtin_amdgcn_exp2f(mc[b] - m);
                mc[b] = m;
                sum[b] *= f;
#pragma unroll
                for (int d = 0; d < kDim / 32; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[b][d][i] *= f;
            }
        };
        uint32_t pk[kBlk][8];
        auto weights = [&](int h) {
#pragma unroll
            for (int b = 0; b < kBlk; ++b) {
                float t[4];
#pragma unroll
                for (int i = 0; i < 16; i += 2) {
                    const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[h][b][i], a.c, -mc[b]));
                    const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(s[h][b][i + 1], a.c, -mc[b]));
                    t[i & 3] = i < 4 ? x : t[i & 3] + x;
                    t[(i & 3) + 1] = i < 4 ? y : t[(i & 3) + 1] + y;
                    pk[b][i / 2] = E::pack(x, y);
                }
                sum[b] += (t[0] + t[1]) + (t[2] + t[3]);
            }
        };
        auto values = [&](const uint16_t* lv, int h) {
#pragma unroll
            for (int ks = 0; ks < 2; ++ks)
#pragma unroll
                for (int d = 0; d < kDim / 32; ++d) {
                    s16x4 vf[2];
#pragma unroll
                    for (int y = 0; y < 2; ++y) vf[y] = read_tr(lv + v_lane + d * kValRun + (h * 32u + ks * 16u + y * 8u) * 32u);
#pragma unroll
                    for (int b = 0; b < kBlk; ++b) {
                        const u32x4 w = {pk[b][ks * 4], pk[b][ks * 4 + 1], pk[b][ks * 4 + 2], pk[b][ks * 4 + 3]};
                        o[b][d] = E::mfma(__builtin_shufflevector(vf[0], vf[1], 0, 1, 2, 3, 4, 5, 6, 7), __builtin_bit_cast(s16x8, w), o[b][d]);
                    }
                }
        };

        // Order of instructions: every matrix product with its share of vector work behind it, the
        // fragments read two products ahead.
        auto order_scores = [&]() {
            constexpr int kSteps = kDim / 16, kTrans = 16 * kBlk / kSteps, kVec = 40 * kBlk / kSteps;
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
#pragma unroll
            for (int d = 0; d < kSteps; ++d) {
                __builtin_amdgcn_sched_group_barrier(0x008, kBlk, 0);
                __builtin_amdgcn_sched_group_barrier(0x400, kTrans, 0);
                __builtin_amdgcn_sched_group_barrier(0x002, kVec, 0);
                if (d + 2 < kSteps) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
        };
        auto order_values = [&]() {
            constexpr int kSteps = kDim / 16;
            __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
            for (int d = 0; d < kSteps; ++d) {
                __builtin_amdgcn_sched_group_barrier(0x008, kBlk, 0);
                __builtin_amdgcn_sched_group_barrier(0x002, 2 * kBlk, 0);
                if (d + 2 < kSteps) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
        };

        // Loads behind the last key repeat its row, so they need no branch.
        ld.store(lds_k[0], lds_v[0]);
        ld.load(a, it.begin + kKeys);
        ld.pages(a, it, it.begin + 2u * kKeys);
        __syncthreads();
        scores(lds_k[0], 0);
        mask(it.begin, 0);
        maxima(0);
        rescale();
        uint32_t kbuf = 0, vbuf = 0, k0 = it.begin;
        // The next tile into LDS, the one behind it into registers. The keys' buffer was last read before
        // the last barrier, the values' two tiles ago.
        auto stage = [&]() {
            kbuf ^= 1u;
            vbuf = vbuf == 2u ? 0u : vbuf + 1u;
            if (k0 + kKeys < it.end) ld.store(lds_k[kbuf], lds_v[vbuf]);
            ld.load(a, k0 + 2u * kKeys);
            ld.pages(a, it, k0 + 3u * kKeys);
            __syncthreads();
        };
        auto tile = [&](auto masked) {
            const uint16_t* lv = lds_v[vbuf];
            scores(lds_k[kbuf], 1);
            weights(0);
            order_scores();
            if (masked) mask(k0, 1);
            values(lv, 0);
            maxima(1);
            order_values();
            rescale();
            stage();
            scores(lds_k[kbuf], 0);  // behind the last tile: of whatever lies there, all masked
            weights(1);
            order_scores();
            if (masked) mask(k0 + kKeys, 0);
            values(lv, 1);
            maxima(0);
            order_values();
            rescale();
            k0 += kKeys;
        };
        while (k0 + 2u * kKeys <= w_full) tile(std::false_type{});
        while (k0 < w_end) tile(std::true_type{});
        for (; k0 < it.end; k0 += kKeys) stage();  // keys that only other waves' rows see
    }

#pragma unroll
    for (int b = 0; b < kBlk; ++b) {
        const float total = both_sum(sum[b]);
        if (wrow + b * 32u + col >= it.rows) continue;
        const bool none = total == 0.f;  // the largest weight of a row that sees a key is 1 or more
        const float inv = none ? 0.f : 1.f / total;
        const float lse2 = none ? -INFINITY : mc[b] + log2f(total);
        const uint64_t orow = (uint64_t)tok[b] * a.heads_q + head[b];
        if (a.part_o) {
            const uint64_t at = (uint64_t)it.slot * a.total_q * a.heads_q + orow;
            if (half == 0) a.part_lse[at] = lse2;
            if (none) continue;
#pragma unroll
            for (int d = 0; d < kDim / 32; ++d)
#pragma unroll
                for (int i = 0; i < 16; i += 4)
                    *reinterpret_cast<f32x4*>(a.part_o + at * kDim + d * 32 + 2 * i + half * 4u) =
                        f32x4{o[b][d][i] * inv, o[b][d][i + 1] * inv, o[b][d][i + 2] * inv, o[b][d][i + 3] * inv};
            continue;
        }
        if (a.lse && half == 0) a.lse[orow] = lse2 * kLn2;
        uint16_t* op = (uint16_t*)a.out.p + (int64_t)tok[b] * a.out.token_stride + (int64_t)head[b] * a.out.head_stride;
#pragma unroll
        for (int d = 0; d < kDim / 32; ++d)
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                *reinterpret_cast<uint2*>(op + d * 32 + 2 * i + half * 4u) =
                    uint2{E::pack(o[b][d][i] * inv, o[b][d][i + 1] * inv), E::pack(o[b][d][i + 2] * inv, o[b][d][i + 3] * inv)};
    }
}

// Joins the partial results of a row: 4 elements per thread.
template <typename E, int kDim>
__global__ __launch_bounds__(256) void k_attn_join(const Attn a)
{
    constexpr uint32_t kPer = kDim / 4;
    const uint64_t rows = (uint64_t)a.total_q * a.heads_q;
    const uint64_t x = (uint64_t)blockIdx.x * 256u + threadIdx.x, row = x / kPer;
    if (row >= rows) return;
    const uint32_t e = (uint32_t)(x % kPer) * 4u, slots = a.splits + a.own_splits;
    float mx = -INFINITY;
    for (uint32_t s = 0; s < slots; ++s) mx = fmaxf(mx, a.part_lse[s * rows + row]);
    float sum = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    if (mx != -INFINITY) {
        for (uint32_t s = 0; s < slots; ++s) {
            const float l = a.part_lse[s * rows + row];
            if (l == -INFINITY) continue;
            const float w = __builtin_amdgcn_exp2f(l - mx);
            const f32x4 v = *reinterpret_cast<const f32x4*>(a.part_o + (s * rows + row) * kDim + e);
            sum += w;
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[i] = __builtin_fmaf(w, v[i], acc[i]);
        }
    }
    const float inv = sum > 0.f ? 1.f / sum : (mx == -INFINITY ? 0.f : 1.f / sum);
    const uint32_t tok = (uint32_t)(row / a.heads_q), head = (uint32_t)(row % a.heads_q);
    uint16_t* op = (uint16_t*)a.out.p + (int64_t)tok * a.out.token_stride + (int64_t)head * a.out.head_stride + e;
    *reinterpret_cast<uint2*>(op) = uint2{E::pack(acc[0] * inv, acc[1] * inv), E::pack(acc[2] * inv, acc[3] * inv)};
    if (a.lse && e == 0) a.lse[row] = mx == -INFINITY ? -INFINITY : (mx + log2f(sum)) * kLn2;
}

// Keys a block should have at least where a call is split, and workgroups that fill the GPU.
constexpr uint32_t kSplitKeys = 256, kSplitMax = 32;

// Parts of `keys` so that `blocks` workgroups of one part each become enough to fill the GPU.
inline uint32_t split_of(uint64_t blocks, uint64_t keys)
{
    const uint64_t want = 512u / (blocks ? blocks : 1u), most = keys / kSplitKeys;
    uint64_t s = want < most ? want : most;
    s = s < kSplitMax ? s : kSplitMax;
    return (uint32_t)(s ? s : 1u);
}

inline bool good_scale(float s) { return s > 0.f && s <= 3.0e38f; }

inline bool good_heads(uint32_t hq, uint32_t hkv) { return hkv >= 1 && hq >= hkv && hq <= CR_MAX_HEADS && hq % hkv == 0; }

inline bool good_prompt_sizes(const cr_attn_prompt_args* p)
{
    return p && p->dtype <= CR_F16 && good_heads(p->heads_q, p->heads_kv) && (p->dim == 64 || p->dim == 128) &&
           p->causal <= 1 && good_scale(p->scale) && (uint64_t)p->total_q * p->heads_q < (1ull << 31) &&
           p->total_k < (1u << 31) && p->batch <= (1u << 24) && (p->batch > 0 || p->total_q == 0);
}

inline bool good_shared_sizes(const cr_kv_cache* c, const cr_attn_shared_args* p)
{
    return good_cache_sizes(c) && p && good_heads(p->heads_q, c->heads) && p->layer < c->layers && good_scale(p->scale) &&
           (uint64_t)p->total_q * p->heads_q < (1ull << 31) && p->batch <= (1u << 24) && p->groups <= p->batch &&
           (p->total_q == 0 || p->groups > 0) && ((uint64_t)p->prefix_width * c->page_tokens) < (1ull << 31) &&
           ((uint64_t)p->own_width * c->page_tokens) < (1ull << 31);
}

// Query rows per block: 256 where the tiles of 256 fill the GPU by themselves, else 128.
inline uint32_t rows_of(uint64_t rows, uint32_t heads_kv) { return rows * heads_kv >= 256ull * 256u ? 256u : 128u; }

// Tiles that a call's rows make, about: whole ones, and one for each sequence's rest.
inline uint64_t tiles_of(uint64_t rows, uint32_t per, uint32_t seqs) { return rows / per + (rows < (uint64_t)seqs * per ? seqs : 1u); }

inline void prompt_shape(const cr_attn_prompt_args* p, uint32_t* per, uint32_t* splits)
{
    const uint64_t rows = (uint64_t)p->total_q * (p->heads_q / p->heads_kv);
    *per = rows_of(rows, p->heads_kv);
    *splits = p->total_q ? split_of(tiles_of(rows, *per, p->batch) * p->heads_kv, p->total_k / p->batch) : 1u;
}

inline void shared_shape(const cr_kv_cache* c, const cr_attn_shared_args* p, uint32_t* per, uint32_t* prefix, uint32_t* own)
{
    const uint64_t rows = (uint64_t)p->total_q * (p->heads_q / c->heads);
    *per = rows_of(rows, c->heads);
    *prefix = split_of(tiles_of(rows, *per, p->groups) * c->heads, (uint64_t)p->prefix_width * c->page_tokens);
    *own = split_of(tiles_of(rows, *per, p->batch) * c->heads, (uint64_t)p->own_width * c->page_tokens);
}

inline size_t part_bytes(uint64_t slots, uint64_t rows, uint32_t dim) { return slots * rows * (dim + 4u) * sizeof(float); }

inline void set_parts(Attn* a, void* ws, uint64_t slots, uint32_t dim)
{
    a->part_o = (float*)ws;
    a->part_lse = a->part_o + slots * a->total_q * a->heads_q * dim;
}

template <typename E, int kDim, bool kPaged>
void launch(const Attn& a, hipStream_t st)
{
    const uint64_t items = (uint64_t)a.tiles * a.splits + (uint64_t)a.own_tiles * a.own_splits;
    const dim3 grid((uint32_t)(items * a.heads_kv));
    if (a.rows == 256u) hipLaunchKernelGGL((k_attn<E, kDim, kPaged, 2>), grid, dim3(kThreads), 0, st, a);
    else hipLaunchKernelGGL((k_attn<E, kDim, kPaged, 1>), grid, dim3(kThreads), 0, st, a);
    if (a.part_o) {
        const uint64_t threads = (uint64_t)a.total_q * a.heads_q * (kDim / 4);
        hipLaunchKernelGGL((k_attn_join<E, kDim>), dim3((uint32_t)((threads + 255u) / 256u)), dim3(256), 0, st, a);
    }
}

template <bool kPaged>
cr_status dispatch(const Attn& a, uint32_t dtype, uint32_t dim, void* stream)
{
    const hipStream_t st = as_stream(stream);
    const uint64_t items = (uint64_t)a.tiles * a.splits + (uint64_t)a.own_tiles * a.own_splits;
    if (items * a.heads_kv >= (1ull << 31)) return CR_EINVAL;
    (void)hipGetLastError();
    if (dtype == CR_BF16 && dim == 128) launch<Bf16, 128, kPaged>(a, st);
    else if (dtype == CR_BF16) launch<Bf16, 64, kPaged>(a, st);
    else if (dim == 128) launch<F16, 128, kPaged>(a, st);
    else launch<F16, 64, kPaged>(a, st);
    return hipGetLastError() == hipSuccess ? CR_OK : CR_EHIP;
}

}  // namespace
}  // namespace cr

extern "C" size_t cr_attn_prompt_workspace_bytes(const cr_attn_prompt_args* p)
{
    using namespace cr;
    if (!good_prompt_sizes(p)) return 0;
    uint32_t per, s;
    prompt_shape(p, &per, &s);
    return s > 1 ? part_bytes(s, (uint64_t)p->total_q * p->heads_q, p->dim) : 0;
}

extern "C" cr_status cr_attn_prompt(const cr_attn_prompt_args* p, void* ws, size_t ws_bytes, uint32_t* err, void* stream)
{
    using namespace cr;
    if (!good_prompt_sizes(p) || !err) return CR_EINVAL;
    if (p->total_q == 0) return CR_OK;
    if (!good_rows(p->q) || !good_rows(p->out) || !p->q_off || !p->k_off ||
        (p->total_k > 0 && (!good_rows(p->k) || !good_rows(p->v))) || (p->lse && !aligned4(p->lse)))
        return CR_EINVAL;
    const size_t need = cr_attn_prompt_workspace_bytes(p);
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
    prompt_shape(p, &a.rows, &a.splits);
    a.tiles = (uint32_t)((uint64_t)p->total_q * a.group / a.rows) + p->batch;
    if (a.splits > 1) set_parts(&a, ws, a.splits, p->dim);
    a.err = err;
    return dispatch<false>(a, p->dtype, p->dim, stream);
}

extern "C" size_t cr_attn_shared_workspace_bytes(const cr_kv_cache* c, const cr_attn_shared_args* p)
{
    using namespace cr;
    if (!good_shared_sizes(c, p)) return 0;
    uint32_t per, s1, s2;
    shared_shape(c, p, &per, &s1, &s2);
    return part_bytes((uint64_t)s1 + s2, (uint64_t)p->total_q * p->heads_q, c->dim);
}

extern "C" cr_status cr_attn_shared(const cr_kv_cache* c, const cr_attn_shared_args* p, void* ws, size_t ws_bytes,
                                    uint32_t* err, void* stream)
{
    using namespace cr;
    if (!good_cache(c) || !good_shared_sizes(c, p) || !err) return CR_EINVAL;
    if (p->total_q == 0) return CR_OK;
    if (!good_rows(p->q) || !good_rows(p->out) || !p->q_off || !p->group_off || !p->prefix_len || !p->own_len ||
        (p->prefix_width && !p->prefix_table) || (p->own_width && !p->own_table) || (p->lse && !aligned4(p->lse)) || !ws ||
        !aligned16(ws))
        return CR_EINVAL;
    if (ws_bytes < cr_attn_shared_workspace_bytes(c, p)) return CR_ESIZE;
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
    shared_shape(c, p, &a.rows, &a.splits, &a.own_splits);
    const uint64_t rows = (uint64_t)p->total_q * a.group;
    a.tiles = (uint32_t)(rows / a.rows) + p->groups;
    a.own_tiles = (uint32_t)(rows / a.rows) + p->batch;
    set_parts(&a, ws, (uint64_t)a.splits + a.own_splits, c->dim);
    a.err = err;
    return dispatch<true>(a, c->dtype, c->dim, stream);
}
