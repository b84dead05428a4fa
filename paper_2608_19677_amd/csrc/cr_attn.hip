// Attention of a destination: whole prompts (packed, causal, grouped heads) and requests that share a
// cached prefix in pages.
//
// Mathematics: scores s_j = scale q.k_j, running maximum m and sum l of exp(s_j - m) over the keys
// in one pass, o = sum_j exp(s_j - m) v_j / l, lse = m + ln l. Results over disjoint sets of keys
// are joined by lse = ln sum exp(lse_p), o = sum exp(lse_p - lse) o_p. Exponentials are taken base
// 2 with log2(e) folded into the scale.
#include "cr_kv.h"

namespace cr {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr uint32_t kWaves = 4;
constexpr uint32_t kThreads = kWaves * kWave;
constexpr uint32_t kRows = kWaves * 32;  // query rows (token, head of the group) per block
constexpr uint32_t kKeys = 64;           // keys per step
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

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

// Tile t of sequence x starts at floor(first row / kRows) + x: steps of at least
// ceil(rows / kRows), so that the tiles of all sequences fit into floor(all rows / kRows) +
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
        auto start = [&](uint32_t g) {
            return ((uint64_t)a.q_off[min(a.group_off[g], a.batch)] * a.group) / kRows + g;
        };
        x = wave_find(a.groups, tile, start);
        const uint32_t r0 = a.group_off[x], r1 = a.group_off[x + 1];
        if (r0 > r1 || r1 > a.batch) return bad_seq(a, CR_ERR_SEQ);
        t0 = a.q_off[r0];
        t1 = a.q_off[r1];
        n = a.prefix_len[x];
        if (pages_of(n, a.pg.log_tokens) > a.prefix_width) return bad_seq(a, CR_ERR_SEQ);
        it->table = a.prefix_table + (uint64_t)x * a.prefix_width;
        it->causal = 0;
        tile -= (uint32_t)min(start(x), (uint64_t)tile);
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
        auto start = [&](uint32_t r) { return ((uint64_t)a.q_off[r] * a.group) / kRows + r; };
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
        tile -= (uint32_t)min(start(x), (uint64_t)tile);
    }
    if (t0 > t1 || t1 > a.total_q) return bad_seq(a, CR_ERR_SEQ);
    const uint32_t nq = t1 - t0, rows = nq * a.group;
    it->row0 = tile * kRows;
    if (it->row0 >= rows) return false;
    it->rows = min(kRows, rows - it->row0);
    it->tok0 = t0;
    it->first_lim = it->causal ? (int32_t)n - (int32_t)nq + 1 : (int32_t)n;
    uint32_t top = n;  // keys that the last row sees
    if (it->causal) top = (uint32_t)max(0, it->first_lim + (int32_t)((it->row0 + it->rows - 1u) / a.group));
    const uint32_t per = ((top + splits - 1u) / splits + kKeys - 1u) / kKeys * kKeys;
    it->begin = min(top, split * per);
    it->end = min(top, it->begin + per);
    return true;
}

// Swizzles of the tiles in LDS, by 16-byte pieces of a row. Keys are read a row per lane: 16 rows
// at one piece must fall on all 64 banks. Values are read transposed, 4 rows of 64 bytes by 32
// lanes: these rows must fall on different banks.
template <int kDim>
__device__ __forceinline__ uint32_t k_piece(uint32_t row, uint32_t piece)
{
    return kDim == 128 ? piece ^ (row & 15u) : piece ^ ((row >> 1) & 7u);
}

template <int kDim>
__device__ __forceinline__ uint32_t v_piece(uint32_t row, uint32_t piece)
{
    return kDim == 128 ? piece ^ ((row & 3u) << 2) : piece ^ (((row >> 1) & 1u) << 2);
}

__device__ __forceinline__ s16x4 read_tr(const uint16_t* p)
{
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (__attribute__((address_space(3))) s16x4*)(__attribute__((address_space(3))) void*)const_cast<uint16_t*>(p));
}

// The other half-wave's value of the same column.
__device__ __forceinline__ float other_half(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(lane_id() < 32u ? r[1] : r[0]);
}

// A wavefront keeps 32 rows: their queries as the second operand of S^T = K Q^T, so that a lane
// holds one row's scores of 16 of 32 keys (the other half-wave the other 16), the row's maximum
// needs one exchange, and the weights are the second operand of O^T = V^T P^T as they lie: the
// order of keys inside a product is the same on both sides, 4 + 4 of 16 per half-wave, which is
// what two transposed LDS reads of the values give.
template <typename E, int kDim, bool kPaged>
__global__ __launch_bounds__(kThreads, 2) void k_attn(const Attn a)
{
    constexpr uint32_t kPieces = kDim / 8, kRowsPerPass = kThreads / kPieces, kPasses = kKeys / kRowsPerPass;
    __shared__ __align__(16) uint16_t lds_k[kKeys * kDim];
    __shared__ __align__(16) uint16_t lds_v[kKeys * kDim];

    const uint32_t head_kv = blockIdx.x % a.heads_kv;
    Item it;
    if (!find_item<kPaged>(a, blockIdx.x / a.heads_kv, &it)) return;

    const uint32_t lane = lane_id(), wv = wave_in_block(), half = lane >> 5, col = lane & 31u;
    const uint32_t m_local = wv * 32u + col;
    const bool row_ok = m_local < it.rows;
    const uint32_t m = it.row0 + min(m_local, it.rows - 1u);
    const uint32_t tok = it.tok0 + m / a.group, head = head_kv * a.group + m % a.group;
    const uint64_t orow = (uint64_t)tok * a.heads_q + head;
    const int32_t lim = it.causal ? min(it.first_lim + (int32_t)(m / a.group), (int32_t)it.end) : (int32_t)it.end;

    f32x16 o[kDim / 32];
#pragma unroll
    for (int d = 0; d < kDim / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
    float mx = -INFINITY, sum = 0.f;

    if (it.begin < it.end) {
        s16x8 qf[kDim / 16];
        const uint16_t* qp = (const uint16_t*)a.q.p + (int64_t)tok * a.q.token_stride + (int64_t)head * a.q.head_stride;
#pragma unroll
        for (int s = 0; s < kDim / 16; ++s) qf[s] = *reinterpret_cast<const s16x8*>(qp + s * 16 + half * 8u);

        const uint32_t piece = threadIdx.x % kPieces, lrow = threadIdx.x / kPieces;
        const uint16_t *kb, *vb;
        if (kPaged) {
            kb = a.pg.k + (int64_t)head_kv * a.pg.head_stride + piece * 8u;
            vb = a.pg.v + (int64_t)head_kv * a.pg.head_stride + piece * 8u;
        } else {
            kb = (const uint16_t*)a.k.p + (int64_t)head_kv * a.k.head_stride + (int64_t)it.key0 * a.k.token_stride + piece * 8u;
            vb = (const uint16_t*)a.v.p + (int64_t)head_kv * a.v.head_stride + (int64_t)it.key0 * a.v.token_stride + piece * 8u;
        }
        for (uint32_t k0 = it.begin; k0 < it.end; k0 += kKeys) {
            uint4 rk[kPasses], rv[kPasses];
#pragma unroll
            for (uint32_t p = 0; p < kPasses; ++p) {
                // rows behind the last key repeat it: their weights are 0, and nothing foreign is read
                const uint32_t j = min(k0 + p * kRowsPerPass + lrow, it.end - 1u);
                int64_t ak, av;
                if (kPaged) {
                    uint32_t page = it.table[j >> a.pg.log_tokens];
                    if (page >= a.pg.num_pages) {
                        atomicOr(a.err, CR_ERR_PAGE);
                        page = 0;
                    }
                    ak = (int64_t)page * a.pg.page_stride + (int64_t)(j & ((1u << a.pg.log_tokens) - 1u)) * a.pg.token_stride;
                    av = ak;
                } else {
                    ak = (int64_t)j * a.k.token_stride;
                    av = (int64_t)j * a.v.token_stride;
                }
                rk[p] = *reinterpret_cast<const uint4*>(kb + ak);
                rv[p] = *reinterpret_cast<const uint4*>(vb + av);
            }
            __syncthreads();
#pragma unroll
            for (uint32_t p = 0; p < kPasses; ++p) {
                const uint32_t r = p * kRowsPerPass + lrow;
                *reinterpret_cast<uint4*>(lds_k + r * kDim + k_piece<kDim>(r, piece) * 8u) = rk[p];
                *reinterpret_cast<uint4*>(lds_v + r * kDim + v_piece<kDim>(r, piece) * 8u) = rv[p];
            }
            __syncthreads();
            f32x16 s[2];
#pragma unroll
            for (int b = 0; b < 2; ++b) {
#pragma unroll
                for (int i = 0; i < 16; ++i) s[b][i] = 0.f;
#pragma unroll
                for (int d = 0; d < kDim / 16; ++d) {
                    const uint32_t r = b * 32u + col;
                    s[b] = E::mfma(*reinterpret_cast<const s16x8*>(lds_k + r * kDim + k_piece<kDim>(r, d * 2u + half) * 8u), qf[d], s[b]);
                }
            }
            float top = -INFINITY;
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int32_t j = (int32_t)(k0 + b * 32u + 8u * (i / 4) + 4u * half + (i & 3));
                    s[b][i] = j < lim ? s[b][i] : -INFINITY;
                    top = fmaxf(top, s[b][i]);
                }
            top = fmaxf(top, other_half(top));
            const float mn = fmaxf(mx, top);
            const float mc = mn == -INFINITY ? 0.f : mn * a.c;
            const float keep = __builtin_amdgcn_exp2f(__builtin_fmaf(mx, a.c, -mc));  // 0 before the first key
            mx = mn;
            sum *= keep;
#pragma unroll
            for (int d = 0; d < kDim / 32; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= keep;
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    s[b][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][i], a.c, -mc));
                    sum += s[b][i];
                }
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) {
                uint32_t pk[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) pk[i] = E::pack(s[ks / 2][(ks & 1) * 8 + 2 * i], s[ks / 2][(ks & 1) * 8 + 2 * i + 1]);
                const s16x8 pf = __builtin_bit_cast(s16x8, pk);
#pragma unroll
                for (int d = 0; d < kDim / 32; ++d) {
                    s16x4 vf[2];
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const uint32_t r = ks * 16u + y * 8u + half * 4u + (lane & 15u) / 4u;
                        const uint32_t e = d * 32u + ((lane >> 4) & 1u) * 16u + (lane & 3u) * 4u;
                        vf[y] = read_tr(lds_v + r * kDim + v_piece<kDim>(r, e / 8u) * 8u + (e & 7u));
                    }
                    o[d] = E::mfma(__builtin_bit_cast(s16x8, vf), pf, o[d]);
                }
            }
        }
    }

    sum += other_half(sum);
    if (!row_ok) return;
    const bool none = !(sum > 0.f) && mx == -INFINITY;
    const float inv = none ? 0.f : 1.f / sum;
    const float lse2 = none ? -INFINITY : __builtin_fmaf(mx, a.c, log2f(sum));
    if (a.part_o) {
        const uint64_t at = (uint64_t)it.slot * a.total_q * a.heads_q + orow;
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

inline uint32_t prompt_splits(const cr_attn_prompt_args* p)
{
    if (p->total_q == 0) return 1;
    const uint64_t rows = (uint64_t)p->total_q * (p->heads_q / p->heads_kv);
    const uint64_t tiles = rows / kRows + (rows < (uint64_t)p->batch * kRows ? p->batch : 1u);
    return split_of(tiles * p->heads_kv, p->total_k / p->batch);
}

inline void shared_splits(const cr_kv_cache* c, const cr_attn_shared_args* p, uint32_t* prefix, uint32_t* own)
{
    const uint64_t rows = (uint64_t)p->total_q * (p->heads_q / c->heads);
    const uint64_t t1 = rows / kRows + (rows < (uint64_t)p->groups * kRows ? p->groups : 1u);
    const uint64_t t2 = rows / kRows + (rows < (uint64_t)p->batch * kRows ? p->batch : 1u);
    *prefix = split_of(t1 * c->heads, (uint64_t)p->prefix_width * c->page_tokens);
    *own = split_of(t2 * c->heads, (uint64_t)p->own_width * c->page_tokens);
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
    hipLaunchKernelGGL((k_attn<E, kDim, kPaged>), dim3((uint32_t)(items * a.heads_kv)), dim3(kThreads), 0, st, a);
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
    const uint32_t s = prompt_splits(p);
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
    a.tiles = (uint32_t)((uint64_t)p->total_q * a.group / kRows) + p->batch;
    a.splits = prompt_splits(p);
    if (a.splits > 1) set_parts(&a, ws, a.splits, p->dim);
    a.err = err;
    return dispatch<false>(a, p->dtype, p->dim, stream);
}

extern "C" size_t cr_attn_shared_workspace_bytes(const cr_kv_cache* c, const cr_attn_shared_args* p)
{
    using namespace cr;
    if (!good_shared_sizes(c, p)) return 0;
    uint32_t s1, s2;
    shared_splits(c, p, &s1, &s2);
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
    const uint64_t rows = (uint64_t)p->total_q * a.group;
    a.tiles = (uint32_t)(rows / kRows) + p->groups;
    a.own_tiles = (uint32_t)(rows / kRows) + p->batch;
    shared_splits(c, p, &a.splits, &a.own_splits);
    set_parts(&a, ws, (uint64_t)a.splits + a.own_splits, c->dim);
    a.err = err;
    return dispatch<true>(a, c->dtype, c->dim, stream);
}
