// The cache held in 8 bits: new tokens rounded into it, and tokens read back.
//
// Mathematics: a block (block_tokens tokens of one head, keys or values) holds codes c of an 8-bit float and one exponent
// e, x = c 2^e. e is the smallest integer with max |x| <= 1.75 * 2^kTop * 2^e (1.75 * 2^kTop is the largest code), or the e the block has from
// before if that is larger; c = x 2^-e rounded to the nearest. The products with powers of two are exact, so each element is
// rounded once. Exponents come from the bits of the largest magnitude, which is found among the elements' bits
// as integers (magnitudes of floats are ordered like their bits).
#include "cr_codes.h"

#include <type_traits>

namespace cr {
namespace {

constexpr uint32_t kQThreads = 256;
constexpr uint32_t kQWaves = kQThreads / kWave;
constexpr uint32_t kQBlocks = 1u << 20;  // of a launch; waves take more work in turn

// Magnitude bits of the largest element that both types have: the largest exponent, all of the code's bits set.
template <typename T, typename C>
constexpr uint32_t most_bits()
{
    return T::kInf - (1u << (T::kBits - C::kBits));
}

// Stored exponent for a largest magnitude (its bits in the element type, at most most_bits()).
template <typename T, typename C>
__device__ __forceinline__ uint32_t exponent_of(uint32_t top)
{
    const uint32_t f = __float_as_uint(T::first(top));  // f16's small ones are normal floats
    const int e = (int)(f >> 23) - C::kTop + ((f & 0x7FFFFFu) > 0x600000u ? 1 : 0);  // 1.75 = 1 + 0x600000 / 2^23
    return (uint32_t)max(e, 1);
}

// The larger magnitudes of two pairs of elements.
__device__ __forceinline__ uint32_t max_pair(uint32_t a, uint32_t b)
{
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}

struct QCall {
    KvqPages c;
    uint16_t* scale;       // the layer's scales, by pairs
    cr_rows k, v;
    const uint32_t* off;
    const uint32_t* length;
    const uint32_t* table;
    uint32_t total, n, width;
    uint32_t log_span;     // append: tokens of a wave's piece of work
    uint32_t items;        // append: spans x heads
    uint32_t* err;
};

// Whether sequence x's rows and length fit; o0, o1, len are filled.
__device__ __forceinline__ bool q_fits(const QCall& a, uint32_t x, uint32_t* o0, uint32_t* o1, uint32_t* len)
{
    *o0 = a.off[x];
    *o1 = a.off[x + 1u];
    *len = a.length[x];
    return *o0 <= *o1 && *o1 <= a.total && *o1 - *o0 <= *len && pages_of(*len, a.c.log_tokens) <= a.width;
}

// Every sequence's offsets and length are looked at by the wave of its number.
__device__ __forceinline__ void q_check(const QCall& a, uint64_t x)
{
    uint32_t o0, o1, len;
    if (x >= a.n || lane_id() != 0) return;
    if (!q_fits(a, (uint32_t)x, &o0, &o1, &len) || (x == 0 && o0 != 0u) || (x + 1u == a.n && o1 != a.total)) atomicOr(a.err, CR_ERR_SEQ);
}

// First span of sequence x whose rows start at `first`. n rows touch no more than n spans, nor more than floor(n / span) + 2, so
// no pass counts them; a decode step has one for each row.
__host__ __device__ __forceinline__ uint64_t span_start(uint32_t first, uint32_t x, uint32_t log_span)
{
    const uint64_t few = (uint64_t)(first >> log_span) + 2u * (uint64_t)x;
    return few < first ? few : first;
}

// New tokens. A wave takes a span of one head's keys and values: a block, or as many blocks as its lanes hold rows of (4 rows of
// 128 elements, 8 of 64; a lane has 8 elements of a row). The magnitudes' maximum goes over the lanes of a block; rows from before that
// share a block are rounded again only where its exponent grows.
//
// Bound by memory: 17,221 new tokens of 8 heads of 128 (106 MB read and written) take 19.4 us, 5.5 TB/s (24 in its
// first form, with ordinary stores); by the chain of dependent loads where there are few: a token for each of 256 requests
// 5.9 us (8.2 in its first form, with a wave for keys and one for values). A block of more than kHold steps of rows (16 of 128 elements,
// 32 of 64) is read twice, for its largest magnitude and for its codes, and a wave has nothing beside it: the 17,221 tokens take 32 us
// with blocks of 64 tokens and 40 with blocks of 128, the 256 requests' 10 and 15.
template <typename T, typename C, int kDim>
__device__ __forceinline__ void append_span(const QCall& a, uint8_t* ck, uint8_t* cv, uint32_t item)
{
    constexpr uint32_t kPieces = kDim / 8, kRows = kWave / kPieces;  // lanes of a row, rows of a wave
    constexpr uint32_t kHold = 4;                                    // steps of rows held in registers
    constexpr uint32_t kMostBits = most_bits<T, C>();
    const uint32_t lane = lane_id(), piece = lane % kPieces, row = lane / kPieces;
    const uint32_t bl = a.c.log_block, mask = (1u << a.c.log_tokens) - 1u;
    const uint32_t u = item / a.c.heads, head = item % a.c.heads;
    auto start = [&](uint32_t x) { return span_start(a.off[x], x, a.log_span); };
    const uint32_t x = wave_find(a.n, u, start);
    uint32_t o0, o1, len;
    const bool fits = q_fits(a, x, &o0, &o1, &len);
    const uint64_t s = span_start(o0, x, a.log_span);
    if (!fits || o0 == o1 || u < s) return;
    const uint32_t p0 = len - (o1 - o0);  // place of the first new token
    const uint64_t s0 = ((p0 >> a.log_span) + (u - s)) << a.log_span;
    if (s0 >= len) return;
    // The lane's rows are pos, pos + kRows, ...: in one block, or there is one step. A span ends below 2^32.
    const uint32_t pos = (uint32_t)s0 + row, block = pos >> bl << bl, steps = ((1u << a.log_span) + kRows - 1u) / kRows;
    const uint32_t page = a.table[(uint64_t)x * a.width + (min(pos, len - 1u) >> a.c.log_tokens)];

    u32x4 r[2][kHold];
    auto is_new = [&](uint32_t step) { return step < steps && pos + step * kRows >= p0 && pos + step * kRows < len; };
    auto load = [&](uint32_t step0) {  // 0 where there is no new token
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const cr_rows& rows = j ? a.v : a.k;
            const uint16_t* src = (const uint16_t*)rows.p + (int64_t)head * rows.head_stride + piece * 8u;
#pragma unroll
            for (uint32_t y = 0; y < kHold; ++y) {
                r[j][y] = u32x4{0, 0, 0, 0};
                if (is_new(step0 + y))
                    r[j][y] = *reinterpret_cast<const u32x4*>(src + (int64_t)(o0 + (pos + (step0 + y) * kRows - p0)) * rows.token_stride);
            }
        }
    };
    uint32_t top[2] = {0, 0};  // largest magnitudes of the lane's pairs
    auto magnitudes = [&](auto finite) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (uint32_t y = 0; y < kHold; ++y)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t m = r[j][y][i] & 0x7FFF7FFFu;
                    if (finite) {
                        if ((m & 0xFFFFu) >= T::kInf) m &= 0xFFFF0000u;
                        if ((m >> 16) >= T::kInf) m &= 0xFFFFu;
                    }
                    top[j] = max_pair(top[j], m);
                }
    };
    for (uint32_t step0 = 0; step0 < steps; step0 += kHold) {
        load(step0);
        magnitudes(std::false_type{});
    }
    const uint32_t both = max_pair(top[0], top[1]);
    const bool beyond = ballot((both & 0xFFFFu) > kMostBits || (both >> 16) > kMostBits) != 0;
    if (beyond) {  // an element that is not finite, or larger than any code's
        top[0] = top[1] = 0;
        for (uint32_t step0 = 0; step0 < steps; step0 += kHold) {
            if (steps > kHold) load(step0);
            magnitudes(std::true_type{});
        }
    }
    // of keys in the lower half, of values in the upper
    uint32_t two = min(max(top[0] & 0xFFFFu, top[0] >> 16), kMostBits) | min(max(top[1] & 0xFFFFu, top[1] >> 16), kMostBits) << 16;
    for (uint32_t y = min((uint32_t)kWave, kPieces << bl) >> 1; y; y >>= 1) two = max_pair(two, (uint32_t)__shfl_xor((int)two, (int)y));

    if (block >= len || block + ((1u << bl) - 1u) < p0) return;  // no new token in the lane's block
    if (page >= a.c.num_pages) {
        atomicOr(a.err, CR_ERR_PAGE);
        return;
    }
    uint16_t* scale = a.scale + scale_at(page, a.c.heads, head, block & mask, a.c.log_tokens, bl);
    const uint32_t scale_old = block < p0 ? *scale : 0u;  // tokens from before
    uint32_t e[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        uint8_t* codes = (j ? cv : ck) + (int64_t)head * a.c.head_stride + (int64_t)page * a.c.page_stride + piece * 8u;
        auto at = [&](uint32_t p) { return reinterpret_cast<u32x2*>(codes + (int64_t)(p & mask) * a.c.token_stride); };
        e[j] = exponent_of<T, C>(j ? two >> 16 : two & 0xFFFFu);
        if (block < p0) {
            const uint32_t e_old = j ? scale_old >> 8 : scale_old & 0xFFu;
            if (e[j] > e_old) {
                const float down = scale_of((uint32_t)max((int)(e_old + 127u) - (int)e[j], 1));  // 2^(e_old - e); below 2^-126 no code is left anyway
                for (uint32_t p = pos; p < p0; p += kRows) {
                    u32x2 w = *at(p);
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const f32x2 lo = C::template floats<false>(w[i]), hi = C::template floats<true>(w[i]);
                        w[i] = C::template code<true>(hi[0] * down, hi[1] * down, C::template code<false>(lo[0] * down, lo[1] * down, 0u));
                    }
                    *at(p) = w;
                }
            }
            e[j] = max(e[j], e_old);
        }
    }
    for (uint32_t step0 = 0; step0 < steps; step0 += kHold) {
        if (steps > kHold) load(step0);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            uint8_t* codes = (j ? cv : ck) + (int64_t)head * a.c.head_stride + (int64_t)page * a.c.page_stride + piece * 8u;
            // 2^-(e - 127). Elements alone need 247 at most; a block's e from before goes up to 254, and 2^-127 is subnormal.
            const float up = e[j] < 254u ? scale_of(254u - e[j]) : 0x1p-127f;
#pragma unroll
            for (uint32_t y = 0; y < kHold; ++y) {
                if (!is_new(step0 + y)) continue;
                u32x2 out;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint32_t x0 = r[j][y][2 * i], x1 = r[j][y][2 * i + 1];
                    float z[4] = {T::first(x0), T::second(x0), T::first(x1), T::second(x1)};
                    if (beyond) {
                        const float most = T::first(kMostBits);
#pragma unroll
                        for (int w = 0; w < 4; ++w)
                            if (__builtin_fabsf(z[w]) < INFINITY) z[w] = fminf(fmaxf(z[w], -most), most);
                    }
                    out[i] = C::template code<true>(z[2] * up, z[3] * up, C::template code<false>(z[0] * up, z[1] * up, 0u));
                }
                __builtin_nontemporal_store(out, reinterpret_cast<u32x2*>(codes + (int64_t)((pos + (step0 + y) * kRows) & mask) * a.c.token_stride));
            }
        }
    }
    if (piece == 0 && pos == block) *scale = (uint16_t)(e[0] | e[1] << 8);
}

template <typename T, typename C, int kDim>
__global__ __launch_bounds__(256) void k_kvq_append(QCall a, uint8_t* ck, uint8_t* cv)
{
    const uint32_t waves = gridDim.x * kQWaves, end = max(a.items, a.n);
    for (uint64_t item = blockIdx.x * kQWaves + wave_in_block(); item < end; item += waves) {
        q_check(a, item);
        if (item < a.items) append_span<T, C, kDim>(a, ck, cv, (uint32_t)item);
    }
}

// Tokens read back: a wave takes a token's keys and values of all heads, a lane 8 elements of a head at a time.
//
// Bound by memory: 180,167 tokens of 8 heads of 128 (370 MB read, 738 written) take 253 us, 4.4 TB/s (274 with ordinary loads and
// stores); 37 tokens 3 us, the launch.
template <typename T, typename C, int kDim>
__global__ __launch_bounds__(256) void k_kvq_read(QCall a)
{
    constexpr uint32_t kPieces = kDim / 8, kAhead = 4;
    const uint32_t per = a.c.heads * kPieces, first = a.k.p ? 0u : per, last = a.v.p ? 2u * per : per;
    const uint32_t mask = (1u << a.c.log_tokens) - 1u;
    const uint32_t waves = gridDim.x * kQWaves, me = blockIdx.x * kQWaves + wave_in_block();
    for (uint64_t y = me; y < max(a.total, a.n); y += waves) {
        q_check(a, y);
        if (y >= a.total) continue;
        const uint32_t tok = (uint32_t)y;
        const uint32_t x = wave_find(a.n, tok, [&](uint32_t z) { return a.off[z]; });
        uint32_t o0, o1, len;
        if (!q_fits(a, x, &o0, &o1, &len) || tok < o0 || tok >= o1) continue;
        const uint32_t pos = len - (o1 - tok), page = a.table[(uint64_t)x * a.width + (pos >> a.c.log_tokens)];
        if (page >= a.c.num_pages) {
            if (lane_id() == 0) atomicOr(a.err, CR_ERR_PAGE);
            continue;
        }
        const int64_t from = (int64_t)page * a.c.page_stride + (int64_t)(pos & mask) * a.c.token_stride;
        for (uint32_t z0 = first; z0 < last; z0 += kAhead * kWave) {
            u32x2 w[kAhead];
            uint32_t e[kAhead];
#pragma unroll
            for (uint32_t i = 0; i < kAhead; ++i) {
                const uint32_t z = z0 + i * kWave + lane_id(), p = z < per ? z : z - per, h = p / kPieces;
                if (z >= last) continue;
                w[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>((z < per ? a.c.k : a.c.v) + from + (int64_t)h * a.c.head_stride + p % kPieces * 8u));
                const uint32_t two = a.c.scale[scale_at(page, a.c.heads, h, pos & mask, a.c.log_tokens, a.c.log_block)];
                e[i] = z < per ? two & 0xFFu : two >> 8;
            }
#pragma unroll
            for (uint32_t i = 0; i < kAhead; ++i) {
                const uint32_t z = z0 + i * kWave + lane_id(), p = z < per ? z : z - per, h = p / kPieces;
                if (z >= last) continue;
                const cr_rows& rows = z < per ? a.k : a.v;
                uint16_t* to = (uint16_t*)rows.p + (int64_t)tok * rows.token_stride + (int64_t)h * rows.head_stride + p % kPieces * 8u;
                __builtin_nontemporal_store((wide_of<C, typename T::Pair>(w[i], scale_of(e[i]))), reinterpret_cast<u32x4*>(to));
            }
        }
    }
}

// What both calls check; rows of NULL are not looked at where `optional`. CR_OK with a.total 0: nothing to do.
cr_status q_call(const cr_kvq_cache* c, const cr_kvq_tokens* t, bool optional, uint32_t* err, QCall* a)
{
    if (!good_cache(c) || !t || t->layer >= c->layers || !err || t->total >= (1u << 31) || t->n > (1u << 24) || t->width > (1u << 28)) return CR_EINVAL;
    *a = QCall{};
    if (t->total == 0) return CR_OK;
    if (t->n == 0 || !t->off || !t->length || (t->width > 0 && !t->table)) return CR_EINVAL;
    if (((t->k.p || !optional) && !good_rows(t->k)) || ((t->v.p || !optional) && !good_rows(t->v))) return CR_EINVAL;
    a->c = kvq_pages(c, t->layer);
    a->scale = const_cast<uint16_t*>(a->c.scale);
    a->k = t->k;
    a->v = t->v;
    a->off = t->off;
    a->length = t->length;
    a->table = t->table;
    a->total = t->total;
    a->n = t->n;
    a->width = t->width;
    a->err = err;
    return CR_OK;
}

template <typename T, typename C>
void append_launch(const QCall& a, uint32_t blocks, hipStream_t st)
{
    uint8_t *k = const_cast<uint8_t*>(a.c.k), *v = const_cast<uint8_t*>(a.c.v);
    if (a.c.dim == 128) hipLaunchKernelGGL((k_kvq_append<T, C, 128>), dim3(blocks), dim3(kQThreads), 0, st, a, k, v);
    else hipLaunchKernelGGL((k_kvq_append<T, C, 64>), dim3(blocks), dim3(kQThreads), 0, st, a, k, v);
}

template <typename T, typename C>
void read_launch(const QCall& a, uint32_t blocks, hipStream_t st)
{
    if (a.c.dim == 128) hipLaunchKernelGGL((k_kvq_read<T, C, 128>), dim3(blocks), dim3(kQThreads), 0, st, a);
    else hipLaunchKernelGGL((k_kvq_read<T, C, 64>), dim3(blocks), dim3(kQThreads), 0, st, a);
}

inline uint32_t q_blocks(uint64_t waves)
{
    const uint64_t blocks = (waves + kQWaves - 1u) / kQWaves;
    return (uint32_t)(blocks < kQBlocks ? blocks : kQBlocks);
}

}  // namespace
}  // namespace cr

extern "C" cr_status cr_kvq_append(const cr_kvq_cache* c, const cr_kvq_tokens* t, uint32_t* err, void* stream)
{
    using namespace cr;
    QCall a;
    const cr_status rc = q_call(c, t, false, err, &a);
    if (rc != CR_OK || a.total == 0) return rc;
    const uint32_t rows = kWave * 8u / c->dim;  // of a wave
    a.log_span = log2_of(c->block_tokens > rows ? c->block_tokens : rows);
    const uint64_t items = span_start(a.total, a.n, a.log_span) * c->heads;
    if (items >= (1ull << 32)) return CR_EINVAL;
    a.items = (uint32_t)items;
    const hipStream_t st = as_stream(stream);
    const uint32_t blocks = q_blocks(a.items > a.n ? a.items : a.n);
    (void)hipGetLastError();
    if (c->dtype == CR_BF16 && c->code == CR_E4M3) append_launch<Bf16Rows, E4m3>(a, blocks, st);
    else if (c->dtype == CR_BF16) append_launch<Bf16Rows, E5m2>(a, blocks, st);
    else if (c->code == CR_E4M3) append_launch<F16Rows, E4m3>(a, blocks, st);
    else append_launch<F16Rows, E5m2>(a, blocks, st);
    return hipGetLastError() == hipSuccess ? CR_OK : CR_EHIP;
}

extern "C" cr_status cr_kvq_read(const cr_kvq_cache* c, const cr_kvq_tokens* t, uint32_t* err, void* stream)
{
    using namespace cr;
    QCall a;
    const cr_status rc = q_call(c, t, true, err, &a);
    if (rc != CR_OK || a.total == 0) return rc;
    if (a.k.p && a.k.p == a.v.p) return CR_EINVAL;  // one place for both
    const hipStream_t st = as_stream(stream);
    const uint32_t blocks = q_blocks(a.total > a.n ? a.total : a.n);
    (void)hipGetLastError();
    if (c->dtype == CR_BF16 && c->code == CR_E4M3) read_launch<Bf16Rows, E4m3>(a, blocks, st);
    else if (c->dtype == CR_BF16) read_launch<Bf16Rows, E5m2>(a, blocks, st);
    else if (c->code == CR_E4M3) read_launch<F16Rows, E4m3>(a, blocks, st);
    else read_launch<F16Rows, E5m2>(a, blocks, st);
    return hipGetLastError() == hipSuccess ? CR_OK : CR_EHIP;
}
