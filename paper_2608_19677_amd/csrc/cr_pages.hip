// Pages of a destination's key/value cache: taking, sharing, freeing, moving and copying them, and
// writing new tokens into them. The only state is refs (how many table entries name a page), so
// every result is a function of the inputs: free pages are ranked by id, counts change by integer
// atomics, whose order does not show.
#include "cr_kv.h"

namespace cr {
namespace {

constexpr uint32_t kPgThreads = 256;
constexpr uint32_t kPgPer = 16;                      // pages per thread of a scan
constexpr uint32_t kPgChunk = kPgThreads * kPgPer;   // pages per block
constexpr uint32_t kCopyThreads = 256;

// Workspace: free pages per chunk [chunks], pages live, pages that move, then the first page of each
// sequence in the order of taking [n + 1] and the page its tail is copied from [n] (extend, fork) or, for
// compact, holes, pages by live rank and live rank by page [3][num_pages].
struct PgWs {
    uint32_t* free_in;
    uint32_t* live;
    uint32_t* moves;
    uint32_t* first;
    uint32_t* from;
    uint32_t* holes;
    uint32_t* by_rank;
    uint32_t* rank;
};

inline uint32_t pg_chunks(uint32_t num_pages) { return (num_pages + kPgChunk - 1) / kPgChunk; }

inline PgWs pg_ws(void* ws, uint32_t num_pages, uint32_t n)
{
    PgWs w;
    w.free_in = reinterpret_cast<uint32_t*>(ws);
    w.live = w.free_in + pg_chunks(num_pages);
    w.moves = w.live + 1;
    w.first = w.moves + 1;
    w.from = w.first + n + 1;
    w.holes = w.moves + 1;
    w.by_rank = w.holes + num_pages;
    w.rank = w.by_rank + num_pages;
    return w;
}

// The sequences of cr_pages_extend (parent NULL) and cr_pages_fork.
struct PgTake {
    const uint32_t* len_old;  // extend
    const uint32_t* len_new;
    const uint32_t* parent;   // fork
    const uint32_t* length;
    const uint32_t* table;    // fork: the parents'
    uint32_t* out;            // extend: the table; fork: the children's
    uint32_t n, rows, width, out_width, log_tokens, num_pages;
};

// Pages that sequence i takes; 0 and a bit of *bad if it does not fit.
__device__ __forceinline__ uint32_t pg_need(const PgTake& t, uint32_t i, uint32_t* bad)
{
    if (t.parent) {
        const uint32_t len = t.length[i], pages = pages_of(len, t.log_tokens);
        if (t.parent[i] >= t.rows || pages > t.width || pages > t.out_width) {
            *bad |= CR_ERR_SEQ;
            return 0u;
        }
        return (len & ((1u << t.log_tokens) - 1u)) != 0u;
    }
    const uint32_t a = pages_of(t.len_old ? t.len_old[i] : 0u, t.log_tokens), b = pages_of(t.len_new[i], t.log_tokens);
    if (a > b || b > t.out_width) {
        *bad |= CR_ERR_SEQ;
        return 0u;
    }
    return b - a;
}

// Free pages among this thread's kPgPer, as a bit mask (pages behind the end count as taken).
__device__ __forceinline__ uint32_t pg_free_mask(const uint32_t* __restrict__ refs, uint32_t num_pages, uint32_t p0)
{
    uint32_t m = 0;
#pragma unroll
    for (uint32_t x = 0; x < kPgPer; ++x)
        if (p0 + x < num_pages && refs[p0 + x] == 0u) m |= 1u << x;
    return m;
}

// Free pages in all chunks, and in those before this block's.
__device__ __forceinline__ void pg_sums(const uint32_t* __restrict__ free_in, uint32_t chunks, uint32_t* sh, uint32_t* before,
                                        uint32_t* all)
{
    uint32_t b = 0, a = 0;
    for (uint32_t c = threadIdx.x; c < chunks; c += kPgThreads) {
        const uint32_t f = free_in[c];
        a += f;
        b += c < blockIdx.x ? f : 0u;
    }
    block_exscan_u32(a, sh, all);
    block_exscan_u32(b, sh, before);
}

// Blocks 0 .. chunks-1: free pages of each chunk. Block `chunks`: exclusive prefix of the sequences'
// needs. Blocks behind: a child's row each, its parent's full pages and CR_NO_PAGE behind them, and the page
// its tail is copied from. Counts are as they were before the call here only: pages taken later look live.
__global__ __launch_bounds__(256) void k_pages_count(const uint32_t* __restrict__ refs, uint32_t chunks, PgWs w, PgTake t,
                                                     uint32_t* __restrict__ err)
{
    __shared__ uint32_t sh[16];
    uint32_t tot, bad = 0;
    if (blockIdx.x < chunks) {
        const uint32_t m = pg_free_mask(refs, t.num_pages, blockIdx.x * kPgChunk + threadIdx.x * kPgPer);
        block_exscan_u32((uint32_t)__popc(m), sh, &tot);
        if (threadIdx.x == 0) w.free_in[blockIdx.x] = tot;
    } else if (blockIdx.x == chunks) {
        uint32_t base = 0;
        for (uint32_t i0 = 0; i0 < t.n; i0 += kPgThreads) {
            const uint32_t i = i0 + threadIdx.x;
            const uint32_t need = i < t.n ? pg_need(t, i, &bad) : 0u;
            const uint32_t pre = block_exscan_u32(need, sh, &tot);
            if (i < t.n) w.first[i] = base + pre;
            base += tot;
        }
        if (threadIdx.x == 0) w.first[t.n] = base;
    } else {
        const uint32_t i = blockIdx.x - chunks - 1u;
        const uint32_t p = t.parent[i], len = t.length[i], pages = pages_of(len, t.log_tokens), full = len >> t.log_tokens;
        const bool fits = p < t.rows && pages <= t.width && pages <= t.out_width;
        if (threadIdx.x == 0 && !(fits && full < pages)) w.from[i] = CR_NO_PAGE;  // no tail
        for (uint32_t j = threadIdx.x; j < t.out_width; j += kPgThreads) {
            uint32_t g = CR_NO_PAGE;
            if (fits && j < pages) {
                g = t.table[(uint64_t)p * t.width + j];
                if (g >= t.num_pages || refs[g] == 0u) {
                    bad |= CR_ERR_PAGE;
                    g = CR_NO_PAGE;
                }
            }
            if (fits && j == full && full < pages) w.from[i] = g;
            t.out[(uint64_t)i * t.out_width + j] = j < full ? g : CR_NO_PAGE;
        }
    }
    if (bad) atomicOr(err, bad);
}

// The sequence that takes the page of rank r: first[i] <= r < first[i + 1].
__device__ __forceinline__ uint32_t pg_taker(const uint32_t* first, uint32_t n, uint32_t r)
{
    uint32_t lo = 0, hi = n;
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) >> 1;
        if (first[mid] <= r) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Pages that its row has before those it takes.
__device__ __forceinline__ uint32_t pg_had(const PgTake& t, uint32_t i)
{
    return t.parent ? t.length[i] >> t.log_tokens : pages_of(t.len_old ? t.len_old[i] : 0u, t.log_tokens);
}

// Blocks 0 .. chunks-1 hand their chunk's free pages out by rank; for a fork, the blocks behind count
// a child's shared pages each.
__global__ __launch_bounds__(256) void k_pages_take(uint32_t* __restrict__ refs, uint32_t chunks, PgWs w, PgTake t,
                                                    uint32_t* __restrict__ err)
{
    __shared__ uint32_t sh[16];
    uint32_t before, all;
    pg_sums(w.free_in, chunks, sh, &before, &all);
    const uint32_t want = w.first[t.n];
    const bool short_of = want > all;
    if (blockIdx.x >= chunks) {
        const uint32_t i = blockIdx.x - chunks, full = min(t.length[i] >> t.log_tokens, t.out_width);
        for (uint32_t j = threadIdx.x; j < full; j += kPgThreads) {
            uint32_t* e = &t.out[(uint64_t)i * t.out_width + j];
            if (short_of) *e = CR_NO_PAGE;
            else if (*e != CR_NO_PAGE) atomicAdd(&refs[*e], 1u);
        }
        return;
    }
    if (short_of) {
        if (blockIdx.x == 0 && threadIdx.x == 0) atomicOr(err, CR_ERR_PAGES_OUT);
        return;
    }
    if (before >= want) return;
    const uint32_t p0 = blockIdx.x * kPgChunk + threadIdx.x * kPgPer;
    uint32_t m = pg_free_mask(refs, t.num_pages, p0), tot;
    uint32_t r = before + block_exscan_u32((uint32_t)__popc(m), sh, &tot);
    for (; m && r < want; ++r, m &= m - 1u) {
        const uint32_t p = p0 + (uint32_t)__builtin_ctz(m), i = pg_taker(w.first, t.n, r);
        t.out[(uint64_t)i * t.out_width + pg_had(t, i) + (r - w.first[i])] = p;
        refs[p] = 1u;
    }
}

// A page in 16-byte pieces: rows of dim elements at the cache's strides.
struct PgGeom {
    uint32_t row16;     // 16-byte pieces per (head, token) row
    uint32_t page16;    // pieces per page and layer
    uint32_t heads, log_tokens;
    uint32_t whole;     // 1: a page is one run of page16 pieces in memory
    int64_t head_stride, token_stride;
};

// Rows of `dim` elements of 2 bytes; codes go by pairs.
inline PgGeom pg_geom(uint32_t heads, uint32_t page_tokens, uint32_t dim, int64_t head_stride, int64_t token_stride)
{
    PgGeom g;
    g.row16 = dim / 8u;
    g.heads = heads;
    g.log_tokens = log2_of(page_tokens);
    g.page16 = (heads * g.row16) << g.log_tokens;
    g.head_stride = head_stride;
    g.token_stride = token_stride;
    const int64_t d = dim, pt = page_tokens, h = heads;
    g.whole = (token_stride == d && head_stride == d * pt) || (head_stride == d && token_stride == d * h);
    return g;
}

// Where the pages' contents lie: keys and values, and the pairs of scales of a cache held in 8 bits.
struct PgPlanes {
    uint16_t* k;
    uint16_t* v;
    int64_t layer_stride, page_stride;
    PgGeom g;
    uint32_t planes;
    uint32_t log_block, scale_page;  // tokens per scale; pairs per page and layer
    uint16_t* scale;                 // NULL: 16-bit elements
    uint64_t scale_layer;
};

inline PgPlanes pg_planes(const cr_kv_cache* c)
{
    return PgPlanes{(uint16_t*)c->k, (uint16_t*)c->v, c->layer_stride, c->page_stride,
                    pg_geom(c->heads, c->page_tokens, c->dim, c->head_stride, c->token_stride), 2u * c->layers, 0, 0, nullptr, 0};
}

inline PgPlanes pg_planes(const cr_kvq_cache* c)
{
    return PgPlanes{(uint16_t*)c->k, (uint16_t*)c->v, c->layer_stride / 2, c->page_stride / 2,
                    pg_geom(c->heads, c->page_tokens, c->dim / 2u, c->head_stride / 2, c->token_stride / 2), 2u * c->layers,
                    log2_of(c->block_tokens), scales_of_page(c), (uint16_t*)c->scale, scales_of_layer(c)};
}

// Offset in elements of piece x of a page.
__device__ __forceinline__ int64_t pg_piece(const PgGeom& g, uint32_t x)
{
    if (g.whole) return (int64_t)x * 8;
    const uint32_t row = x / g.row16, tok = row & ((1u << g.log_tokens) - 1u), head = row >> g.log_tokens;
    return (int64_t)head * g.head_stride + (int64_t)tok * g.token_stride + (int64_t)(x % g.row16) * 8;
}

// A fork's tail: the tokens behind a child's full pages in one plane (keys or values of a layer), copied from page
// src to page dst by `movers` threads. Bound by memory: 192 children's tails of 32 layers (336 MB read, from cache where children
// share a parent, and 336 MB written) take 110 us.
__device__ __forceinline__ void pg_copy_tail(const PgPlanes& c, uint32_t src, uint32_t dst, uint32_t tail, uint32_t plane, uint32_t mover,
                                             uint32_t movers)
{
    const PgGeom& g = c.g;
    uint16_t* base = ((plane & 1u) ? c.v : c.k) + (int64_t)(plane >> 1) * c.layer_stride;
    const uint16_t* s = base + (int64_t)src * c.page_stride;
    uint16_t* d = base + (int64_t)dst * c.page_stride;
    const uint32_t per_head = tail * g.row16, all = per_head * g.heads;
    for (uint32_t x = mover; x < all; x += movers) {
        const uint32_t head = x / per_head, r = x % per_head;
        const int64_t at =
            (int64_t)head * g.head_stride + (int64_t)(r / g.row16) * g.token_stride + (int64_t)(r % g.row16) * 8;
        *reinterpret_cast<uint4*>(d + at) = *reinterpret_cast<const uint4*>(s + at);
    }
    if (!c.scale || (plane & 1u)) return;  // with the keys: the scales of the tail's blocks
    const uint32_t blocks = ((tail - 1u) >> c.log_block) + 1u, per = 1u << (g.log_tokens - c.log_block);
    uint16_t* scale = c.scale + (uint64_t)(plane >> 1) * c.scale_layer;
    for (uint32_t x = mover; x < blocks * g.heads; x += movers) {
        const uint32_t at = x / blocks * per + x % blocks;
        scale[(uint64_t)dst * c.scale_page + at] = scale[(uint64_t)src * c.scale_page + at];
    }
}

__global__ __launch_bounds__(256) void k_pages_tail(PgPlanes c, PgWs w, PgTake t)
{
    for (uint64_t u = blockIdx.x; u < (uint64_t)t.n * c.planes; u += gridDim.x) {
        const uint32_t i = (uint32_t)(u / c.planes);
        const uint32_t src = w.from[i];
        if (src == CR_NO_PAGE) continue;  // no tail, or reported with the rows
        const uint32_t len = t.length[i];
        const uint32_t dst = t.out[(uint64_t)i * t.out_width + (len >> t.log_tokens)];
        if (dst == CR_NO_PAGE) continue;  // not served
        pg_copy_tail(c, src, dst, len & ((1u << t.log_tokens) - 1u), (uint32_t)(u % c.planes), threadIdx.x, kCopyThreads);
    }
}

// cr_pages_extend and cr_pages_fork of few sequences in one block, which holds the free pages among up to
// kOnePages in registers: three launches' work in one. Bound by its chain of dependent loads, so what the steps
// hand on stays in registers and LDS: four children of a 512-page cache forked and freed take 12.5 us a pass (13.0
// through global memory, 20 with the three launches). Every read of refs comes before the first write; pages that are shared and
// pages that are taken are different ones, as are the entries that name them.
constexpr uint32_t kOneThreads = 1024, kOnePages = kOneThreads * kPgPer;
// Sequences, a thread each; table entries of a fork; 16-byte pieces of the pages it may copy.
constexpr uint32_t kOneSeqs = kOneThreads, kOneEntries = 8 * kOneThreads, kOnePieces = 16384;

__global__ __launch_bounds__(1024) void k_pages_one(uint32_t* __restrict__ refs, PgTake t, PgPlanes c, uint32_t* __restrict__ err)
{
    __shared__ uint32_t sh[16], first[kOneSeqs + 1], had[kOneSeqs], from[kOneSeqs], to[kOneSeqs];
    uint32_t tot, want, bad = 0;
    const uint32_t p0 = threadIdx.x * kPgPer, me = threadIdx.x, mask = (1u << t.log_tokens) - 1u;
    uint32_t m = pg_free_mask(refs, t.num_pages, p0);
    const uint32_t need = me < t.n ? pg_need(t, me, &bad) : 0u;
    if (me < t.n) {
        had[me] = pg_had(t, me);
        from[me] = to[me] = CR_NO_PAGE;
    }
    const uint32_t pre = block_exscan_u32(need, sh, &want);
    if (me < t.n) first[me] = pre;
    if (me == 0) first[t.n] = want;
    uint32_t r = block_exscan_u32((uint32_t)__popc(m), sh, &tot);
    const bool short_of = want > tot;
    if (short_of) bad |= CR_ERR_PAGES_OUT;
    uint32_t shared[kOneEntries / kOneThreads];
#pragma unroll
    for (uint32_t y = 0; y < kOneEntries / kOneThreads; ++y) {
        shared[y] = CR_NO_PAGE;
        const uint32_t x = y * kOneThreads + me;
        if (!t.parent || x >= t.n * t.out_width) continue;
        const uint32_t i = x / t.out_width, j = x % t.out_width;
        const uint32_t p = t.parent[i], len = t.length[i], pages = pages_of(len, t.log_tokens), full = len >> t.log_tokens;
        uint32_t g = CR_NO_PAGE;
        if (p < t.rows && pages <= t.width && pages <= t.out_width && j < pages) {
            g = t.table[(uint64_t)p * t.width + j];
            if (g >= t.num_pages || refs[g] == 0u) {
                bad |= CR_ERR_PAGE;
                g = CR_NO_PAGE;
            }
            if (j == full) {  // the page of the tail: copied, and its entry the taken page's
                from[i] = g;
                if (!short_of) continue;
            }
        }
        if (j < full && !short_of) shared[y] = g;
        t.out[x] = shared[y];
    }
    if (bad) atomicOr(err, bad);
    if (short_of) return;
    __syncthreads();
#pragma unroll
    for (uint32_t y = 0; y < kOneEntries / kOneThreads; ++y)
        if (shared[y] != CR_NO_PAGE) atomicAdd(&refs[shared[y]], 1u);
    for (; m && r < want; ++r, m &= m - 1u) {
        const uint32_t p = p0 + (uint32_t)__builtin_ctz(m), i = pg_taker(first, t.n, r);
        t.out[(uint64_t)i * t.out_width + had[i] + (r - first[i])] = p;
        to[i] = p;  // a fork's child takes one
        refs[p] = 1u;
    }
    if (!t.parent) return;
    __syncthreads();
    // sixteen waves, a child's plane each
    for (uint32_t u = threadIdx.x >> 6; u < t.n * c.planes; u += kOneThreads / 64u) {
        const uint32_t i = u / c.planes, src = from[i], dst = to[i];
        if (src != CR_NO_PAGE && dst != CR_NO_PAGE) pg_copy_tail(c, src, dst, t.length[i] & mask, u % c.planes, lane_id(), 64u);
    }
}

__global__ __launch_bounds__(256) void k_pages_free(uint32_t* __restrict__ refs, uint32_t num_pages, uint32_t log_tokens,
                                                    const uint32_t* __restrict__ table, uint32_t width,
                                                    const uint32_t* __restrict__ length, uint32_t n, uint32_t* __restrict__ err)
{
    const uint64_t x = (uint64_t)blockIdx.x * kPgThreads + threadIdx.x;
    const uint32_t per = max(width, 1u);  // threads per row; one looks at the length where there are no entries
    if (x >= (uint64_t)n * per) return;
    const uint32_t i = (uint32_t)(x / per), j = (uint32_t)(x % per);
    const uint32_t pages = pages_of(length[i], log_tokens);
    if (pages > width) {
        if (j == 0) atomicOr(err, CR_ERR_SEQ);
        return;
    }
    if (j >= pages) return;
    const uint32_t g = table[x];
    if (g >= num_pages) {
        atomicOr(err, CR_ERR_PAGE);
        return;
    }
    // A decrement below 0 is put back. One fails only when as many have succeeded as the count
    // allows, so the final count does not depend on their order.
    if ((int32_t)atomicSub(&refs[g], 1u) <= 0) {
        atomicAdd(&refs[g], 1u);
        atomicOr(err, CR_ERR_PAGE);
    }
}

// Ranks for compaction. With L live pages: free pages below L in order of id go to holes[]; a live
// page's rank is the number of live pages before it, so those at or above L have the ranks from
// L - moves on. A free page's rank is CR_NO_PAGE. kCounted: the chunks' counts are there; else one block of
// kOneThreads counts all pages itself (up to kOnePages of them, a launch less).
template <bool kCounted>
__global__ __launch_bounds__(kCounted ? 256 : 1024) void k_pages_rank(const uint32_t* __restrict__ refs, uint32_t num_pages,
                                                                      uint32_t chunks, PgWs w)
{
    __shared__ uint32_t sh[16];
    uint32_t before = 0, all, tot;
    if (kCounted) pg_sums(w.free_in, chunks, sh, &before, &all);
    const uint32_t p0 = (kCounted ? blockIdx.x * kPgChunk : 0u) + threadIdx.x * kPgPer;
    const uint32_t m = pg_free_mask(refs, num_pages, p0);
    uint32_t f = before + block_exscan_u32((uint32_t)__popc(m), sh, &tot);  // free pages before p
    if (!kCounted) all = tot;
    const uint32_t live = num_pages - all;
    for (uint32_t x = 0; x < kPgPer && p0 + x < num_pages; ++x) {
        const uint32_t p = p0 + x;
        if (p == live) *w.moves = f;
        w.rank[p] = ((m >> x) & 1u) ? CR_NO_PAGE : p - f;
        if ((m >> x) & 1u) {
            if (p < live) w.holes[f] = p;
            ++f;
        } else {
            w.by_rank[p - f] = p;
        }
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        *w.live = live;
        if (live == num_pages) *w.moves = 0u;
    }
}

constexpr uint32_t kCopyPer = 4;                           // pieces per thread and unit
constexpr uint32_t kCopyUnit = kCopyThreads * kCopyPer;    // pieces per unit of a block

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// One unit of a page's contents, all loads before the stores; pieces behind the page repeat its last. Bound by
// memory: 1,500 pages of 128 KB (393 MB read and written) move in 69 to 78 us.
__device__ __forceinline__ void pg_copy_unit(const uint16_t* __restrict__ s, uint16_t* __restrict__ d, const PgGeom& g, uint32_t part)
{
    u32x4 r[kCopyPer];
    int64_t at[kCopyPer];
#pragma unroll
    for (uint32_t y = 0; y < kCopyPer; ++y) {
        at[y] = pg_piece(g, min(part * kCopyUnit + y * kCopyThreads + threadIdx.x, g.page16 - 1u));
        r[y] = *reinterpret_cast<const u32x4*>(s + at[y]);
    }
#pragma unroll
    for (uint32_t y = 0; y < kCopyPer; ++y) *reinterpret_cast<u32x4*>(d + at[y]) = r[y];
}

// Contents of pages: of the `moves` pages behind the live ones into the holes (w.holes set), or src
// to dst. A unit is one part of one plane (keys or values of a layer) of one page.
struct PgCopy {
    PgPlanes c;
    uint32_t parts, num_pages, n;
    const uint32_t* src;
    const uint32_t* dst;
};

// Part `part` of plane `plane` of page s copied to page d; the scales go with the keys' first part.
__device__ __forceinline__ void pg_copy_part(const PgPlanes& c, uint32_t s, uint32_t d, uint32_t plane, uint32_t part)
{
    uint16_t* base = ((plane & 1u) ? c.v : c.k) + (int64_t)(plane >> 1) * c.layer_stride;
    pg_copy_unit(base + (int64_t)s * c.page_stride, base + (int64_t)d * c.page_stride, c.g, part);
    if (!c.scale || part != 0u || (plane & 1u)) return;
    uint16_t* scale = c.scale + (uint64_t)(plane >> 1) * c.scale_layer;
    for (uint32_t x = threadIdx.x; x < c.scale_page; x += kCopyThreads)
        scale[(uint64_t)d * c.scale_page + x] = scale[(uint64_t)s * c.scale_page + x];
}

__global__ __launch_bounds__(256) void k_pages_copy(PgCopy c, uint32_t* __restrict__ err)
{
    const uint64_t units = (uint64_t)c.n * c.c.planes * c.parts;
    for (uint64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const uint32_t part = (uint32_t)(u % c.parts), plane = (uint32_t)(u / c.parts % c.c.planes);
        const uint32_t i = (uint32_t)(u / c.parts / c.c.planes);
        const uint32_t s = c.src[i], d = c.dst[i];
        if (s >= c.num_pages || d >= c.num_pages) {
            if (threadIdx.x == 0) atomicOr(err, CR_ERR_PAGE);
            continue;
        }
        pg_copy_part(c.c, s, d, plane, part);
    }
}

// Compaction, second part. The first `name_blocks` blocks write the new counts and rename the tables'
// entries; the others move contents.
__global__ __launch_bounds__(256) void k_pages_move(PgCopy c, PgWs w, uint32_t name_blocks, const uint32_t* refs,
                                                    uint32_t* refs_out, const uint32_t* table, uint32_t* table_out,
                                                    const uint32_t* __restrict__ length, uint32_t rows, uint32_t width,
                                                    uint32_t log_tokens, uint32_t* __restrict__ err)
{
    const uint32_t live = *w.live, moves = *w.moves, first = live - moves;
    if (blockIdx.x < name_blocks) {
        uint32_t bad = 0;
        const uint32_t x0 = blockIdx.x * kPgThreads + threadIdx.x, stride = name_blocks * kPgThreads;
        for (uint32_t p = x0; p < c.num_pages; p += stride) {
            // a page's count is read and written by its own thread, a hole's written by its mover's
            const uint32_t r = w.rank[p], count = refs[p];
            if (r != CR_NO_PAGE) refs_out[p < live ? p : w.holes[r - first]] = count;
            if (p >= live) refs_out[p] = 0u;
        }
        for (uint64_t x = x0; x < (uint64_t)rows * width; x += stride) {
            const uint32_t i = (uint32_t)(x / width), j = (uint32_t)(x % width);
            const uint32_t pages = pages_of(length[i], log_tokens);
            uint32_t g = table[x];
            if (pages > width) {
                bad |= CR_ERR_SEQ;
            } else if (j < pages) {
                const uint32_t r = g < c.num_pages ? w.rank[g] : CR_NO_PAGE;
                if (r == CR_NO_PAGE) bad |= CR_ERR_PAGE;
                else if (g >= live) g = w.holes[r - first];
            }
            table_out[x] = g;
        }
        if (width == 0u)  // no entries to go by
            for (uint32_t i = x0; i < rows; i += stride) bad |= length[i] ? CR_ERR_SEQ : 0u;
        if (bad) atomicOr(err, bad);
        return;
    }
    const uint64_t units = (uint64_t)moves * c.c.planes * c.parts;
    for (uint64_t u = blockIdx.x - name_blocks; u < units; u += gridDim.x - name_blocks) {
        const uint32_t part = (uint32_t)(u % c.parts), plane = (uint32_t)(u / c.parts % c.c.planes);
        const uint32_t i = (uint32_t)(u / c.parts / c.c.planes);
        const uint32_t s = w.by_rank[first + i], d = w.holes[i];
        pg_copy_part(c.c, s, d, plane, part);
    }
}

// New tokens: a block per token (of more than kAppendBlocks: in turn), a thread per 16 bytes of its keys
// and values.
constexpr uint32_t kAppendBlocks = 1u << 20;

__global__ __launch_bounds__(256) void k_kv_append(KvPages c, uint16_t* __restrict__ ck, uint16_t* __restrict__ cv, cr_rows k,
                                                   cr_rows v, uint32_t total, const uint32_t* __restrict__ off,
                                                   const uint32_t* __restrict__ length, uint32_t n,
                                                   const uint32_t* __restrict__ table, uint32_t width,
                                                   uint32_t* __restrict__ err)
{
    const uint32_t row16 = c.dim / 8u, per = c.heads * row16;
    for (uint32_t tok = blockIdx.x; tok < total; tok += gridDim.x) {
        const uint32_t i = wave_find(n, tok, [&](uint32_t x) { return off[x]; });
        const uint32_t o0 = off[i], o1 = off[i + 1], len = length[i];
        if (tok < o0 || tok >= o1 || o1 > total || o1 - o0 > len || pages_of(len, c.log_tokens) > width) {
            if (threadIdx.x == 0) atomicOr(err, CR_ERR_SEQ);
            continue;
        }
        const uint32_t pos = len - (o1 - tok), page = table[(uint64_t)i * width + (pos >> c.log_tokens)];
        if (page >= c.num_pages) {
            if (threadIdx.x == 0) atomicOr(err, CR_ERR_PAGE);
            continue;
        }
        const int64_t at = (int64_t)page * c.page_stride + (int64_t)(pos & ((1u << c.log_tokens) - 1u)) * c.token_stride;
        for (uint32_t x = threadIdx.x; x < 2u * per; x += kCopyThreads) {
            const uint32_t y = x < per ? x : x - per, h = y / row16, e = y % row16 * 8u;
            const cr_rows& r = x < per ? k : v;
            const uint16_t* s = (const uint16_t*)r.p + (int64_t)tok * r.token_stride + (int64_t)h * r.head_stride + e;
            *reinterpret_cast<uint4*>((x < per ? ck : cv) + at + (int64_t)h * c.head_stride + e) = *reinterpret_cast<const uint4*>(s);
        }
    }
}

template <typename C>
PgCopy pg_copy(const C* c)
{
    PgCopy m{};
    m.c = pg_planes(c);
    m.parts = (m.c.g.page16 + kCopyUnit - 1) / kCopyUnit;
    m.num_pages = c->num_pages;
    return m;
}

// The page calls, for a cache of either kind.
template <typename C>
cr_status pages_extend(const C* c, const uint32_t* len_old, const uint32_t* len_new, uint32_t n, uint32_t* table,
                       uint32_t width, void* ws, size_t ws_bytes, uint32_t* err, void* stream)
{
    if (!good_cache(c) || !c->refs || !err || !ws || !aligned4(ws) || (n > 0 && (!len_new || (width > 0 && !table))) ||
        n > (1u << 24) || width > (1u << 28))
        return CR_EINVAL;
    if ((uint64_t)n * width >= ((uint64_t)1 << 32)) return CR_EINVAL;  // pages that the sequences take are counted in 32 bits
    if (ws_bytes < cr_pages_workspace_bytes(c->num_pages, n)) return CR_ESIZE;
    if (n == 0) return CR_OK;
    const uint32_t chunks = pg_chunks(c->num_pages);
    const PgWs w = pg_ws(ws, c->num_pages, n);
    PgTake t{};
    t.len_old = len_old;
    t.len_new = len_new;
    t.out = table;
    t.n = n;
    t.out_width = width;
    t.log_tokens = log2_of(c->page_tokens);
    t.num_pages = c->num_pages;
    const hipStream_t st = as_stream(stream);
    (void)hipGetLastError();
    if (c->num_pages <= kOnePages && n <= kOneSeqs) {
        hipLaunchKernelGGL(k_pages_one, dim3(1), dim3(kOneThreads), 0, st, c->refs, t, PgPlanes{}, err);
    } else {
        hipLaunchKernelGGL(k_pages_count, dim3(chunks + 1), dim3(kPgThreads), 0, st, c->refs, chunks, w, t, err);
        hipLaunchKernelGGL(k_pages_take, dim3(chunks), dim3(kPgThreads), 0, st, c->refs, chunks, w, t, err);
    }
    return hipGetLastError() == hipSuccess ? CR_OK : CR_EHIP;
}

template <typename C>
cr_status pages_fork(const C* c, const uint32_t* table, uint32_t rows, uint32_t width, const uint32_t* parent,
                     const uint32_t* length, uint32_t n, uint32_t* child, uint32_t child_width, void* ws,
                     size_t ws_bytes, uint32_t* err, void* stream)
{
    if (!good_cache(c) || !c->refs || !err || !ws || !aligned4(ws) || n > (1u << 24) || width > (1u << 28) ||
        child_width > (1u << 28) ||
        (n > 0 && (!parent || !length || (rows > 0 && width > 0 && !table) || (child_width > 0 && !child) || child == table)))
        return CR_EINVAL;
    const uint32_t chunks = pg_chunks(c->num_pages);
    if ((uint64_t)chunks + 1u + n >= ((uint64_t)1 << 32) / kPgThreads) return CR_EINVAL;  // threads of a launch
    if (ws_bytes < cr_pages_workspace_bytes(c->num_pages, n)) return CR_ESIZE;
    if (n == 0) return CR_OK;
    const PgWs w = pg_ws(ws, c->num_pages, n);
    PgTake t{};
    t.parent = parent;
    t.length = length;
    t.table = table;
    t.out = child;
    t.n = n;
    t.rows = rows;
    t.width = width;
    t.out_width = child_width;
    t.log_tokens = log2_of(c->page_tokens);
    t.num_pages = c->num_pages;
    const hipStream_t st = as_stream(stream);
    (void)hipGetLastError();
    const PgPlanes planes = pg_planes(c);
    const uint64_t units = (uint64_t)n * planes.planes;
    if (c->num_pages <= kOnePages && n <= kOneSeqs && (uint64_t)n * child_width <= kOneEntries && units * planes.g.page16 <= kOnePieces) {
        hipLaunchKernelGGL(k_pages_one, dim3(1), dim3(kOneThreads), 0, st, c->refs, t, planes, err);
    } else {
        hipLaunchKernelGGL(k_pages_count, dim3(chunks + 1 + n), dim3(kPgThreads), 0, st, c->refs, chunks, w, t, err);
        hipLaunchKernelGGL(k_pages_take, dim3(chunks + n), dim3(kPgThreads), 0, st, c->refs, chunks, w, t, err);
        hipLaunchKernelGGL(k_pages_tail, dim3((uint32_t)(units < (1u << 20) ? units : (1u << 20))), dim3(kCopyThreads), 0, st, planes, w, t);
    }
    return hipGetLastError() == hipSuccess ? CR_OK : CR_EHIP;
}

template <typename C>
cr_status pages_free(const C* c, const uint32_t* table, uint32_t width, const uint32_t* length, uint32_t n,
                     uint32_t* err, void* stream)
{
    if (!good_cache(c) || !c->refs || !err || n > (1u << 24) || width > (1u << 28) || (n > 0 && (!length || (width > 0 && !table))))
        return CR_EINVAL;
    if ((uint64_t)n * (width ? width : 1u) >= ((uint64_t)1 << 32) - kPgThreads) return CR_EINVAL;  // threads of a launch
    if (n == 0) return CR_OK;
    const uint64_t threads = (uint64_t)n * (width ? width : 1u);
    (void)hipGetLastError();
    hipLaunchKernelGGL(k_pages_free, dim3((uint32_t)((threads + kPgThreads - 1) / kPgThreads)), dim3(kPgThreads), 0,
                       as_stream(stream), c->refs, c->num_pages, log2_of(c->page_tokens), table, width, length, n, err);
    return hipGetLastError() == hipSuccess ? CR_OK : CR_EHIP;
}

template <typename C>
cr_status pages_compact(const C* c, const uint32_t* table, const uint32_t* length, uint32_t rows, uint32_t width,
                        uint32_t* table_out, uint32_t* refs_out, void* ws, size_t ws_bytes, uint32_t* err, void* stream)
{
    if (!good_cache(c) || !c->refs || !refs_out || !err || !ws || !aligned4(ws) || rows > (1u << 24) || width > (1u << 28) ||
        (rows > 0 && (!length || (width > 0 && (!table || !table_out)))))
        return CR_EINVAL;
    if (ws_bytes < cr_pages_workspace_bytes(c->num_pages, 0)) return CR_ESIZE;
    const uint32_t chunks = pg_chunks(c->num_pages);
    const PgWs w = pg_ws(ws, c->num_pages, 0);
    PgTake t{};
    t.num_pages = c->num_pages;
    const PgCopy m = pg_copy(c);
    const uint64_t names = (uint64_t)rows * width > c->num_pages ? (uint64_t)rows * width : c->num_pages;
    const uint32_t cus = (uint32_t)device_cus();
    const uint64_t want = (names + kPgThreads - 1) / kPgThreads;
    const uint32_t name_blocks = (uint32_t)(want < cus ? want : cus);
    const uint64_t units = (uint64_t)(c->num_pages / 2u) * m.c.planes * m.parts;  // no more pages than that can move
    const uint32_t copy_blocks = (uint32_t)(units < 8u * cus ? (units ? units : 1u) : 8u * cus);
    const hipStream_t st = as_stream(stream);
    (void)hipGetLastError();
    if (c->num_pages <= kOnePages) {
        hipLaunchKernelGGL(k_pages_rank<false>, dim3(1), dim3(kOneThreads), 0, st, c->refs, c->num_pages, chunks, w);
    } else {
        hipLaunchKernelGGL(k_pages_count, dim3(chunks), dim3(kPgThreads), 0, st, c->refs, chunks, w, t, err);
        hipLaunchKernelGGL(k_pages_rank<true>, dim3(chunks), dim3(kPgThreads), 0, st, c->refs, c->num_pages, chunks, w);
    }
    hipLaunchKernelGGL(k_pages_move, dim3(name_blocks + copy_blocks), dim3(kPgThreads), 0, st, m, w, name_blocks, c->refs,
                       refs_out, table, table_out, length, rows, width, log2_of(c->page_tokens), err);
    return hipGetLastError() == hipSuccess ? CR_OK : CR_EHIP;
}

template <typename C>
cr_status pages_copy(const C* c, const uint32_t* src, const uint32_t* dst, uint32_t n, uint32_t* err, void* stream)
{
    if (!good_cache(c) || !err || (n > 0 && (!src || !dst)) || n > CR_MAX_PAGES) return CR_EINVAL;
    if (n == 0) return CR_OK;
    PgCopy m = pg_copy(c);
    m.n = n;
    m.src = src;
    m.dst = dst;
    const uint64_t units = (uint64_t)n * m.c.planes * m.parts, cap = 8u * (uint64_t)device_cus();
    (void)hipGetLastError();
    hipLaunchKernelGGL(k_pages_copy, dim3((uint32_t)(units < cap ? units : cap)), dim3(kCopyThreads), 0, as_stream(stream), m,
                       err);
    return hipGetLastError() == hipSuccess ? CR_OK : CR_EHIP;
}

}  // namespace
}  // namespace cr

extern "C" size_t cr_pages_workspace_bytes(uint32_t num_pages, uint32_t n)
{
    const size_t a = 2u * (size_t)n + 1u, b = 3u * (size_t)num_pages;
    return ((size_t)cr::pg_chunks(num_pages) + 2u + (a > b ? a : b)) * sizeof(uint32_t);
}

extern "C" cr_status cr_pages_extend(const cr_kv_cache* c, const uint32_t* len_old, const uint32_t* len_new, uint32_t n,
                                     uint32_t* table, uint32_t width, void* ws, size_t ws_bytes, uint32_t* err,
                                     void* stream)
{
    return cr::pages_extend(c, len_old, len_new, n, table, width, ws, ws_bytes, err, stream);
}

extern "C" cr_status cr_kvq_extend(const cr_kvq_cache* c, const uint32_t* len_old, const uint32_t* len_new, uint32_t n,
                                   uint32_t* table, uint32_t width, void* ws, size_t ws_bytes, uint32_t* err,
                                   void* stream)
{
    return cr::pages_extend(c, len_old, len_new, n, table, width, ws, ws_bytes, err, stream);
}

extern "C" cr_status cr_pages_fork(const cr_kv_cache* c, const uint32_t* table, uint32_t rows, uint32_t width,
                                   const uint32_t* parent, const uint32_t* length, uint32_t n, uint32_t* child,
                                   uint32_t child_width, void* ws, size_t ws_bytes, uint32_t* err, void* stream)
{
    return cr::pages_fork(c, table, rows, width, parent, length, n, child, child_width, ws, ws_bytes, err, stream);
}

extern "C" cr_status cr_kvq_fork(const cr_kvq_cache* c, const uint32_t* table, uint32_t rows, uint32_t width,
                                 const uint32_t* parent, const uint32_t* length, uint32_t n, uint32_t* child,
                                 uint32_t child_width, void* ws, size_t ws_bytes, uint32_t* err, void* stream)
{
    return cr::pages_fork(c, table, rows, width, parent, length, n, child, child_width, ws, ws_bytes, err, stream);
}

extern "C" cr_status cr_pages_free(const cr_kv_cache* c, const uint32_t* table, uint32_t width, const uint32_t* length,
                                   uint32_t n, uint32_t* err, void* stream)
{
    return cr::pages_free(c, table, width, length, n, err, stream);
}

extern "C" cr_status cr_kvq_free(const cr_kvq_cache* c, const uint32_t* table, uint32_t width, const uint32_t* length,
                                 uint32_t n, uint32_t* err, void* stream)
{
    return cr::pages_free(c, table, width, length, n, err, stream);
}

extern "C" cr_status cr_pages_compact(const cr_kv_cache* c, const uint32_t* table, const uint32_t* length,
                                      uint32_t rows, uint32_t width, uint32_t* table_out, uint32_t* refs_out, void* ws,
                                      size_t ws_bytes, uint32_t* err, void* stream)
{
    return cr::pages_compact(c, table, length, rows, width, table_out, refs_out, ws, ws_bytes, err, stream);
}

extern "C" cr_status cr_kvq_compact(const cr_kvq_cache* c, const uint32_t* table, const uint32_t* length, uint32_t rows,
                                    uint32_t width, uint32_t* table_out, uint32_t* refs_out, void* ws, size_t ws_bytes,
                                    uint32_t* err, void* stream)
{
    return cr::pages_compact(c, table, length, rows, width, table_out, refs_out, ws, ws_bytes, err, stream);
}

extern "C" cr_status cr_pages_copy(const cr_kv_cache* c, const uint32_t* src, const uint32_t* dst, uint32_t n,
                                   uint32_t* err, void* stream)
{
    return cr::pages_copy(c, src, dst, n, err, stream);
}

extern "C" cr_status cr_kvq_copy(const cr_kvq_cache* c, const uint32_t* src, const uint32_t* dst, uint32_t n,
                                 uint32_t* err, void* stream)
{
    return cr::pages_copy(c, src, dst, n, err, stream);
}

extern "C" cr_status cr_kv_append(const cr_kv_cache* c, uint32_t layer, const cr_rows* k, const cr_rows* v, uint32_t total,
                                  const uint32_t* off, const uint32_t* length, uint32_t n, const uint32_t* table,
                                  uint32_t width, uint32_t* err, void* stream)
{
    using namespace cr;
    if (!good_cache(c) || layer >= c->layers || !err || total >= (1u << 31) || n > (1u << 24) || width > (1u << 28))
        return CR_EINVAL;
    if (total == 0) return CR_OK;
    if (n == 0 || !k || !v || !good_rows(*k) || !good_rows(*v) || !off || !length || (width > 0 && !table)) return CR_EINVAL;
    KvPages p = kv_pages(c);
    const int64_t at = (int64_t)layer * c->layer_stride;
    (void)hipGetLastError();
    hipLaunchKernelGGL(k_kv_append, dim3(total < kAppendBlocks ? total : kAppendBlocks), dim3(kCopyThreads), 0, as_stream(stream), p, (uint16_t*)c->k + at,
                       (uint16_t*)c->v + at, *k, *v, total, off, length, n, table, width, err);
    return hipGetLastError() == hipSuccess ? CR_OK : CR_EHIP;
}
