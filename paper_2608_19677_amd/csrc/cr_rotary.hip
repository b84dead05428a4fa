// Rotary positions of packed queries and keys.
//
// Mathematics: pair (x1, x2) turns by the fraction t of a turn, x1' = m (x1 cos 2 pi t - x2 sin 2 pi t), x2' = m (x2 cos 2 pi t +
// x1 sin 2 pi t). t is positions[token] * freq / 2^64 modulo 1: an integer product modulo 2^64, exact for every position, of
// which the upper 32 bits are taken as a signed fraction (rounded to fp32: within 2^-26 of a turn, 0.94e-7 of a cosine). The hardware's sine and
// cosine take turns; on all multiples of 2^-24 they are within 1.26e-7: 2.2e-7 together, below 2^-22.
#include "cr_codes.h"

namespace cr {
namespace {

constexpr uint32_t kRotThreads = 256;
constexpr uint32_t kRotWaves = kRotThreads / kWave;
constexpr uint32_t kRotBlocks = 1u << 20;  // of a launch; waves take more work in turn

struct Rot {
    cr_rows q, k, q_out, k_out;
    const int32_t* positions;
    const uint64_t* freq;
    uint32_t heads_q, heads, rotated, pairs;  // heads: of queries and keys; pairs: layout
    uint32_t total, steps;                    // steps: waves that share a token's heads
    uint32_t in_place_q, in_place_k;
    float magnitude;
};

// Pair (x, z) turned, as a pair of elements.
template <typename T>
__device__ __forceinline__ uint32_t turned(float x, float z, float c, float s)
{
    return pack_pair<T>(__builtin_fmaf(x, c, -(z * s)), __builtin_fmaf(z, c, x * s));
}

// A wave takes 8 (dim 128) or 16 (dim 64) heads of a token; a lane two pieces of 8 elements of a head: 8 pairs, or 16
// elements that are only copied. Cosines and sines are computed again for every such step of heads: what else the vector units have
// to do is little, and waves that take several steps one after the other are slower.
//
// Bound by memory: 16,384 tokens of 64 heads and 8 key heads of 128 (604 MB read and written) take 104 us, 5.8 TB/s (124 with ordinary
// loads and stores and a quarter of the waves: what is written is not kept in the cache's way); a token by the launch, 3 us.
template <typename T, int kDim>
__global__ __launch_bounds__(256) void k_rotary(const Rot a)
{
    constexpr uint32_t kLanes = kDim / 16, kHeads = kWave / kLanes;  // lanes of a head, heads of a step
    const uint32_t lane = lane_id(), y = lane % kLanes, head0 = lane / kLanes;
    const bool turns = y < a.rotated / 16u;
    const uint32_t ea = turns && !a.pairs ? y * 8u : y * 16u, eb = turns && !a.pairs ? ea + a.rotated / 2u : ea + 8u;
    const uint64_t waves = (uint64_t)gridDim.x * kRotWaves, items = (uint64_t)a.total * a.steps;
    for (uint64_t item = (uint64_t)blockIdx.x * kRotWaves + wave_in_block(); item < items; item += waves) {
        const uint32_t tok = (uint32_t)(item / a.steps), h = (uint32_t)(item % a.steps) * kHeads + head0;
        if (h >= a.heads) continue;
        const bool is_q = h < a.heads_q;
        if (!turns && (is_q ? a.in_place_q : a.in_place_k)) continue;
        const uint32_t hh = is_q ? h : h - a.heads_q;
        const cr_rows &in = is_q ? a.q : a.k, &to = is_q ? a.q_out : a.k_out;
        const uint16_t* from = (const uint16_t*)in.p + (int64_t)tok * in.token_stride + (int64_t)hh * in.head_stride;
        uint16_t* out = (uint16_t*)to.p + (int64_t)tok * to.token_stride + (int64_t)hh * to.head_stride;
        u32x4 ra = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(from + ea)), rb = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(from + eb));
        if (turns) {
            const uint64_t pos = (uint64_t)(int64_t)a.positions[tok];
            float c[8], s[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float t = (float)(int32_t)((pos * a.freq[y * 8u + i]) >> 32) * 0x1p-32f;
                c[i] = __builtin_amdgcn_cosf(t) * a.magnitude;
                s[i] = __builtin_amdgcn_sinf(t) * a.magnitude;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (a.pairs) {
                    ra[i] = turned<T>(T::first(ra[i]), T::second(ra[i]), c[i], s[i]);
                    rb[i] = turned<T>(T::first(rb[i]), T::second(rb[i]), c[4 + i], s[4 + i]);
                } else {
                    const float x[2] = {T::first(ra[i]), T::second(ra[i])}, z[2] = {T::first(rb[i]), T::second(rb[i])};
                    const float c0 = c[2 * i], s0 = s[2 * i], c1 = c[2 * i + 1], s1 = s[2 * i + 1];
                    ra[i] = pack_pair<T>(__builtin_fmaf(x[0], c0, -(z[0] * s0)), __builtin_fmaf(x[1], c1, -(z[1] * s1)));
                    rb[i] = pack_pair<T>(__builtin_fmaf(z[0], c0, x[0] * s0), __builtin_fmaf(z[1], c1, x[1] * s1));
                }
            }
        }
        __builtin_nontemporal_store(ra, reinterpret_cast<u32x4*>(out + ea));
        __builtin_nontemporal_store(rb, reinterpret_cast<u32x4*>(out + eb));
    }
}

template <typename T>
void rotary_launch(const Rot& a, uint32_t dim, uint32_t blocks, hipStream_t st)
{
    if (dim == 128) hipLaunchKernelGGL((k_rotary<T, 128>), dim3(blocks), dim3(kRotThreads), 0, st, a);
    else hipLaunchKernelGGL((k_rotary<T, 64>), dim3(blocks), dim3(kRotThreads), 0, st, a);
}

inline bool same_rows(const cr_rows& x, const cr_rows& y, uint32_t tokens, uint32_t heads)
{
    return x.p == y.p && (tokens == 1 || x.token_stride == y.token_stride) && (heads == 1 || x.head_stride == y.head_stride);
}

}  // namespace
}  // namespace cr

extern "C" cr_status cr_rotary(const cr_rotary_args* p, void* stream)
{
    using namespace cr;
    if (!p || p->dtype > CR_F16 || p->heads_q < 1 || p->heads_q > CR_MAX_HEADS || p->heads_k > CR_MAX_HEADS || (p->dim != 64 && p->dim != 128) ||
        p->rotated < 16 || p->rotated > p->dim || p->rotated % 16 != 0 || p->layout > CR_ROTARY_PAIRS ||
        !(__builtin_fabsf(p->magnitude) <= 3.4e38f) || (uint64_t)p->total * (p->heads_q + p->heads_k) >= (1ull << 31))
        return CR_EINVAL;
    if (p->total == 0) return CR_OK;
    if (!good_rows(p->q) || !good_rows(p->q_out) || (p->heads_k && (!good_rows(p->k) || !good_rows(p->k_out))) || !p->positions ||
        !aligned4(p->positions) || !p->freq || ((uintptr_t)p->freq & 7u) != 0)
        return CR_EINVAL;
    Rot a{p->q, p->k, p->q_out, p->k_out, p->positions, p->freq, p->heads_q, p->heads_q + p->heads_k, p->rotated, p->layout, p->total, 1,
          same_rows(p->q, p->q_out, p->total, p->heads_q), p->heads_k && same_rows(p->k, p->k_out, p->total, p->heads_k), p->magnitude};
    if ((p->q.p == p->q_out.p && !a.in_place_q) || (p->heads_k && p->k.p == p->k_out.p && !a.in_place_k)) return CR_EINVAL;  // over itself
    if (p->heads_k && (p->q_out.p == p->k_out.p || p->q_out.p == p->k.p || p->k_out.p == p->q.p)) return CR_EINVAL;  // over the other
    const uint32_t heads = kWave * 16u / p->dim;  // of a wave
    a.steps = (a.heads + heads - 1u) / heads;
    const uint64_t need = ((uint64_t)a.total * a.steps + kRotWaves - 1u) / kRotWaves;
    const uint32_t blocks = (uint32_t)(need < kRotBlocks ? need : kRotBlocks);
    const hipStream_t st = as_stream(stream);
    (void)hipGetLastError();
    if (p->dtype == CR_BF16) rotary_launch<Bf16Rows>(a, p->dim, blocks, st);
    else rotary_launch<F16Rows>(a, p->dim, blocks, st);
    return hipGetLastError() == hipSuccess ? CR_OK : CR_EHIP;
}
