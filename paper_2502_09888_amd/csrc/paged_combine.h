// The join of the parts of the keys, for the launches that do it (internal).
#pragma once
#include "paged.h"

namespace climber {
namespace paged_join {

typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4;

static __device__ __forceinline__ void store4(float *p, f32x4 x) { *(f32x4 *)p = x; }
static __device__ __forceinline__ void store4(__bf16 *p, f32x4 x)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = (__bf16)x[i];
}

// Partial results of the parts of the keys, joined.  32 lanes have a row's dimensions; GROUPS such groups share its parts, and 8 / GROUPS
// rows x heads are a workgroup's (64 parts of 32 rows x heads: 65 us with a wave for each, which takes one part after the other, 5 with 8 groups).
// A launch as short as this is bound by its trips to memory: whatever a thread can need is requested at once, before it is known to be needed.
// (block: the workgroup's number among those that join)
template <typename E, int GROUPS>
static __device__ __forceinline__ void combine_rows(const PagedArgs &p, unsigned block)
{
    constexpr int kFirst = GROUPS > 1 ? 8 : 4;  // parts of a group requested at once
    __shared__ f32x4 sums[8][32];
    const int lane = threadIdx.x & 31, group = threadIdx.x >> 5, g = group % GROUPS, c = lane * 4;
    const int64_t all = (int64_t)p.m_total * p.H, rh = (int64_t)block * (8 / GROUPS) + group / GROUPS, row = rh / p.H;
    const int h = (int)(rh % p.H);
    float M = -INFINITY, L = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    if (rh < all) {
        auto part = [&](int i) { return *(const float2 *)(p.part_ml + (i * all + rh) * 2); };
        auto sum = [&](int i) { return c < p.d ? *(const f32x4 *)(p.part_o + (i * all + rh) * p.d + c) : f32x4{0.f, 0.f, 0.f, 0.f}; };
        f32x4 x[kFirst];
        float2 ml[kFirst];
#pragma unroll
        for (int k = 0; k < kFirst; ++k)
            if (g + k * GROUPS < p.n_split) {
                ml[k] = part(g + k * GROUPS);
                x[k] = sum(g + k * GROUPS);
            }
        for (int i = lane; i < p.n_split; i += 32) {
            const float2 y = part(i);
            if (y.y != 0.f) M = fmaxf(M, y.x);  // (0: no key of the part is seen)
        }
#pragma unroll
        for (int o = 1; o < 32; o *= 2) M = fmaxf(M, __shfl_xor(M, o, 64));
        for (int i = lane; i < p.n_split; i += 32) {
            const float2 y = part(i);
            if (y.y != 0.f) L += y.y * __builtin_amdgcn_exp2f(y.x - M);
        }
#pragma unroll
        for (int o = 1; o < 32; o *= 2) L += __shfl_xor(L, o, 64);
        // A part's mean, no larger than its values, by its share of all weights: the parts' sums may pass the largest number together.
        const float inv = 1.f / L;
        auto add = [&](float2 y, f32x4 o) {
            if (y.y != 0.f) {
                const float share = y.y * __builtin_amdgcn_exp2f(y.x - M) * inv, mean = 1.f / y.y;
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[e] += share * (o[e] * mean);
            }
        };
        if (L == 0.f) acc[0] = acc[1] = acc[2] = acc[3] = NAN;  // (all logits -inf)
#pragma unroll
        for (int k = 0; k < kFirst; ++k)
            if (g + k * GROUPS < p.n_split) add(ml[k], x[k]);
#pragma unroll 4
        for (int i = g + kFirst * GROUPS; i < p.n_split; i += GROUPS) add(part(i), sum(i));
    }
    const bool mine = rh < all && row >= max(p.off[0], 0) && row < p.off[p.n_seqs];  // a row of no sequence stays as it is
    if constexpr (GROUPS > 1) {
        sums[group][lane] = acc;
        __syncthreads();
        if (g != 0) return;
#pragma unroll
        for (int i = 1; i < GROUPS; ++i) acc += sums[group + i][lane];
    }
    if (!mine) return;
    if (c < p.d) store4((E *)(p.o + row * p.ld_o) + (int64_t)h * p.d + c, acc);
    if (lane == 0 && p.lse) p.lse[rh] = float2{paged_row_scale(p, row), M + __builtin_amdgcn_logf(L)};
}

}  // namespace paged_join
}  // namespace climber
