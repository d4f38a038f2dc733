// Rotary positions of query and key rows (gfx950): pairs of a head's first rot_dims elements are turned by the angle position * frequency,
//   (a, b) -> scale (a cos - b sin, a sin + b cos),
// pairs being neighbours (interleaved) or an element and the one rot_dims / 2 behind it (halves).  inverse turns the other way, which is also the
// gradient (the transposed matrix).
//
// A position may be far, so the angle is made in 64 bits and its whole quarter turns are taken off there; what is left, at most an eighth of
// a turn, fits 32 bits, and the sine's and cosine's Taylor sums to the powers 9 and 10 are off by less than 2e-9 on it.  They are made once per row and pair
// and shared by all heads through LDS.  Bound by memory: every element is read and written once, 16 bytes a thread.
// 20000 rows of 40 heads of 128 in bf16 71 us (410 MB at 5.8 TB/s), 64 rows 5.9 (the host's call; 3.7 on the device).
#include "../../include/climber.h"

#include <algorithm>
#include <cmath>

#include "internal.h"
#include "paged_host.h"

namespace climber {
namespace {

struct RotaryArgs {
    const uint8_t *in[2];  // q, k
    uint8_t *out[2];
    int64_t ld_in[2], ld_out[2];  // bytes
    int heads[2];
    const double *freq;
    const int32_t *pos;
    float scale;
    int64_t m;
    int d, half, rows, inverse;  // rows: of a workgroup
};

constexpr int kMostHalf = 256, kTurns = 1024;  // sines and cosines of a workgroup

// cosine and sine of 2 pi turns, times scale
static __device__ __forceinline__ float2 turn(double turns, float scale, int inverse)
{
    const double quarters = turns * 4.0, whole = rint(quarters);
    const float y = (float)(quarters - whole) * 1.57079637f, z = y * y;
    const float s = y * fmaf(z, fmaf(z, fmaf(z, fmaf(z, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), 1.f);
    const float c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
    const int q = (int)(whole - 4.0 * floor(whole * 0.25));  // 0 .. 3
    float co = q & 1 ? s : c, si = q & 1 ? c : s;
    if (q == 1 || q == 2) co = -co;
    if (q >= 2) si = -si;
    return float2{co * scale, (inverse ? -si : si) * scale};
}

// N elements of type T, of whichever alignment that makes.  N: elements that travel together, 16 bytes where rows, heads and halves allow it.
template <typename T, int N>
struct alignas(sizeof(T) * N) Some {
    T x[N];
};

template <typename T, bool INTER, int N>
__global__ __launch_bounds__(256) void rotary_kernel(const RotaryArgs p)
{
    typedef Some<T, N> V;
    __shared__ float2 cs[kTurns];
    const int heads = p.heads[0] + p.heads[1], rot = 2 * p.half;
    // pieces of a head: of pairs, then of elements that stay
    const int pairs = (INTER && N > 1 ? rot : p.half) / N, rest = (p.d - rot) / N, pieces = pairs + rest;
    const int64_t groups = (p.m + p.rows - 1) / p.rows;
    for (int64_t g = blockIdx.x; g < groups; g += gridDim.x) {
        const int64_t row0 = g * p.rows;
        const int rows = (int)min((int64_t)p.rows, p.m - row0);
        __syncthreads();
        for (int i = threadIdx.x; i < rows * p.half; i += 256) {
            const int r = i / p.half, j = i - r * p.half;
            cs[i] = turn((double)p.pos[row0 + r] * p.freq[j] * 0.15915494309189535, p.scale, p.inverse);
        }
        __syncthreads();
        const int units = rows * heads * pieces;
        for (int u = threadIdx.x; u < units; u += 256) {
            const int rh = u / pieces, piece = u - rh * pieces, r = rh / heads, hh = rh - r * heads;
            const int which = hh >= p.heads[0], h = which ? hh - p.heads[0] : hh;
            const T *x = (const T *)(p.in[which] + (row0 + r) * p.ld_in[which]) + (int64_t)h * p.d;
            T *y = (T *)(p.out[which] + (row0 + r) * p.ld_out[which]) + (int64_t)h * p.d;
            const float2 *t = cs + r * p.half;
            if (piece >= pairs) {
                const int at = rot + (piece - pairs) * N;
                if (x != y) *(V *)(y + at) = *(const V *)(x + at);
            } else if constexpr (INTER && N > 1) {
                V v = *(const V *)(x + piece * N);
#pragma unroll
                for (int e = 0; e < N / 2; ++e) {
                    const float2 w = t[piece * (N / 2) + e];
                    const float a = (float)v.x[2 * e], b = (float)v.x[2 * e + 1];
                    v.x[2 * e] = (T)fmaf(a, w.x, -(b * w.y));
                    v.x[2 * e + 1] = (T)fmaf(a, w.y, b * w.x);
                }
                *(V *)(y + piece * N) = v;
            } else {
                // (neighbours of an odd alignment: one by one too)
                const int ia = INTER ? 2 * piece : piece * N, ib = INTER ? 2 * piece + 1 : piece * N + p.half;
                V v = *(const V *)(x + ia), z = *(const V *)(x + ib);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float2 w = t[piece * N + e];
                    const float a = (float)v.x[e], b = (float)z.x[e];
                    v.x[e] = (T)fmaf(a, w.x, -(b * w.y));
                    z.x[e] = (T)fmaf(a, w.y, b * w.x);
                }
                *(V *)(y + ia) = v;
                *(V *)(y + ib) = z;
            }
        }
    }
}

template <typename T, bool INTER>
hipError_t launch(RotaryArgs p, hipStream_t s)
{
    // the most elements that a place in any of the rows is a multiple of
    uint64_t odd = (uint64_t)(INTER ? 2 * p.half : p.half) * sizeof(T) | (uint64_t)p.d * sizeof(T) | 16;
    for (int i = 0; i < 2; ++i)
        if (p.heads[i]) odd |= (uint64_t)p.in[i] | (uint64_t)p.out[i] | (uint64_t)p.ld_in[i] | (uint64_t)p.ld_out[i];
    const int n = (int)((odd & -odd) / sizeof(T));
    // Rows of a workgroup: one where that has work for all of its threads, more of smaller ones where there are rows enough.  us with 1 / 2 / 4:
    // 20000 rows of 40 heads of 128 70.6 / 74.8 / 77.7, 5000 of 12 heads of 64 in fp32 9.5 / 8.9 / 8.5.
    const int64_t units = (int64_t)(p.heads[0] + p.heads[1]) * ((INTER && n > 1 ? 2 * p.half : p.half) / n + (p.d - 2 * p.half) / n);
    p.rows = units >= 256 ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(768 / units, kTurns / p.half), p.m / 1024));
    const int64_t groups = (p.m + p.rows - 1) / p.rows;
    const dim3 grid((unsigned)std::min<int64_t>(groups, 1 << 16));
    void (*kernel)(RotaryArgs) = rotary_kernel<T, INTER, 1>;
    if (n == 2) kernel = rotary_kernel<T, INTER, 2>;
    if (n == 4) kernel = rotary_kernel<T, INTER, 4>;
    if constexpr (sizeof(T) == 2)
        if (n == 8) kernel = rotary_kernel<T, INTER, 8>;
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, p);
    return hipGetLastError();
}

}  // namespace
}  // namespace climber

using namespace climber;
using namespace climber::paged_host;

extern "C" {

int climber_rotary_frequencies(int32_t rot_dims, double base, int32_t kind, double factor, double made_for, double fast, double slow, double *freq,
                               float *scale)
{
    if (rot_dims < 2 || rot_dims % 2 != 0 || rot_dims > 2 * kMostHalf) return CLIMBER_ERR_SHAPE;
    if (!freq || !scale) return CLIMBER_ERR_NULL;
    if (kind < CLIMBER_ROTARY_PLAIN || kind > CLIMBER_ROTARY_PARTS) return CLIMBER_ERR_UNSUPPORTED;
    if (!(base > 0) || !std::isfinite(base)) return CLIMBER_ERR_RANGE;
    if (kind != CLIMBER_ROTARY_PLAIN && (!(factor > 0) || !std::isfinite(factor))) return CLIMBER_ERR_RANGE;
    if (kind == CLIMBER_ROTARY_BASE && rot_dims == 2) return CLIMBER_ERR_SHAPE;
    if (kind == CLIMBER_ROTARY_PARTS && (!(made_for > 0) || !std::isfinite(made_for) || !(slow >= 0) || !(fast > slow) || !std::isfinite(fast)))
        return CLIMBER_ERR_RANGE;
    if (kind == CLIMBER_ROTARY_BASE) base *= std::pow(factor, (double)rot_dims / (rot_dims - 2));
    *scale = kind == CLIMBER_ROTARY_PARTS ? (float)(0.1 * std::log(factor) + 1.0) : 1.f;
    for (int i = 0; i < rot_dims / 2; ++i) {
        double f = std::pow(base, -2.0 * i / rot_dims);
        if (kind == CLIMBER_ROTARY_LINEAR) f /= factor;
        if (kind == CLIMBER_ROTARY_PARTS) {
            const double turns = made_for * f / 6.283185307179586, r = std::min(1.0, std::max(0.0, (turns - slow) / (fast - slow)));
            f = f * r + f / factor * (1.0 - r);
        }
        freq[i] = f;
    }
    return CLIMBER_OK;
}

int climber_rotary(const climber_config *cfg, const climber_rotary_plan *rot, const int32_t *pos, int64_t m, int32_t n_kv_heads, const void *q,
                   int64_t ld_q, const void *k, int64_t ld_k, void *q_out, int64_t ld_qo, void *k_out, int64_t ld_ko, void *stream)
{
    if (!cfg || !rot) return CLIMBER_ERR_NULL;
    if (cfg->dtype != CLIMBER_F32 && cfg->dtype != CLIMBER_BF16) return CLIMBER_ERR_UNSUPPORTED;
    if (cfg->n_heads < 1 || cfg->d_head < 1 || cfg->d_model != (int64_t)cfg->n_heads * cfg->d_head || n_kv_heads < 0 || m < 0) return CLIMBER_ERR_SHAPE;
    if (rot->rot_dims < 2 || rot->rot_dims % 2 != 0 || rot->rot_dims > cfg->d_head || !std::isfinite(rot->scale)) return CLIMBER_ERR_SHAPE;
    if (rot->rot_dims > 2 * kMostHalf) return CLIMBER_ERR_UNSUPPORTED;
    const int64_t elem = (int64_t)elem_of(cfg), wide = cfg->d_model, kv_wide = (int64_t)n_kv_heads * cfg->d_head, most = (int64_t)1 << 24;
    if (ld_q < wide || ld_qo < wide || (n_kv_heads > 0 && (ld_k < kv_wide || ld_ko < kv_wide))) return CLIMBER_ERR_SHAPE;
    if (ld_q > most || ld_qo > most || (n_kv_heads > 0 && (ld_k > most || ld_ko > most)) || wide + kv_wide > (int64_t)1 << 24 || m > (int64_t)1 << 31)
        return CLIMBER_ERR_RANGE;
    if (!rot->freq) return CLIMBER_ERR_NULL;
    if (!aligned(rot->freq, 8)) return CLIMBER_ERR_ALIGN;
    if (m == 0) return CLIMBER_OK;
    if (!pos || !q || !q_out || (n_kv_heads > 0 && (!k || !k_out))) return CLIMBER_ERR_NULL;
    if (!aligned(pos, 4) || !aligned(q, elem) || !aligned(q_out, elem) || (n_kv_heads > 0 && (!aligned(k, elem) || !aligned(k_out, elem))))
        return CLIMBER_ERR_ALIGN;
    // rows may be turned in place; otherwise nothing that is written is read or written elsewhere
    auto meet = [&](const void *a, int64_t la, int64_t wa, const void *b, int64_t lb, int64_t wb) {
        return overlap(a, la * elem, wa * elem, b, lb * elem, wb * elem, m);
    };
    if (meet(q_out, ld_qo, wide, q, ld_q, wide) && !(q_out == q && ld_qo == ld_q)) return CLIMBER_ERR_UNSUPPORTED;
    if (n_kv_heads > 0 && ((meet(k_out, ld_ko, kv_wide, k, ld_k, kv_wide) && !(k_out == k && ld_ko == ld_k)) || meet(q_out, ld_qo, wide, k, ld_k, kv_wide) ||
                           meet(k_out, ld_ko, kv_wide, q, ld_q, wide) || meet(q_out, ld_qo, wide, k_out, ld_ko, kv_wide)))
        return CLIMBER_ERR_UNSUPPORTED;
    RotaryArgs a{};
    a.in[0] = (const uint8_t *)q;
    a.in[1] = (const uint8_t *)k;
    a.out[0] = (uint8_t *)q_out;
    a.out[1] = (uint8_t *)k_out;
    a.ld_in[0] = ld_q * elem;
    a.ld_in[1] = ld_k * elem;
    a.ld_out[0] = ld_qo * elem;
    a.ld_out[1] = ld_ko * elem;
    a.heads[0] = cfg->n_heads;
    a.heads[1] = n_kv_heads;
    a.freq = rot->freq;
    a.pos = pos;
    a.scale = rot->scale;
    a.m = m;
    a.d = cfg->d_head;
    a.half = rot->rot_dims / 2;
    a.inverse = rot->inverse != 0;
    const hipStream_t s = (hipStream_t)stream;
    if (cfg->dtype == CLIMBER_BF16) return rt(rot->interleaved ? launch<__bf16, true>(a, s) : launch<__bf16, false>(a, s));
    return rt(rot->interleaved ? launch<float, true>(a, s) : launch<float, false>(a, s));
}

}  // extern "C"
