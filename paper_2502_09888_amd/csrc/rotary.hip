// Rotary positions of query and key rows (gfx950): pairs of a head's first rot_dims elements are turned by the angle position * frequency,
//   (a, b) -> scale (a cos - b sin, a sin + b cos),
// pairs being neighbours (interleaved) or an element and the one rot_dims / 2 behind it (halves).  inverse turns the other way, which is also the
// gradient (the transposed matrix).
//
// A position may be far, so the angle is made in 64 bits and its whole quarter turns are taken off there; what is left, at most an eighth of
// a turn, fits 32 bits, and the sine's and cosine's Taylor sums to the powers 9 and 10 are off by less than 2e-9 on it.  They are made once per row and pair
// and shared by all heads through LDS.  Bound by memory: every element is read and written once, 16 bytes a thread.
// 20000 rows of 40 heads of 128 in bf16 71 us (410 MB at 5.8 TB/s), 64 rows 5.4 (the host's call; 3.8 on the device).
#include "../../include/climber.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

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
    int d, half, rows, inverse, in_place;  // rows: of a workgroup
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

// 16 bytes, at any element: a head's halves may begin at an odd one.
typedef uint32_t Words2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t Words4 __attribute__((ext_vector_type(4), aligned(4)));
template <typename T>
struct Some {
    static constexpr int N = 16 / sizeof(T);
    typedef std::conditional_t<sizeof(T) == 2, Words2, Words4> Words;
    T x[N];
    __device__ __forceinline__ void load(const T *p) { *this = __builtin_bit_cast(Some, *(const Words *)p); }
    __device__ __forceinline__ void store(T *p) const { *(Words *)p = __builtin_bit_cast(Words, *this); }
};
template <typename T>
static __device__ __forceinline__ void turn_pair(T &a, T &b, float2 w)
{
    const float x = (float)a, y = (float)b;
    a = (T)fmaf(x, w.x, -(y * w.y));
    b = (T)fmaf(x, w.y, y * w.x);
}
// (an entry left out behind every eight: lanes that read eight each meet in different banks; 20000 rows of 40 heads of 64 in fp32, 32 of them turned, 86 / 75)
static __device__ __forceinline__ int in_lds(int i) { return i + (i >> 3); }

// A thread has 16 bytes of a head, and those that they are turned with.  EVEN: they divide what is turned, and the rest.  Otherwise the last ones
// overlap those before them, which is the same values twice; in place, where it would turn them twice, what is left over goes one by one.
// us with as many elements together as the alignment allows / this way: 6458 rows of 72 heads of 256, 114 of them turned in halves of 57, 351 / 101, in
// place 222 / 70.
struct Pieces {
    int pairs, singles, rest, stay;  // of a head: of pairs, pairs, of elements that stay, such elements
    int part, all;
};
template <int N, bool INTER, bool EVEN>
static __host__ __device__ __forceinline__ Pieces pieces_of(const RotaryArgs &p)
{
    Pieces x{};
    const int rest = p.d - 2 * p.half;
    x.part = INTER ? 2 * p.half : p.half;
    x.pairs = x.part / N, x.rest = rest / N;
    if (!EVEN) {
        const int left = x.part % N, stay = rest % N;
        if (left && x.pairs > 0 && !p.in_place) ++x.pairs;
        else x.singles = INTER ? left / 2 : left;
        if (stay && x.rest > 0) ++x.rest;
        else x.stay = stay;
    }
    x.all = x.pairs + x.singles + x.rest + x.stay;
    return x;
}
template <typename T, bool INTER, bool EVEN>
__global__ __launch_bounds__(256) void rotary_kernel(const RotaryArgs p)
{
    typedef Some<T> V;
    constexpr int N = V::N;
    __shared__ float2 cs[kTurns + kTurns / 8];
    const int heads = p.heads[0] + p.heads[1], rot = 2 * p.half;
    const Pieces n = pieces_of<N, INTER, EVEN>(p);
    const int64_t groups = (p.m + p.rows - 1) / p.rows;
    for (int64_t g = blockIdx.x; g < groups; g += gridDim.x) {
        const int64_t row0 = g * p.rows;
        const int rows = (int)min((int64_t)p.rows, p.m - row0);
        __syncthreads();
        for (int i = threadIdx.x; i < rows * p.half; i += 256) {
            const int r = i / p.half, j = i - r * p.half;
            cs[in_lds(i)] = turn((double)p.pos[row0 + r] * p.freq[j] * 0.15915494309189535, p.scale, p.inverse);
        }
        __syncthreads();
        const int units = rows * heads * n.all;
        for (int u = threadIdx.x; u < units; u += 256) {
            const int rh = u / n.all, r = rh / heads, hh = rh - r * heads;
            int piece = u - rh * n.all;
            const int which = hh >= p.heads[0], h = which ? hh - p.heads[0] : hh;
            const T *x = (const T *)(p.in[which] + (row0 + r) * p.ld_in[which]) + (int64_t)h * p.d;
            T *y = (T *)(p.out[which] + (row0 + r) * p.ld_out[which]) + (int64_t)h * p.d;
            const int t = r * p.half;
            if (piece < n.pairs) {
                const int at = EVEN ? piece * N : min(piece * N, n.part - N), first = t + (INTER ? at / 2 : at), first_lds = in_lds(first);
                // (EVEN: a piece's entries are all of the same eight)
                auto entry = [&](int i) { return cs[EVEN ? first_lds + i : in_lds(first + i)]; };
                V v, z;
                v.load(x + at);
                if constexpr (INTER) {
#pragma unroll
                    for (int e = 0; e < N; e += 2) turn_pair(v.x[e], v.x[e + 1], entry(e / 2));
                } else {
                    z.load(x + at + p.half);
#pragma unroll
                    for (int e = 0; e < N; ++e) turn_pair(v.x[e], z.x[e], entry(e));
                    z.store(y + at + p.half);
                }
                v.store(y + at);
                continue;
            }
            piece -= n.pairs;
            if (!EVEN && piece < n.singles) {
                const int j = (INTER ? p.half : n.part) - n.singles + piece, ia = INTER ? 2 * j : j, ib = INTER ? 2 * j + 1 : j + p.half;
                T a = x[ia], b = x[ib];
                turn_pair(a, b, cs[in_lds(t + j)]);
                y[ia] = a, y[ib] = b;
                continue;
            }
            piece -= n.singles;
            if (x == y) continue;
            if (EVEN || piece < n.rest) {
                const int at = rot + (EVEN ? piece * N : min(piece * N, p.d - rot - N));
                V v;
                v.load(x + at);
                v.store(y + at);
            } else {
                const int at = rot + piece - n.rest;  // (fewer than 16 bytes of them)
                y[at] = x[at];
            }
        }
    }
}

template <typename T, bool INTER>
hipError_t launch(RotaryArgs p, hipStream_t s)
{
    constexpr int N = Some<T>::N;
    const bool even = (INTER ? 2 * p.half : p.half) % N == 0 && (p.d - 2 * p.half) % N == 0;
    p.in_place = p.in[0] == p.out[0] || (p.heads[1] > 0 && p.in[1] == p.out[1]);
    // Rows of a workgroup: one where that has work for all of its threads, more of smaller ones where there are rows enough.  us with 1 / 2 / 4:
    // 20000 rows of 40 heads of 128 70.6 / 74.8 / 77.7, 5000 of 12 heads of 64 in fp32 9.5 / 8.9 / 8.5.
    const int64_t units = (int64_t)(p.heads[0] + p.heads[1]) * (even ? pieces_of<N, INTER, true>(p) : pieces_of<N, INTER, false>(p)).all;
    p.rows = units >= 256 ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(768 / units, kTurns / p.half), p.m / 1024));
    const int64_t groups = (p.m + p.rows - 1) / p.rows;
    const dim3 grid((unsigned)std::min<int64_t>(groups, 1 << 16));
    void (*kernel)(RotaryArgs) = even ? rotary_kernel<T, INTER, true> : rotary_kernel<T, INTER, false>;
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
