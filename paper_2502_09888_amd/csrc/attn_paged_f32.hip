// Attention over the paged history cache in fp32 (gfx950): a chunk of new behaviours, or candidates, of every sequence against
// its cached tokens and its own rows (Eq. (3) of Climber, arXiv 2502.09888; the mask of Sec. 3.2 for candidates), the join of partial
// results, and the accumulation of the attention weights per cached token.
#include "paged_combine.h"

#include <algorithm>
#include <type_traits>

namespace climber {
namespace {

typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;

using paged_join::combine_rows;
using paged_join::f32x4;
using paged_join::store4;

constexpr int kKeys = 32;              // keys of a tile
constexpr float kNoRef = -3.40282347e38f;  // "no reference yet": no finite logit is below it

static __device__ __forceinline__ f32x4 load4(const float *p) { return *(const f32x4 *)p; }

static __device__ __forceinline__ float half_max(float x) { return fmaxf(x, __shfl_xor(x, 32, 64)); }

// 32 keys (rows pointed to by key_ptr) into LDS, pitch DP + 4 floats, zeros beyond d
template <int DP, int NT, typename Ptr>
static __device__ __forceinline__ void load_tile(float *to, int d, Ptr key_ptr)
{
    constexpr int C = DP / 4;
    for (int i = threadIdx.x; i < kKeys * C; i += NT) {
        const int r = i / C, c = (i % C) * 4;
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
        if (c < d) x = load4((const float *)key_ptr(r) + c);
        *(f32x4 *)(to + r * (DP + 4) + c) = x;
    }
}

// The new tokens of packed rows r0 .. r1 - 1 go into their pages.  (No call reads them from there before this one is done.)
template <int NT>
static __device__ __forceinline__ void store_new(const PagedArgs &p, const PagedSeq &s, int b, int hk, int r0, int r1)
{
    const int t0 = (r0 + p.G - 1) / p.G, t1 = (r1 + p.G - 1) / p.G, C = p.row_bytes / 16;
    for (int i = threadIdx.x; i < (t1 - t0) * C; i += NT) {
        const int t = t0 + i / C, c = (i % C) * 16, slot = s.n + t;
        if (slot >= p.max_len) break;
        const int page = p.table[(int64_t)b * p.table_ld + (slot >> p.page_shift)];
        if (page < 0 || page >= p.n_pages) continue;
        const int64_t to = paged_row(p, page, hk, slot) + c, from = (s.row0 + t) * p.ld_kv + (int64_t)hk * p.row_bytes + c;
        *(uint4 *)(p.k_pages + to) = *(const uint4 *)(p.k + from);
        *(uint4 *)(p.v_pages + to) = *(const uint4 *)(p.v + from);
        if (hk == 0 && c == 0 && p.stamp) p.stamp[((int64_t)page << p.page_shift) + (slot & ((1 << p.page_shift) - 1))] = p.stamp_new[s.row0 + t];
    }
}

// a candidate's own key and value: the first member of its softmax
template <int DP>
static __device__ __forceinline__ void own_first(const PagedArgs &p, int64_t row, int hk, int hf, const f32x4 (&q)[DP / 8], float &m, float &l,
                                                 f32x16 (&O)[DP / 32])
{
    const float *kp = (const float *)(p.k + row * p.ld_kv) + (int64_t)hk * p.d, *vp = (const float *)(p.v + row * p.ld_kv) + (int64_t)hk * p.d;
    float dot = 0.f;
#pragma unroll
    for (int i = 0; i < DP / 8; ++i)
        if (8 * i + 4 * hf < p.d) {
            const f32x4 x = load4(kp + 8 * i + 4 * hf);
            dot += q[i][0] * x[0] + q[i][1] * x[1] + q[i][2] * x[2] + q[i][3] * x[3];
        }
    m = dot + __shfl_xor(dot, 32, 64);
    l = hf == 0 ? 1.f : 0.f;
    if (m != m) l = m, m = kNoRef;  // (a logit that is no number makes the row none)
    if (m == -INFINITY) {           // (one of -inf has no part in it)
        l = 0.f, m = kNoRef;
        return;
    }
#pragma unroll
    for (int db = 0; db < DP / 32; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            if (32 * db + 8 * g + 4 * hf < p.d) {
                const f32x4 x = load4(vp + 32 * db + 8 * g + 4 * hf);
#pragma unroll
                for (int e = 0; e < 4; ++e) O[db][4 * g + e] = x[e];
            }
}

// 32 keys from k0 on: logits S, values by value(db, i), the operand of step i; the lane's row sees keys below `top`, and all rows of the
// wave see all keys unless masked
template <int DP, typename Value>
static __device__ __forceinline__ void block_softmax(f32x16 &S, float &m, float &l, f32x16 (&O)[DP / 32], float c, int k0, int hf, int top, bool masked,
                                                     Value value)
{
    constexpr int NB = DP / 32;
    auto key_of = [&](int i) { return k0 + 8 * (i >> 2) + 4 * hf + (i & 3); };
    if (masked) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (key_of(i) >= top) S[i] = -INFINITY;
    }
    float mx = S[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, S[i]);
    mx = fmaxf(half_max(mx), m);
    const float alpha = __builtin_amdgcn_exp2f((m - mx) * c);
    m = mx;
    l *= alpha;
#pragma unroll
    for (int db = 0; db < NB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) O[db][i] *= alpha;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        S[i] = __builtin_amdgcn_exp2f((S[i] - m) * c);
        l += S[i];
    }
    if (!masked) {
#pragma unroll
        for (int db = 0; db < NB; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) O[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(value(db, i), S[i], O[db], 0, 0, 0);
        return;
    }
    // A row must not meet the values of keys that it does not see, not even with probability 0, where they are infinite or
    // no numbers: those take part as zeros, and the rows that do see one get it by a count of such values.
#pragma unroll
    for (int db = 0; db < NB; ++db) {
        bool odd = false;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float x = value(db, i);
            const bool fine = fabsf(x) < INFINITY;
            odd |= !fine;
            O[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(fine ? x : 0.f, S[i], O[db], 0, 0, 0);
        }
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(odd) == 0, 1)) continue;
#pragma unroll 1
        for (int kind = 0; kind < 2; ++kind) {  // infinities of a sign; what is no number counts as both
            f32x16 n;
#pragma unroll
            for (int i = 0; i < 16; ++i) n[i] = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float x = value(db, i);
                const bool is = x != x || x == (kind == 0 ? INFINITY : -INFINITY);
                n = __builtin_amdgcn_mfma_f32_32x32x2f32(is ? 1.f : 0.f, key_of(i) < top ? 1.f : 0.f, n, 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (n[i] > 0.f) O[db][i] += kind == 0 ? INFINITY : -INFINITY;
        }
    }
}

// The transposed problem, as in the bf16 kernels: S^T = K Q^T and O^T = V^T P^T with v_mfma_f32_32x32x2_f32.  A lane owns one packed
// row (lane % 32), its probabilities leave the accumulator as the operand of the value product (step r of it takes the keys of
// accumulator register r).  The sum over the dimensions is taken in an order that lets a lane read four of them at once.  Four waves
// with 32 rows each share the keys of a stage.  Chunks of 1000 behaviours of eight users on 1000, 8 heads of 64: 327 us, 75 TFLOP/s (a library
// product reaches 155; with keys requested when their turn comes a sixth more time); 256 candidates of each of 16 users on 1000 102 us,
// 82 TFLOP/s (a quarter more time with registers for one workgroup per CU).  There are two barriers for each 32 keys, and a page number's trip
// to memory in front of each request.
template <int DP, bool SUMI>
__global__ __launch_bounds__(256, 2) void attn_paged_f32_kernel(const PagedArgs p)
{
    constexpr int kPitch = DP + 4, NB = DP / 32, NW = 4;
    __shared__ __attribute__((aligned(16))) float tk[kKeys * kPitch], tv[kKeys * kPitch];
    const int lane = threadIdx.x & 63, l32 = lane & 31, hf = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    PagedWork w;
    PagedSeq s;
    if (!paged_work(p, w, s)) return;
    const int rows = s.T * p.G, r_tile = w.tile * NW * 32;
    if (r_tile >= rows) return;
    const int r_wave = r_tile + wave * 32, r = min(r_wave + l32, rows - 1), t = r / p.G, h = w.hk * p.G + r % p.G;
    const int64_t row = s.row0 + t;
    const bool causal = !SUMI && p.causal;
    const int k_all = SUMI ? s.n : paged_keys(p, s);
    auto sees = [&](int i) { return causal ? min(s.n + min(i, rows - 1) / p.G + 1, k_all) : k_all; };  // packed row i sees keys below it
    // this lane's row's, the tile's and the wave's bounds
    const int lim = sees(r), k_end = sees(r_tile + NW * 32 - 1), lim_lo = sees(r_wave), lim_hi = sees(r_wave + 31);
    int k_lo, k_hi;
    paged_part(p, w.split, k_end, kKeys, k_lo, k_hi);

    if (!SUMI && w.split == 0) store_new<NW * 64>(p, s, w.b, w.hk, r_tile, min(r_tile + NW * 32, rows));

    f32x4 q[DP / 8];
    const float *qp = (const float *)(p.q + row * p.ld_q) + (int64_t)h * p.d;
#pragma unroll
    for (int i = 0; i < DP / 8; ++i) q[i] = 8 * i + 4 * hf < p.d ? load4(qp + 8 * i + 4 * hf) : f32x4{0.f, 0.f, 0.f, 0.f};
    const float c = paged_row_scale(p, row);
    float m = kNoRef, l = 0.f;
    f32x16 O[NB];
#pragma unroll
    for (int db = 0; db < NB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) O[db][i] = 0.f;
    if (SUMI && w.split == 0) own_first<DP>(p, row, w.hk, hf, q, m, l, O);

    // The next keys are on their way, in registers, while these are worked on.
    constexpr int C = DP / 4, kMine = kKeys * C / 256;
    f32x4 next_k[kMine], next_v[kMine];
    auto request = [&](int k0) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < kMine; ++u) {
            const int i = threadIdx.x + u * 256, j = min(k0 + i / C, k_hi - 1), x = (i % C) * 4;  // keys behind the last one: that one again, and masked
            const bool old = j < s.n;
            const int64_t cached = old ? paged_row(p, paged_page(p, w.b, j), w.hk, j) : 0, fresh = (s.row0 + j - s.n) * p.ld_kv + (int64_t)w.hk * p.row_bytes;
            const float *from_k = (const float *)(old ? p.k_pages + cached : p.k + fresh), *from_v = (const float *)(old ? p.v_pages + cached : p.v + fresh);
            next_k[u] = x < p.d ? load4(from_k + x) : f32x4{0.f, 0.f, 0.f, 0.f};
            next_v[u] = x < p.d ? load4(from_v + x) : f32x4{0.f, 0.f, 0.f, 0.f};
        }
    };
    if (k_lo < k_hi) request(k_lo);
    for (int k0 = k_lo; k0 < k_hi; k0 += kKeys) {
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kMine; ++u) {
            const int i = threadIdx.x + u * 256, to = i / C * kPitch + i % C * 4;
            *(f32x4 *)(tk + to) = next_k[u];
            *(f32x4 *)(tv + to) = next_v[u];
        }
        __syncthreads();
        if (k0 + kKeys < k_hi) request(k0 + kKeys);
        if (r_wave >= rows || k0 >= lim_hi) continue;  // (no row here, or none that sees a key of the tile)
        f32x16 S;
#pragma unroll
        for (int i = 0; i < 16; ++i) S[i] = 0.f;
#pragma unroll
        for (int i = 0; i < DP / 8; ++i) {
            const f32x4 x = *(const f32x4 *)(tk + l32 * kPitch + 8 * i + 4 * hf);
#pragma unroll
            for (int e = 0; e < 4; ++e) S = __builtin_amdgcn_mfma_f32_32x32x2f32(x[e], q[i][e], S, 0, 0, 0);
        }
        block_softmax<DP>(S, m, l, O, c, k0, hf, min(lim, k_hi), k0 + kKeys > min(lim_lo, k_hi),
                          [&](int db, int i) { return tv[(8 * (i >> 2) + 4 * hf + (i & 3)) * kPitch + 32 * db + l32]; });
    }

    if (r_wave + l32 >= rows) return;
    l += __shfl_xor(l, 32, 64);
    const int64_t rh = row * p.H + h;
    if (p.n_split > 1) {
        float *po = p.part_o + ((int64_t)w.split * p.m_total * p.H + rh) * p.d;
#pragma unroll
        for (int db = 0; db < NB; ++db)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                if (32 * db + 8 * g + 4 * hf < p.d)
                    *(f32x4 *)(po + 32 * db + 8 * g + 4 * hf) = f32x4{O[db][4 * g], O[db][4 * g + 1], O[db][4 * g + 2], O[db][4 * g + 3]};
        if (hf == 0) *(float2 *)(p.part_ml + ((int64_t)w.split * p.m_total * p.H + rh) * 2) = float2{m * c, l};
        return;
    }
    const float inv = 1.f / l;
    float *op = (float *)(p.o + row * p.ld_o) + (int64_t)h * p.d;
#pragma unroll
    for (int db = 0; db < NB; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            if (32 * db + 8 * g + 4 * hf < p.d)
                store4(op + 32 * db + 8 * g + 4 * hf, f32x4{O[db][4 * g] * inv, O[db][4 * g + 1] * inv, O[db][4 * g + 2] * inv, O[db][4 * g + 3] * inv});
    if (hf == 0 && p.lse) p.lse[rh] = float2{c, m * c + __builtin_amdgcn_logf(l)};
}

// The same without LDS tiles, for few rows: the waves of a workgroup have the same 32 packed rows and take blocks of 32 keys in turn, whose
// keys and values come straight from memory as operands, all requested before the first is used; their results are joined at
// the end.  Such a call is bound by its chain of loads: one behaviour on 64 cached tokens of one user 7 us of which 5 are the host's (13.6
// by tiles), four sessions of up to 130 on up to 1000, 8 heads of 64, 29 us (49 by tiles).  Two workgroups per CU up to d_head 64: 36 us
// with registers for one; the next block's keys requested before this one's softmax: 31.
template <int DP, bool SUMI>
__global__ __launch_bounds__(256, DP <= 64 ? 2 : 1) void attn_paged_few_f32_kernel(const PagedArgs p)
{
    constexpr int NB = DP / 32;
    __shared__ __attribute__((aligned(16))) float joined[4][32 * DP];
    __shared__ float ref[4][32], denom[4][32];
    __shared__ const uint8_t *value_row[4][32];
    const int lane = threadIdx.x & 63, l32 = lane & 31, hf = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    PagedWork w;
    PagedSeq s;
    if (!paged_work(p, w, s)) return;
    const int rows = s.T * p.G, r_tile = w.tile * 32;
    if (r_tile >= rows) return;
    const int r = min(r_tile + l32, rows - 1), t = r / p.G, h = w.hk * p.G + r % p.G;
    const int64_t row = s.row0 + t;
    const bool causal = !SUMI && p.causal;
    const int k_all = SUMI ? s.n : paged_keys(p, s);
    auto sees = [&](int i) { return causal ? min(s.n + min(i, rows - 1) / p.G + 1, k_all) : k_all; };  // packed row i sees keys below it
    const int lim = sees(r), lim_lo = sees(r_tile);
    int k_lo, k_hi;
    paged_part(p, w.split, sees(r_tile + 31), kKeys, k_lo, k_hi);
    const int n_blk = (k_hi - k_lo + kKeys - 1) / kKeys;

    // a block's operands: key row l32, dimensions 8 i + 4 hf + e; values of key 8 (i / 4) + 4 hf + i % 4, dimension 32 db + l32
    f32x4 k[DP / 8];
    float v[NB][16];
    auto request = [&](int blk) __attribute__((always_inline)) {
        const int j = min(k_lo + blk * kKeys + l32, k_hi - 1);  // keys behind the last one: that one again, and masked
        const bool old = j < s.n;
        const int64_t cached = paged_row(p, old ? paged_page(p, w.b, j) : 0, w.hk, j), fresh = (s.row0 + j - s.n) * p.ld_kv + (int64_t)w.hk * p.row_bytes;
        const uint8_t *at_k = old ? p.k_pages + cached : p.k + fresh, *at_v = old ? p.v_pages + cached : p.v + fresh;
        if (hf == 0) value_row[wave][l32] = at_v;  // (read by the same wave: LDS keeps its order)
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < DP / 8; ++i) k[i] = 8 * i + 4 * hf < p.d ? load4((const float *)at_k + 8 * i + 4 * hf) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float *from = (const float *)value_row[wave][8 * (i >> 2) + 4 * hf + (i & 3)];
#pragma unroll
            for (int db = 0; db < NB; ++db) v[db][i] = 32 * db + l32 < p.d ? from[32 * db + l32] : 0.f;
        }
    };
    f32x4 q[DP / 8];
    const float *qp = (const float *)(p.q + row * p.ld_q) + (int64_t)h * p.d;
#pragma unroll
    for (int i = 0; i < DP / 8; ++i) q[i] = 8 * i + 4 * hf < p.d ? load4(qp + 8 * i + 4 * hf) : f32x4{0.f, 0.f, 0.f, 0.f};
    const float c = paged_row_scale(p, row);
    if (wave < n_blk) request(wave);
    if (!SUMI && w.split == 0) store_new<256>(p, s, w.b, w.hk, r_tile, min(r_tile + 32, rows));
    float m = kNoRef, l = 0.f;
    f32x16 O[NB];
#pragma unroll
    for (int db = 0; db < NB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) O[db][i] = 0.f;
    if (SUMI && w.split == 0 && wave == 0) own_first<DP>(p, row, w.hk, hf, q, m, l, O);

    // logits for the weights per token
    float *const logits = p.logits ? p.logits + (((int64_t)w.b * p.Hkv + w.hk) * (p.m_max * p.G) + r_tile + l32) * p.logits_ld + 4 * hf : nullptr;
    for (int blk = wave; blk < n_blk; blk += 4) {
        const int k0 = k_lo + blk * kKeys;
        f32x16 S;
#pragma unroll
        for (int i = 0; i < 16; ++i) S[i] = 0.f;
#pragma unroll
        for (int i = 0; i < DP / 8; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) S = __builtin_amdgcn_mfma_f32_32x32x2f32(k[i][e], q[i][e], S, 0, 0, 0);
        if (logits && r_tile + l32 < rows) {
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                f32x4 x;
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = k0 + 8 * g + 4 * hf + e < min(lim, k_hi) ? S[4 * g + e] * c : -INFINITY;
                *(f32x4 *)(logits + k0 + 8 * g) = x;
            }
        }
        block_softmax<DP>(S, m, l, O, c, k0, hf, min(lim, k_hi), k0 + kKeys > min(lim_lo, k_hi), [&](int db, int i) { return v[db][i]; });
        if (blk + 4 < n_blk) request(blk + 4);
    }
    l += __shfl_xor(l, 32, 64);
    if (hf == 0) ref[wave][l32] = m, denom[wave][l32] = l;
    __syncthreads();
    const float top = fmaxf(fmaxf(ref[0][l32], ref[1][l32]), fmaxf(ref[2][l32], ref[3][l32]));
    const float mine = l == 0.f ? 0.f : __builtin_amdgcn_exp2f((m - top) * c);
#pragma unroll
    for (int db = 0; db < NB; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            f32x4 x;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = l == 0.f ? 0.f : O[db][4 * g + e] * mine;
            *(f32x4 *)(joined[wave] + l32 * DP + (((8 * db + 2 * g + hf) ^ (l32 & 7)) * 4)) = x;  // (pieces permuted: no conflicts)
        }
    float total = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) total += denom[i][l32] == 0.f ? 0.f : denom[i][l32] * __builtin_amdgcn_exp2f((ref[i][l32] - top) * c);
    __syncthreads();
    if (wave == 0 && hf == 0) {
        denom[0][l32] = total;
        if (r_tile + l32 < rows) {
            const int64_t rh = row * p.H + h;
            if (p.n_split > 1) *(float2 *)(p.part_ml + ((int64_t)w.split * p.m_total * p.H + rh) * 2) = float2{top * c, total};
            else if (p.lse) p.lse[rh] = float2{c, top * c + __builtin_amdgcn_logf(total)};
        }
    }
    __syncthreads();
    constexpr int C = DP / 4;
    const int n_rows = min(32, rows - r_tile);
    for (int i = threadIdx.x; i < n_rows * C; i += 256) {
        const int rr = i / C, cc = i % C, tt = (r_tile + rr) / p.G, hh = w.hk * p.G + (r_tile + rr) % p.G;
        if (cc * 4 >= p.d) continue;
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 4; ++j) x += *(const f32x4 *)(joined[j] + rr * DP + ((cc ^ (rr & 7)) * 4));
        const int64_t rh = (s.row0 + tt) * p.H + hh;
        if (p.n_split > 1) {
            *(f32x4 *)(p.part_o + ((int64_t)w.split * p.m_total * p.H + rh) * p.d + cc * 4) = x;
        } else {
            const float inv = 1.f / denom[0][rr];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] *= inv;
            store4((float *)(p.o + (s.row0 + tt) * p.ld_o) + (int64_t)hh * p.d + cc * 4, x);
        }
    }
}

template <typename E, int GROUPS>
__global__ __launch_bounds__(256) void paged_combine_kernel(const PagedArgs p) { combine_rows<E, GROUPS>(p, blockIdx.x); }

// Attention weights per cached token.  One workgroup: 32 keys of one (sequence, cache head), which stay in registers; its waves
// take the packed rows in turn, p = exp2(s c - lse) again from the logits, and each lane adds up those of its keys.  The sums of a
// cache head go to part[b][hk][slot], without atomics: a second kernel adds the heads up in their order.  Chunks of 1000 behaviours of eight users on
// 1000, 8 heads of 64: 178 us of a call's 505, 69 TFLOP/s; queries come straight from memory, a block's when its turn comes.
template <int DP>
__global__ __launch_bounds__(256) void paged_mass_kernel(const PagedArgs p, float *part)
{
    constexpr int kPitch = DP + 4;
    __shared__ __attribute__((aligned(16))) float tk[kKeys * kPitch];
    __shared__ float sums[4][kKeys];
    const int lane = threadIdx.x & 63, l32 = lane & 31, hf = lane >> 5, wave = threadIdx.x >> 6;
    const int tiles = (p.max_len + kKeys - 1) / kKeys, tile = blockIdx.x % tiles, bh = blockIdx.x / tiles, b = bh / p.Hkv, hk = bh % p.Hkv;
    const PagedSeq s = paged_seq(p, b);
    const int keys = paged_keys(p, s), k0 = tile * kKeys, rows = s.T * p.G;
    if (k0 >= keys || rows == 0) return;
    load_tile<DP, 256>(tk, p.d, [&](int i) {
        const int j = min(k0 + i, keys - 1);
        if (j >= s.n) return p.k + (s.row0 + j - s.n) * p.ld_kv + (int64_t)hk * p.row_bytes;
        return (const uint8_t *)p.k_pages + paged_row(p, paged_page(p, b, j), hk, j);
    });
    __syncthreads();
    float sum[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) sum[i] = 0.f;
    const bool causal = !p.sumi && p.causal;
    const int first = causal ? max(0, k0 - s.n) * p.G : 0;  // rows before it see none of these keys
    for (int r0 = first / 32 * 32 + wave * 32; r0 < rows; r0 += 128) {
        const int r = min(r0 + l32, rows - 1), t = r / p.G, h = hk * p.G + r % p.G;
        const int64_t row = s.row0 + t;
        const int lim = r0 + l32 >= rows ? 0 : causal ? s.n + t + 1 : keys;
        const float *qp = (const float *)(p.q + row * p.ld_q) + (int64_t)h * p.d;
        f32x16 S;
#pragma unroll
        for (int i = 0; i < 16; ++i) S[i] = 0.f;
#pragma unroll 4
        for (int i = 0; i < DP / 8; ++i) {
            const f32x4 q = 8 * i + 4 * hf < p.d ? load4(qp + 8 * i + 4 * hf) : f32x4{0.f, 0.f, 0.f, 0.f};
            const f32x4 x = *(const f32x4 *)(tk + l32 * kPitch + 8 * i + 4 * hf);
#pragma unroll
            for (int e = 0; e < 4; ++e) S = __builtin_amdgcn_mfma_f32_32x32x2f32(x[e], q[e], S, 0, 0, 0);
        }
        const float c = p.lse[row * p.H + h].x, lse = p.lse[row * p.H + h].y;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float w = __builtin_amdgcn_exp2f(fmaf(S[i], c, -lse));
            if (k0 + 8 * (i >> 2) + 4 * hf + (i & 3) < lim) sum[i] += w;
        }
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        float x = sum[i];
#pragma unroll
        for (int o = 1; o < 32; o *= 2) x += __shfl_xor(x, o, 64);
        if (l32 == 0) sums[wave][8 * (i >> 2) + 4 * hf + (i & 3)] = x;
    }
    __syncthreads();
    if (threadIdx.x < kKeys && k0 + (int)threadIdx.x < keys)
        part[(int64_t)bh * p.max_len + k0 + threadIdx.x] =
            (sums[0][threadIdx.x] + sums[1][threadIdx.x]) + (sums[2][threadIdx.x] + sums[3][threadIdx.x]);
}

__global__ __launch_bounds__(256) void paged_mass_add_kernel(const PagedArgs p, const float *part, int n_parts)
{
    const int per = (p.max_len + 255) / 256, b = blockIdx.x / per, j = min((int)(blockIdx.x % per) * 256 + (int)threadIdx.x, p.max_len - 1);
    const int raw = p.table[(int64_t)b * p.table_ld + (j >> p.page_shift)];
    float x = 0.f;  // (of no meaning where the sequence has no such token; requested before its length is known)
#pragma unroll 8
    for (int i = 0; i < n_parts; ++i) x += part[((int64_t)b * n_parts + i) * p.max_len + j];
    const PagedSeq s = paged_seq(p, b);
    if (s.T == 0 || j >= paged_keys(p, s) || j != (int)(blockIdx.x % per) * 256 + (int)threadIdx.x) return;
    if (raw < 0 || raw >= p.n_pages) return;
    float *to = p.mass + ((int64_t)raw << p.page_shift) + (j & ((1 << p.page_shift) - 1));
    *to = j < s.n ? *to + x : x;  // a new token has none yet, whatever its slot holds
}

// The same from logits that the attention of few rows has left: a thread per token, cache heads and rows in their order.
__global__ __launch_bounds__(256) void paged_mass_few_kernel(const PagedArgs p)
{
    const int per = (p.max_len + 255) / 256, b = blockIdx.x / per, j = (blockIdx.x % per) * 256 + threadIdx.x;
    const PagedSeq s = paged_seq(p, b);
    if (s.T == 0 || j >= paged_keys(p, s)) return;
    const int raw = p.table[(int64_t)b * p.table_ld + (j >> p.page_shift)];
    if (raw < 0 || raw >= p.n_pages) return;
    float x = 0.f;
    const int rows = s.T * p.G;
    for (int hk = 0; hk < p.Hkv; ++hk) {
        const float *logits = p.logits + ((int64_t)b * p.Hkv + hk) * (p.m_max * p.G) * p.logits_ld + j;
        float at[kMassFewRows];
#pragma unroll
        for (int r = 0; r < kMassFewRows; ++r) at[r] = r < rows ? logits[(int64_t)r * p.logits_ld] : -INFINITY;
#pragma unroll
        for (int r = 0; r < kMassFewRows; ++r)
            if (r < rows) x += __builtin_amdgcn_exp2f(at[r] - p.lse[(s.row0 + r / p.G) * p.H + hk * p.G + r % p.G].y);
    }
    float *to = p.mass + ((int64_t)raw << p.page_shift) + (j & ((1 << p.page_shift) - 1));
    *to = j < s.n ? *to + x : x;
}

template <int DP>
hipError_t launch(const PagedArgs &a, hipStream_t s)
{
    PagedArgs p = a;
    const int64_t rows = (int64_t)a.m_max * a.G;
    const int tile = paged_tile_rows(false, a.d, rows, (int64_t)a.n_seqs * a.Hkv);
    p.n_tiles = (int)((rows + tile - 1) / tile);
    void (*kernel)(PagedArgs) = a.sumi ? attn_paged_few_f32_kernel<DP, true> : attn_paged_few_f32_kernel<DP, false>;
    if constexpr (DP <= 64)
        if (tile == 128) kernel = a.sumi ? attn_paged_f32_kernel<DP, true> : attn_paged_f32_kernel<DP, false>;
    hipLaunchKernelGGL(kernel, dim3(paged_grid(p)), dim3(256), 0, s, p);
    return hipGetLastError();
}

template <int DP>
void launch_mass(const PagedArgs &p, float *part, hipStream_t s)
{
    const int64_t tiles = (p.max_len + kKeys - 1) / kKeys;
    hipLaunchKernelGGL((paged_mass_kernel<DP>), dim3((unsigned)(tiles * p.n_seqs * p.Hkv)), dim3(256), 0, s, p, part);
}

}  // namespace

hipError_t launch_attn_paged_f32(const PagedArgs &a, hipStream_t s)
{
    return a.d <= 32 ? launch<32>(a, s) : a.d <= 64 ? launch<64>(a, s) : launch<128>(a, s);
}

hipError_t launch_paged_combine(const PagedArgs &a, bool bf16, hipStream_t s)
{
    const int64_t all = (int64_t)a.m_total * a.H;
    auto go = [&](auto groups) {
        constexpr int GROUPS = decltype(groups)::value;
        const dim3 grid((unsigned)((all * GROUPS + 7) / 8));
        if (bf16) hipLaunchKernelGGL((paged_combine_kernel<__bf16, GROUPS>), grid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL((paged_combine_kernel<float, GROUPS>), grid, dim3(256), 0, s, a);
    };
    if (a.n_split <= 4) go(std::integral_constant<int, 1>{});
    else go(std::integral_constant<int, 8>{});
    return hipGetLastError();
}

hipError_t launch_paged_mass_f32(const PagedArgs &a, float *part, hipStream_t s)
{
    if (a.d <= 32) launch_mass<32>(a, part, s);
    else if (a.d <= 64) launch_mass<64>(a, part, s);
    else launch_mass<128>(a, part, s);
    return hipGetLastError();
}

hipError_t launch_paged_mass_few(const PagedArgs &a, hipStream_t s)
{
    hipLaunchKernelGGL(paged_mass_few_kernel, dim3((unsigned)((a.max_len + 255) / 256 * a.n_seqs)), dim3(256), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_paged_mass_add(const PagedArgs &a, const float *part, int n_parts, hipStream_t s)
{
    hipLaunchKernelGGL(paged_mass_add_kernel, dim3((unsigned)((a.max_len + 255) / 256 * a.n_seqs)), dim3(256), 0, s, a, part, n_parts);
    return hipGetLastError();
}

}  // namespace climber
