// What the bf16 attention kernels over a paged cache share (internal): a wave's copies of bf16 rows into LDS, the softmax state of its packed
// rows, masks, and values that a row must not meet.
#pragma once
#include "paged_bf16.h"

namespace climber {
namespace paged {

// "no reference yet", as a raw logit: no finite one is below it once scaled by c, and c times it is finite (a hidden key's weight is
// exp2(-inf - c m))
static __device__ __forceinline__ float no_ref(float c) { return -3.4028e38f * __builtin_amdgcn_rcpf(fmaxf(c, 1.f)); }
constexpr float kSlack = 8.0f;      // log2 units that a logit may exceed the reference by
constexpr float kFar = 0x1p100f;    // a denominator over it: the reference was too low, see attn_paged_tile_kernel

// a pointer that is the same in all lanes, in scalar registers
static __device__ __forceinline__ const uint8_t *uniform(const uint8_t *p)
{
    const uint64_t a = (uint64_t)p;
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)a), hi = __builtin_amdgcn_readfirstlane((uint32_t)(a >> 32));
    return (const uint8_t *)(((uint64_t)hi << 32) | lo);
}

// What a wave knows of its sequence, and its copies of keys and values into LDS: LOADS times 1 KiB of the rows of 16 keys, from the
// FIRST-th on.
template <int D, int LOADS>
struct Source {
    using R = Rows<D>;
    const PagedArgs &p;
    PagedSeq s;
    int hk, k_hi, cached, lane, first;         // cached: keys below it are in pages (and below k_hi)
    uint32_t page_off[LOADS], row_off[LOADS];  // of this lane's piece, per load: in rows of a page, in rows of the call
    const uint8_t *k_page, *k_new;             // the head's keys of page 0; of the sequence's first row of the call
    int64_t to_v_page, to_v_new, page_bytes;   // from a key to its value; from a page to the next
    const int32_t *table;

    __device__ __forceinline__ Source(const PagedArgs &p_, const PagedSeq &s_, int b, int hk_, int k_hi_, int lane_, int first_)
        : p(p_), s(s_), hk(hk_), k_hi(k_hi_), cached(min(s_.n, k_hi_)), lane(lane_), first(first_)
    {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            page_off[i] = row(i) * R::kPitch + piece(i);
            row_off[i] = (uint32_t)row(i) * (uint32_t)p.ld_kv + piece(i);
        }
        const int64_t in_page = ((int64_t)hk << p.page_shift) * R::kPitch, at = s.row0 * p.ld_kv + (int64_t)hk * R::kPitch;
        page_bytes = ((int64_t)p.Hkv << p.page_shift) * R::kPitch;
        k_page = uniform(p.k_pages + in_page);
        k_new = uniform(p.k + at);
        to_v_page = p.v_pages - p.k_pages;
        to_v_new = p.v - p.k;
        table = p.table + (int64_t)b * p.table_ld;
    }
    __device__ __forceinline__ int row(int i) const { return (first + i) * R::kPerLoad + lane / R::kPieces; }
    __device__ __forceinline__ int piece(int i) const { return ((lane % R::kPieces) ^ R::f(row(i))) * 16; }
    // of key g (groups of 16 lie in one page), or of the last cached key, which stands for those behind it
    __device__ __forceinline__ int page_number(int g) const
    {
        return min(max(table[max(min(g, cached - 1), 0) >> p.page_shift], 0), p.n_pages - 1);
    }
    // of keys g .. g + 15, which lie in `page`, to LDS at to_k, to_v (wave-uniform)
    __device__ __forceinline__ void issue(int g, int page, lds_u8 *to_k, lds_u8 *to_v) const
    {
        const int in_page = (1 << p.page_shift) - 1;
        if (g + 16 <= cached) {
            const uint8_t *k = uniform(k_page + page * page_bytes + (g & in_page) * R::kPitch), *v = uniform(k + to_v_page);
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                copy16((glb_u8 *)k + page_off[i], to_k + i * 1024);
                copy16((glb_u8 *)v + page_off[i], to_v + i * 1024);
            }
        } else if (g >= s.n && g + 16 <= k_hi) {
            const uint8_t *k = uniform(k_new + (g - s.n) * p.ld_kv), *v = uniform(k + to_v_new);
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                copy16((glb_u8 *)k + row_off[i], to_k + i * 1024);
                copy16((glb_u8 *)v + row_off[i], to_v + i * 1024);
            }
        } else {  // cached and new ones, or fewer than 16: the last key again in the places behind it
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const int j = min(g + row(i), k_hi - 1);
                const bool old = j < s.n;
                const uint8_t *cached_k = k_page + page * page_bytes + (j & in_page) * R::kPitch + piece(i), *new_k = k_new + (j - s.n) * p.ld_kv + piece(i);
                const uint8_t *cached_v = cached_k + to_v_page, *new_v = new_k + to_v_new;
                copy16((glb_u8 *)(old ? cached_k : new_k), to_k + i * 1024);
                copy16((glb_u8 *)(old ? cached_v : new_v), to_v + i * 1024);
            }
        }
    }
};

// 8 dimensions of a row as a lane reads or writes them (16 bytes: the first 8 of 16 in the lower half-wave) <-> as the accumulator has
// them (4 and 4: the first 4 of each 8 in the lower half-wave)
static __device__ __forceinline__ void swap_pieces(u32x4 &x)
{
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const auto r = __builtin_amdgcn_permlane32_swap(x[i], x[2 + i], false, false);
        x[i] = r[0];
        x[2 + i] = r[1];
    }
}

// The softmax state of a wave's QB x 32 packed rows.  WIDE: product s of the logits takes dimensions 32 (s / 2) + 16 hf + 8 (s % 2) of
// half-wave hf, so that a lane reads 16 dimensions of a key at once (keys in 8 bits); otherwise 16 s + 8 hf.
template <int D, int QB, bool WIDE = false>
struct State {
    bf16x8 q[QB][D / 16];
    f32x16 O[QB][D / 32];
    float c[QB], m[QB], l[QB];  // scale; reference (raw logit); this half-wave's share of the denominator

    // A row's inputs are requested together, and made use of later: all of them are on their way before the first is waited for.
    struct Row {
        u32x4 k[D / 16], v[D / 16];
        int at;  // its temperature's place
    };
    template <bool OWN>
    __device__ __forceinline__ void request(const PagedArgs &p, int qb, int64_t row, int h, int hk, int hf, Row &in)
    {
        const int sc = p.scen[row], bh = p.beh[row];
        const int to = WIDE ? 2 * hf : hf;
        auto piece = [](int s) { return WIDE ? 4 * (s >> 1) + (s & 1) : 2 * s; };
        const u32x4 *qp = (const u32x4 *)(p.q + row * p.ld_q + (int64_t)h * (2 * D)) + to;
#pragma unroll
        for (int s = 0; s < D / 16; ++s) q[qb][s] = __builtin_bit_cast(bf16x8, qp[piece(s)]);
        if (OWN) {
            const u32x4 *kp = (const u32x4 *)(p.k + row * p.ld_kv + (int64_t)hk * (2 * D)) + to, *vp = (const u32x4 *)(p.v + row * p.ld_kv + (int64_t)hk * (2 * D)) + hf;
#pragma unroll
            for (int s = 0; s < D / 16; ++s) {
                in.k[s] = kp[piece(s)];
                in.v[s] = vp[2 * s];
            }
        }
        in.at = min(max(sc, 0), p.n_scen - 1) * p.n_beh + min(max(bh, 0), p.n_beh - 1);
    }
    // OWN: the row's own key and value are the first member of its softmax (candidates, one part of the keys)
    template <bool OWN>
    __device__ __forceinline__ void start(const PagedArgs &p, int qb, int hf, const Row &in, bool own)
    {
        c[qb] = p.scale_log2e / p.tau[in.at];
        const float none_yet = no_ref(c[qb]);
        m[qb] = none_yet;
        l[qb] = 0.f;
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) O[qb][db][i] = 0.f;
        if (!OWN || !own) return;
        float dot = 0.f;
#pragma unroll
        for (int s = 0; s < D / 16; ++s) {
            const bf16x8 k = __builtin_bit_cast(bf16x8, in.k[s]);
#pragma unroll
            for (int e = 0; e < 8; ++e) dot += (float)q[qb][s][e] * (float)k[e];
        }
        dot += other_half(dot);
        l[qb] = hf == 0 ? 1.f : 0.f;
        m[qb] = dot;
        const bool none = dot == -INFINITY;           // (has no part in it)
        if (none) l[qb] = 0.f, m[qb] = none_yet;
        if (dot != dot) l[qb] = dot, m[qb] = none_yet;  // (a logit that is no number makes the row none)
#pragma unroll
        for (int s = 0; s < D / 16; ++s) {
            u32x4 v = none ? u32x4{0, 0, 0, 0} : in.v[s];
            swap_pieces(v);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                O[qb][s / 2][8 * (s & 1) + 2 * e] = __uint_as_float(v[e] << 16);
                O[qb][s / 2][8 * (s & 1) + 2 * e + 1] = __uint_as_float(v[e] & 0xffff0000u);
            }
        }
    }
    __device__ __forceinline__ void logits(const KFrags<D> &k, f32x16 (&S)[QB]) const
    {
#pragma unroll
        for (int qb = 0; qb < QB; ++qb)
#pragma unroll
            for (int i = 0; i < 16; ++i) S[qb][i] = 0.f;
#pragma unroll
        for (int s = 0; s < D / 16; ++s)
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) S[qb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k.a[s], q[qb][s], S[qb], 0, 0, 0);
    }
    // S: logits of 32 keys, -inf where masked.  The reference of the rows that may moves where a logit exceeds it by far.
    __device__ __forceinline__ void reference(const f32x16 (&S)[QB], const bool (&may)[QB])
    {
        float v[QB];
        bool need[QB], any = false;
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            float x = fmaxf(S[qb][0], S[qb][1]);
#pragma unroll
            for (int i = 2; i < 16; i += 2) x = fmaxf(fmaxf(x, S[qb][i]), S[qb][i + 1]);
            v[qb] = half_max(x);
            need[qb] = may[qb] && (v[qb] - m[qb]) * c[qb] > kSlack;
            any |= need[qb];
        }
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(any) != 0, 0)) {
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) {
                const float alpha = need[qb] ? __builtin_amdgcn_exp2f((m[qb] - v[qb]) * c[qb]) : 1.f;
                if (need[qb]) m[qb] = v[qb];
                l[qb] *= alpha;
#pragma unroll
                for (int db = 0; db < D / 32; ++db)
#pragma unroll
                    for (int i = 0; i < 16; ++i) O[qb][db][i] *= alpha;
            }
        }
    }
    __device__ __forceinline__ void reference(const f32x16 (&S)[QB])
    {
        bool may[QB];
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) may[qb] = true;
        reference(S, may);
    }
    // P: the operand of the value product for 16 of the 32 keys: weights rounded to bf16, since the matrix instruction takes both operands in one
    // type and weights in two pieces would be twice the products.  It is what outputs are off by beside their own rounding: 2.0e-3 to 2.3e-3 (relative, root
    // mean square) for 1.65e-3 with weights in fp32.  WIDE: the denominator takes them as they are rounded for it (two at a time, in
    // fp32; nothing else is made of them), so that they are shares of one.
    __device__ __forceinline__ void weights(const f32x16 (&S)[QB], bf16x8 (&P)[QB][2], int g)
    {
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            const float sub = m[qb] * c[qb];
            if constexpr (WIDE) {
                typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;
                const bf16x2 ones = {(__bf16)1.f, (__bf16)1.f};
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const bf16x2 x = {(__bf16)__builtin_amdgcn_exp2f(fmaf(S[qb][8 * g + e], c[qb], -sub)),
                                      (__bf16)__builtin_amdgcn_exp2f(fmaf(S[qb][8 * g + e + 1], c[qb], -sub))};
                    P[qb][g][e] = x[0], P[qb][g][e + 1] = x[1];
                    l[qb] = __builtin_amdgcn_fdot2_f32_bf16(x, ones, l[qb], false);
                }
                continue;
            }
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float x = __builtin_amdgcn_exp2f(fmaf(S[qb][8 * g + e], c[qb], -sub));
                sum += x;
                P[qb][g][e] = (__bf16)x;
            }
            l[qb] += sum;
        }
    }
    __device__ __forceinline__ void weights(const f32x16 (&S)[QB], bf16x8 (&P)[QB][2])
    {
        weights(S, P, 0);
        weights(S, P, 1);
    }
    // 16 keys' values
    __device__ __forceinline__ void add(const VFrags<D> &v, const bf16x8 (&P)[QB][2], int g)
    {
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) O[qb][db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag(v.a[db]), P[qb][g], O[qb][db], 0, 0, 0);
    }
};

// A row must not meet the values of keys that it does not see, not even with probability 0, where they are infinite or no numbers.
// In tiles that some rows do not see whole such values become zeros in LDS (ROWS value rows at `rows`, landed, by the wave that
// copied them), and at the end put_odd adds them to the outputs of the rows that do see them.
static __device__ __forceinline__ uint32_t odd_halves(uint32_t x) { return ((x & 0x7f807f80u) + 0x00800080u) & 0x80008000u; }
template <int BYTES>
static __device__ __forceinline__ bool clear_odd(lds_u8 *rows, int lane)
{
    uint32_t odd = 0;
#pragma unroll
    for (int i = 0; i < BYTES / 1024; ++i) {
        auto *at = (__attribute__((address_space(3))) u32x4 *)(rows + i * 1024 + lane * 16);
        u32x4 x = *at;
        uint32_t any = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t h = odd_halves(x[e]);
            any |= h;
            x[e] &= ~((h >> 15) * 0xffffu);
        }
        if (any) *at = x;
        odd |= any;
    }
    return __builtin_amdgcn_ballot_w64(odd != 0) != 0;
}
// (a wave; its outputs, or partial ones, of packed rows r0 .. r1 - 1 are written; `sees(r)` as in the kernels)
template <int D, typename Sees>
static __device__ __forceinline__ void put_odd(const PagedArgs &p, const PagedSeq &s, const PagedWork &w, int k_lo, int k_hi, int r0, int r1,
                                               Sees sees)
{
    const int lane = threadIdx.x & 63;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll 1
    for (int j = k_lo; j < k_hi; ++j) {
        const uint8_t *v = j < s.n ? p.v_pages + paged_row(p, paged_page(p, w.b, j), w.hk, j) : p.v + (s.row0 + j - s.n) * p.ld_kv + (int64_t)w.hk * 2 * D;
        const uint32_t x = lane < D / 2 ? *(const uint32_t *)(v + lane * 4) : 0, odd = odd_halves(x);
        if (__builtin_amdgcn_ballot_w64(odd != 0) == 0) continue;
        const float lo = odd & 0x8000u ? __uint_as_float(x << 16) : 0.f, hi = odd >> 31 ? __uint_as_float(x & 0xffff0000u) : 0.f;
#pragma unroll 1
        for (int r = r0; r < r1; ++r) {
            if (j >= sees(r) || !odd) continue;
            const int64_t row = s.row0 + r / p.G, rh = row * p.H + w.hk * p.G + r % p.G;
            auto load = [](const uint32_t *at) { return __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
            auto store = [](uint32_t *at, uint32_t y) { __hip_atomic_store(at, y, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
            if (p.n_split > 1) {
                uint32_t *at = (uint32_t *)(p.part_o + ((int64_t)w.split * p.m_total * p.H + rh) * D) + 2 * lane;
                store(at, __float_as_uint(__uint_as_float(load(at)) + lo));
                store(at + 1, __float_as_uint(__uint_as_float(load(at + 1)) + hi));
            } else {
                uint32_t *at = (uint32_t *)(p.o + row * p.ld_o + (int64_t)(w.hk * p.G + r % p.G) * 2 * D) + lane;
                const uint32_t y = load(at);
                const float a = __uint_as_float(y << 16) + lo, b = __uint_as_float(y & 0xffff0000u) + hi;
                store(at, (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)a) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)b) << 16);
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (the next key's come on top)
        }
    }
}

static __device__ __forceinline__ void hide(f32x16 &S, int k, int hf, int top)
{
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (k + 8 * (i >> 2) + 4 * hf + (i & 3) >= top) S[i] = -INFINITY;
}

// A wave's outputs of a tile, or its part of them.
template <int D, int QB, bool WIDE>
static __device__ __forceinline__ void store_tile(const PagedArgs &p, const PagedSeq &s, const PagedWork &w, const State<D, QB, WIDE> &st, int r_wave, int rows)
{
    const int lane = threadIdx.x & 63, l32 = lane & 31, hf = lane >> 5;
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const int r = r_wave + qb * 32 + l32;
        const float l = st.l[qb] + other_half(st.l[qb]);
        const int64_t row = s.row0 + r / p.G, rh = row * p.H + w.hk * p.G + r % p.G;  // (r >= rows: not stored)
        if (p.n_split > 1) {
            if (r >= rows) continue;
            float *po = p.part_o + ((int64_t)w.split * p.m_total * p.H + rh) * D + 4 * hf;
#pragma unroll
            for (int db = 0; db < D / 32; ++db)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    *(f32x4 *)(po + 32 * db + 8 * g) =
                        f32x4{st.O[qb][db][4 * g], st.O[qb][db][4 * g + 1], st.O[qb][db][4 * g + 2], st.O[qb][db][4 * g + 3]};
            if (hf == 0) *(float2 *)(p.part_ml + ((int64_t)w.split * p.m_total * p.H + rh) * 2) = float2{st.m[qb] * st.c[qb], l};
            continue;
        }
        const float inv = 1.f / l;
        __bf16 *op = (__bf16 *)(p.o + row * p.ld_o) + (int64_t)(w.hk * p.G + r % p.G) * D + 8 * hf;
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int g = 0; g < 4; g += 2) {
                bf16x8 x;
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = (__bf16)(st.O[qb][db][4 * g + e] * inv);
                u32x4 y = __builtin_bit_cast(u32x4, x);
                swap_pieces(y);
                if (r < rows) *(u32x4 *)(op + 32 * db + 8 * g) = y;
            }
        if (hf == 0 && p.lse && r < rows) p.lse[rh] = float2{st.c[qb], st.m[qb] * st.c[qb] + __builtin_amdgcn_logf(l)};
    }
}

// The four waves of a workgroup have had different keys of the same 32 packed rows: their denominators and outputs in units of the largest
// reference, added up and stored.  room(j): 32 D floats of LDS for wave j (whose copies have arrived and been read).
struct JoinRoom {
    float ref[4][32], denom[4][32];
};
template <int D, bool WIDE, typename Room>
static __device__ __forceinline__ void join_few(const PagedArgs &p, const PagedSeq &s, const PagedWork &w, const State<D, 1, WIDE> &st, JoinRoom &j4,
                                                Room room, int64_t row, int h, int r_tile, int rows)
{
    const int lane = threadIdx.x & 63, l32 = lane & 31, hf = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    auto &ref = j4.ref;
    auto &denom = j4.denom;
    const float l = st.l[0] + other_half(st.l[0]);
    if (hf == 0) ref[wave][l32] = st.m[0], denom[wave][l32] = l;
    __syncthreads();
    const float m = fmaxf(fmaxf(ref[0][l32], ref[1][l32]), fmaxf(ref[2][l32], ref[3][l32]));
    const float mine_w = l == 0.f ? 0.f : __builtin_amdgcn_exp2f((st.m[0] - m) * st.c[0]);
    float *joined = room(wave);
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            f32x4 x;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = l == 0.f ? 0.f : st.O[0][db][4 * g + e] * mine_w;
            // (16-byte piece c of row r at slot c ^ r % 8: lanes of neighbouring rows write to different banks)
            *(f32x4 *)(joined + l32 * D + (((8 * db + 2 * g + hf) ^ (l32 & 7)) * 4)) = x;
        }
    float total = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) total += denom[j][l32] == 0.f ? 0.f : denom[j][l32] * __builtin_amdgcn_exp2f((ref[j][l32] - m) * st.c[0]);
    __syncthreads();
    if (wave == 0 && hf == 0) denom[0][l32] = total;  // (read by all above, before the barrier)
    __syncthreads();
    if (wave == 0 && hf == 0 && r_tile + l32 < rows) {
        const int64_t rh = row * p.H + h;
        if (p.n_split > 1) *(float2 *)(p.part_ml + ((int64_t)w.split * p.m_total * p.H + rh) * 2) = float2{m * st.c[0], total};
        else if (p.lse) p.lse[rh] = float2{st.c[0], m * st.c[0] + __builtin_amdgcn_logf(total)};
    }
    constexpr int C = D / 4;
    const int n_rows = min(32, rows - r_tile);
    for (int i = threadIdx.x; i < n_rows * C; i += 256) {
        const int rr = i / C, c = i % C, tt = (r_tile + rr) / p.G, hh = w.hk * p.G + (r_tile + rr) % p.G;
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 4; ++j) x += *(const f32x4 *)(room(j) + rr * D + ((c ^ (rr & 7)) * 4));
        const int64_t rh = (s.row0 + tt) * p.H + hh;
        if (p.n_split > 1) {
            *(f32x4 *)(p.part_o + ((int64_t)w.split * p.m_total * p.H + rh) * D + c * 4) = x;
        } else {
            const float inv = 1.f / denom[0][rr];
            bf16x4 y;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = (__bf16)(x[e] * inv);
            *(bf16x4 *)((__bf16 *)(p.o + (s.row0 + tt) * p.ld_o) + (int64_t)hh * D + c * 4) = y;
        }
    }
}

}  // namespace paged
}  // namespace climber
