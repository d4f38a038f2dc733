// Attention over the paged history cache in 8 bits (gfx950): rows of the call in bf16, cached keys and values in e4m3 with a power of two
// for each 16 tokens and cache head (Eq. (3) of Climber, arXiv 2502.09888; the mask of Sec. 3.2 for candidates).
//
// The mathematics are those of the bf16 paged attention (transposed problem, a lane owns a packed row, one pass over the keys).  An e4m3 value
// times a power of two is a bf16 number exactly, so that v_cvt_scalef32_pk_bf16_fp8, which multiplies on its way, makes the operands of the bf16
// matrix instructions and nothing is lost behind the cache's own rounding.  (Products of 8-bit operands would round queries and
// probabilities to four bits.)  Every row sees all cached tokens of its sequence; masks only concern the call's own rows, which
// are seen as they were brought.
#include "paged8.h"
#include "paged_combine.h"
#include "paged_state_bf16.h"

namespace climber {
namespace {

using namespace paged;

typedef int i32x2 __attribute__((__vector_size__(8)));
typedef __attribute__((address_space(3))) i32x2 lds_i32x2;
typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;

// 4 codes as bf16 numbers, times `scale` (a power of two)
static __device__ __forceinline__ u32x2 wide4(uint32_t codes, float scale)
{
    const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false), hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true);
    return u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
}
static __device__ __forceinline__ u32x4 wide8(u32x2 codes, float scale)
{
    const u32x2 a = wide4(codes.x, scale), b = wide4(codes.y, scale);
    return u32x4{a.x, a.y, b.x, b.y};
}
static __device__ __forceinline__ float scale_of(uint32_t stored) { return __uint_as_float((stored & 255u) << 23); }

// Rows of D codes in LDS: 16-byte piece c of row r at slot c ^ f(r).  f takes 16 consecutive rows (key fragments: 16 lanes read one piece
// each) to 16 places of the 64 banks, and so it does two pieces of rows r, r + 1, r + 2, r + 3, r + 8, ... r + 11 (value fragments).
template <int D>
struct Rows8 {
    static constexpr int kPieces = D / 16, kPerLoad = 64 / kPieces, kLoads = 16 / kPerLoad;  // (of 16 rows)
    static __device__ __forceinline__ int f(int r)
    {
        return D == 128 ? ((r >> 2) & 1) | (r & 2) | ((r >> 1) & 4) : ((r >> 2) & 1) | ((r >> 2) & 2);
    }
    uint32_t k_at[D / 32], v_at[D / 32];
    __device__ __forceinline__ void init(int lane)
    {
        const int l32 = lane & 31, hf = lane >> 5, G = lane >> 4, i16 = lane & 15;
#pragma unroll
        for (int j = 0; j < D / 32; ++j) k_at[j] = l32 * D + ((2 * j + hf) ^ f(l32)) * 16;
        // transpose reads: a group of 16 lanes names 8 rows of 16 codes, each by two lanes, and each lane gets the 8 codes of one column
        const int j = i16 >> 1, r = 8 * (j >> 2) + 4 * (G >> 1) + (j & 3);
#pragma unroll
        for (int db = 0; db < D / 32; ++db) v_at[db] = r * D + ((2 * db + (G & 1)) ^ f(r)) * 16 + 8 * (i16 & 1);
    }
};

// A wave's copies of the codes of 16 cached keys and their values (one page's) into LDS.
template <int D>
struct Source8 {
    using R = Rows8<D>;
    const Paged8Args &p;
    int hk, cached;              // keys below `cached` are read
    uint32_t at[R::kLoads];
    const uint8_t *k_page;
    int64_t to_v, page_bytes;
    const int32_t *table;

    __device__ __forceinline__ Source8(const Paged8Args &p_, int b, int hk_, int cached_, int lane) : p(p_), hk(hk_), cached(cached_)
    {
#pragma unroll
        for (int i = 0; i < R::kLoads; ++i) {
            const int row = i * R::kPerLoad + lane / R::kPieces;
            at[i] = row * D + ((lane % R::kPieces) ^ R::f(row)) * 16;
        }
        page_bytes = ((int64_t)p.Hkv << p.page_shift) * D;
        k_page = uniform(p.k_pages + ((int64_t)hk << p.page_shift) * D);
        to_v = p.v_pages - p.k_pages;
        table = p.table + (int64_t)b * p.table_ld;
    }
    // of key g, or of the last cached key, which stands for those behind it
    __device__ __forceinline__ int page_number(int g) const { return min(max(table[max(min(g, cached - 1), 0) >> p.page_shift], 0), p.n_pages - 1); }
    // the scales of the 16 keys from g on: of keys in the low byte, of values in the next
    __device__ __forceinline__ uint32_t scales(int g, int page) const
    {
        const int64_t i = (((int64_t)page * p.Hkv + hk) << (p.page_shift - 4)) + ((max(min(g, cached - 1), 0) & ((1 << p.page_shift) - 1)) >> 4);
        return p.k_scale[i] | (uint32_t)p.v_scale[i] << 8;
    }
    __device__ __forceinline__ void issue(int g, int page, lds_u8 *to_k, lds_u8 *to_v_lds) const
    {
        // (a group behind the cached keys: the place in the page is one of the page's, whatever it holds)
        const uint8_t *k = uniform(k_page + page * page_bytes + (g & ((1 << p.page_shift) - 1)) * D), *v = uniform(k + to_v);
#pragma unroll
        for (int i = 0; i < R::kLoads; ++i) {
            copy16((glb_u8 *)k + at[i], to_k + i * 1024);
            copy16((glb_u8 *)v + at[i], to_v_lds + i * 1024);
        }
    }
};

// Key fragments of 32 rows of codes; `scale` is that of this lane's row.
template <int D>
static __device__ __forceinline__ KFrags<D> read_k8(const Rows8<D> &w, const lds_u8 *base, float scale)
{
    KFrags<D> f;
#pragma unroll
    for (int j = 0; j < D / 32; ++j) {
        const u32x4 x = *(const __attribute__((address_space(3))) u32x4 *)(base + w.k_at[j]);
        f.a[2 * j] = frag(wide8(u32x2{x.x, x.y}, scale));
        f.a[2 * j + 1] = frag(wide8(u32x2{x.z, x.w}, scale));
    }
    return f;
}
// Value fragments of 16 rows of codes.  `keep`: bits of the codes that stay (8 keys of this lane).
template <int D>
static __device__ __forceinline__ VFrags<D> read_v8(const Rows8<D> &w, lds_u8 *base, float scale, u32x2 keep)
{
    VFrags<D> f;
#pragma unroll
    for (int db = 0; db < D / 32; ++db) {
        const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2 *)(base + w.v_at[db])));
        f.a[db] = wide8(x & keep, scale);
    }
    return f;
}
// the first n of 4 bytes (n from below 0 to above 4)
static __device__ __forceinline__ uint32_t first_bytes(int n) { return n >= 4 ? ~0u : (1u << (8 * max(n, 0))) - 1u; }

// Fragments of 32 bf16 key rows in the order of a wide state.
template <int D>
static __device__ __forceinline__ KFrags<D> read_k_wide(const lds_u8 *base, int lane)
{
    using R = Rows<D>;
    const int l32 = lane & 31, hf = lane >> 5;
    KFrags<D> f;
#pragma unroll
    for (int s = 0; s < D / 16; ++s)
        f.a[s] = *(const __attribute__((address_space(3))) bf16x8 *)(base + l32 * R::kPitch + ((4 * (s >> 1) + 2 * hf + (s & 1)) ^ R::f(l32)) * 16);
    return f;
}

// ---- tiles ---------------------------------------------------------------------------------------
// A block of 32 keys and their values as codes in LDS: 1 KiB of keys and of values of each wave's 8 keys, or (D = 64) one of both; pieces of a
// row permuted as in Rows8.
template <int D>
struct Block8 {
    static constexpr int kValues = D == 64 ? 512 : 4096, kGroup = 2048;  // from a key to its value; from 16 rows to the next
    static __device__ __forceinline__ int row(int r) { return D == 64 ? (r >> 3) * 1024 + (r & 7) * 64 : r * 128; }
    uint32_t k_at[D / 32], v_at[D / 32];
    __device__ __forceinline__ void init(int lane)
    {
        const int l32 = lane & 31, hf = lane >> 5, G = lane >> 4, i16 = lane & 15, j = i16 >> 1, r = 8 * (j >> 2) + 4 * (G >> 1) + (j & 3);
#pragma unroll
        for (int e = 0; e < D / 32; ++e) {
            k_at[e] = row(l32) + ((2 * e + hf) ^ Rows8<D>::f(l32)) * 16;
            v_at[e] = kValues + row(r) + ((2 * e + (G & 1)) ^ Rows8<D>::f(r)) * 16 + 8 * (i16 & 1);
        }
    }
};

// 4 waves of QB x 32 packed rows share the keys.  Cached blocks of 32 keys travel as codes, by copies that are two blocks ahead, and each wave
// widens the fragments that it takes from them: half the bytes through LDS, which all eight waves of a CU read their operands from (us against one
// widening for all by the wave that copied: sessions 120 / 117, ragged candidates 141 / 133, 512 of each of 64 users 103 / 105).  The call's own
// rows follow as in the bf16 paged cache, in the same LDS.
//
// Bound by the matrix and the vector pipe, which the two waves of a SIMD keep busy at once only in part: of a wave's step of 32 keys 512 cycles are
// products and as many instructions that widen (64, D = 128) and make exponentials (16, or 32 of two blocks of rows).  512 candidates of each of
// 64 users on 1024: 103 us, of them 60 the walk (1.15 PFLOP/s) and 43 the rows' bytes at its ends; 256 to 1024 of each of 16 on 512 to 4096: 129 us
// (0.78 PFLOP/s), the longest one's 128 steps of 0.85 us; chunks of 60 to 500 of eight on 1000 to 4000: 111 us and 6 for the new tokens.
// Built and not kept (us of ragged candidates, of the chunks): parts of the keys for all 170, 135; two teams of four waves in a workgroup, half
// of a tile's keys each, 163, 143, and with their phases in turn 153, 135; one wave per SIMD with 64 rows 162, 166.
template <int D, int QB, bool SUMI>
__global__ __launch_bounds__(256, 2) void attn_paged8_tile_kernel(const Paged8Args p)
{
    using R = Rows<D>;
    constexpr int kRows = 128 * QB, kValues = 32 * R::kPitch;
    constexpr int kShare = 8 * R::kPitch, kCopies = kShare / 1024;  // own rows: a wave's part of either; copies of it
    constexpr int kCopies8 = D / 64;                                // codes: copies of a wave's part of a block
    // (arrays of their own: reads of one do not wait for copies into another.)  Codes in 0 .. 3; own rows: keys and values of stage i in 2 i and 2 i + 1.
    __shared__ __attribute__((aligned(1024))) uint8_t a0[kValues], a1[kValues], a2[kValues], a3[kValues], a4[kValues], a5[kValues], a6[kValues], a7[kValues];
    __shared__ int flags[4];
    auto room = [&](int i) __attribute__((always_inline)) {
        return (lds_u8 *)(i == 0 ? a0 : i == 1 ? a1 : i == 2 ? a2 : i == 3 ? a3 : i == 4 ? a4 : i == 5 ? a5 : i == 6 ? a6 : a7);
    };
    const int lane = threadIdx.x & 63, l32 = lane & 31, hf = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    PagedWork w;
    PagedSeq s;
    if (!paged_work(p, w, s)) return;
    const int rows = s.T * p.G, r_tile = w.tile * kRows;
    if (r_tile >= rows) return;
    const int r_wave = r_tile + wave * 32 * QB;
    const bool causal = !SUMI && p.causal;
    const int k_all = SUMI ? s.n : paged_keys(p, s);
    auto sees = [&](int r) { return causal ? min(s.n + min(r, rows - 1) / p.G + 1, k_all) : k_all; };  // packed row r sees keys below it
    int k_lo, k_hi;
    paged_part(p, w.split, sees(r_tile + kRows - 1), 32, k_lo, k_hi);
    k_lo = __builtin_amdgcn_readfirstlane(k_lo), k_hi = __builtin_amdgcn_readfirstlane(k_hi);
    // cached keys: all rows see them
    const int c_lo = min(k_lo, s.n), c_hi = min(k_hi, s.n), n_blocks = (c_hi - c_lo + 31) / 32, n_whole = (c_hi - c_lo) / 32;

    const Source8<D> src(p, w.b, w.hk, c_hi, lane);
    // page numbers and scales of 32 blocks: the lower 32 lanes have those of the first 16 keys, the upper those of the others; of the 32 after them
    const int k_mine = c_lo - hf * (32 * 32 - 16);
    const int first_pages = src.page_number(k_mine + lane * 32), next_pages = src.page_number(k_mine + (32 + lane) * 32);
    const uint32_t first_scales = src.scales(k_mine + lane * 32, first_pages);
    int pages = first_pages, pages_next = next_pages;
    uint32_t scales = first_scales, scales_next = first_scales;
    // this lane's 16 codes of the wave's 8 keys, or (D = 64, upper half) of their values, in a page
    const int part = D == 64 ? lane & 31 : lane, row16 = (wave & 1) * 8 + part / (D / 16);
    const uint32_t page_off = row16 * D + ((part % (D / 16)) ^ Rows8<D>::f(row16)) * 16;
    auto issue = [&](int j, lds_u8 *stage) __attribute__((always_inline)) {
        if ((j & 31) == 0 && j > 0) {
            pages = pages_next;
            pages_next = src.page_number(k_mine + (j + 32 + lane) * 32);
        }
        const int page = __builtin_amdgcn_readlane(pages, (wave >> 1) * 32 + (j & 31)), g = c_lo + j * 32 + (wave >> 1) * 16;
        const uint8_t *k = uniform(src.k_page + page * src.page_bytes + (g & ((1 << p.page_shift) - 1)) * D);
        if constexpr (D == 64) {
            copy16((glb_u8 *)(k + (lane >= 32 ? src.to_v : 0)) + page_off, stage + wave * 1024);
        } else {
            copy16((glb_u8 *)k + page_off, stage + wave * 1024);
            copy16((glb_u8 *)uniform(k + src.to_v) + page_off, stage + Block8<D>::kValues + wave * 1024);
        }
    };
    // the scales of a block's two groups: to be asked for once for each block, in order
    struct Scales {
        uint32_t a, b;
    };
    auto scales_of = [&](int j) __attribute__((always_inline)) {
        if ((j & 31) == 0 && j > 0) scales = scales_next;
        if ((j & 31) == 16) scales_next = src.scales(k_mine + ((j & ~31) + 32 + lane) * 32, pages_next);
        return Scales{(uint32_t)__builtin_amdgcn_readlane(scales, j & 31), (uint32_t)__builtin_amdgcn_readlane(scales, 32 + (j & 31))};
    };
    Block8<D> at8;
    at8.init(lane);
    auto keys_of = [&](lds_u8 *stage, const Scales &sc) __attribute__((always_inline)) {
        const float scale = scale_of(l32 < 16 ? sc.a : sc.b);
        KFrags<D> f;
#pragma unroll
        for (int e = 0; e < D / 32; ++e) {
            const u32x4 x = *(const __attribute__((address_space(3))) u32x4 *)(stage + at8.k_at[e]);
            f.a[2 * e] = frag(wide8(u32x2{x.x, x.y}, scale));
            f.a[2 * e + 1] = frag(wide8(u32x2{x.z, x.w}, scale));
        }
        return f;
    };
    auto values_of = [&](lds_u8 *stage, int g, const Scales &sc, u32x2 keep) __attribute__((always_inline)) {
        const float scale = scale_of((g ? sc.b : sc.a) >> 8);
        VFrags<D> f;
#pragma unroll
        for (int db = 0; db < D / 32; ++db) {
            const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2 *)(stage + g * Block8<D>::kGroup + at8.v_at[db])));
            f.a[db] = wide8(x & keep, scale);
        }
        return f;
    };

    Rows<D> at;
    at.init(lane);
    State<D, QB, true> st;
    auto start = [&]() __attribute__((always_inline)) {
        typename State<D, QB, true>::Row in[QB];
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            const int r = min(r_wave + qb * 32 + l32, rows - 1);
            st.template request<SUMI>(p, qb, s.row0 + r / p.G, w.hk * p.G + r % p.G, w.hk, hf, in[qb]);
        }
        if (n_blocks > 0) issue(0, room(0));
        if (n_blocks > 1) issue(1, room(1));
        if (n_blocks > 2) issue(2, room(2));
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) st.template start<SUMI>(p, qb, hf, in[qb], w.split == 0);
    };
    // this wave's copies have landed but for those of `later` blocks, the last ones issued
    auto landed8 = [&](int later) __attribute__((always_inline)) {
        if (later >= 2) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * kCopies8) : "memory");
        else if (later == 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kCopies8) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    };
    auto landed = [&](int later) __attribute__((always_inline)) {
        if (later >= 2) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(4 * kCopies) : "memory");
        else if (later == 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * kCopies) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    };
    // (with this wave's reads of a stage done: behind the barrier others copy into it)
    auto meet = [&]() __attribute__((always_inline)) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    // own rows, counted from the sequence's first: [n_lo, n_hi), of which all rows of the tile see the first n_clean blocks whole
    int n_lo = 0, n_hi = 0, n_new = 0, n_clean = 0, top[QB], wave_hi = 0;
    PagedSeq own = s;
    own.n = 0;
    if constexpr (!SUMI) {
        n_lo = max(k_lo - s.n, 0), n_hi = max(k_hi - s.n, 0);
        n_new = (n_hi - n_lo + 31) / 32;
        n_clean = __builtin_amdgcn_readfirstlane(max(0, min(sees(r_tile) - s.n, n_hi) - n_lo) / 32);
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) top[qb] = min(sees(r_wave + qb * 32 + l32) - s.n, n_hi);
        wave_hi = min(sees(r_wave + 32 * QB - 1) - s.n, n_hi);
    }
    bool odd = false, far[QB];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) far[qb] = false;
    auto is_far = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) far[qb] |= !(st.l[qb] + other_half(st.l[qb]) < kFar);
    };

#pragma unroll 1
    for (bool again = false;; again = true) {
        start();
        if (!again && n_whole > 0) {
            f32x16 S0[QB], S1[QB];
            bf16x8 P[QB][2];
            landed8(min(n_blocks - 1, 2));
            meet();
            Scales held = scales_of(0);
            st.logits(keys_of(room(0), held), S0);
            st.reference(S0);
            // block j (i = j % 4): its logits in Sc, its values and the next one's keys behind the barrier, where nobody reads block j - 1 any more
            auto step = [&](int j, int i, f32x16 (&Sc)[QB], f32x16 (&Sn)[QB]) __attribute__((always_inline)) {
                landed8(min(1, n_blocks - 2 - j));
                meet();
                if (j + 3 < n_blocks) issue(j + 3, room((i + 3) & 3));
                Scales next = held;
                if (j + 1 < n_whole) next = scales_of(j + 1);
                const KFrags<D> k = keys_of(room((i + 1) & 3), next);
                __builtin_amdgcn_sched_barrier(0);
                st.weights(Sc, P, 0);
                __builtin_amdgcn_sched_barrier(0);
                // (from here on the matrix pipe has work: before the other wave of the SIMD, which makes its exponentials meanwhile; us without / with:
                // chunks of eight users 129 / 117, ragged candidates 139 / 132, 512 of each of 64 users 106 / 104)
                __builtin_amdgcn_s_setprio(1);
                st.logits(k, Sn);  // (behind the last block: not used)
                st.weights(Sc, P, 1);
                const VFrags<D> v0 = values_of(room(i), 0, held, u32x2{~0u, ~0u}), v1 = values_of(room(i), 1, held, u32x2{~0u, ~0u});
                held = next;
                __builtin_amdgcn_sched_barrier(0x40f);
                st.add(v0, P, 0);
                st.add(v1, P, 1);
                __builtin_amdgcn_s_setprio(0);
            };
            for (int j = 0; j < n_whole;) {
                step(j, 0, S0, S1);
                if (++j == n_whole) break;
                step(j, 1, S1, S0);
                if (++j == n_whole) break;
                step(j, 2, S0, S1);
                if (++j == n_whole) break;
                step(j, 3, S1, S0);
                ++j;
            }
            // (now, and at the end: in the blocks to come the reference may move by more than 2^126, which makes zeros of the sums so far)
            is_far();
        }
        // the block that is not whole, and all of them again
#pragma unroll 1
        for (int j = again ? 0 : n_whole; j < n_blocks; ++j) {
            lds_u8 *const stage = room(j & 3);
            landed8(min(2, n_blocks - 1 - j));
            meet();
            if (j + 3 < n_blocks) issue(j + 3, room((j + 3) & 3));
            const Scales sc = scales_of(j);
            const int k0 = c_lo + j * 32;
            f32x16 S[QB];
            bf16x8 P[QB][2];
            bool may[QB];
            st.logits(keys_of(stage, sc), S);
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) {
                hide(S[qb], k0, hf, c_hi);
                may[qb] = j >= n_whole || j == 0 || far[qb];
            }
            st.reference(S, may);
            st.weights(S, P);
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                const int left = c_hi - (k0 + 16 * g + 4 * hf);  // (codes of hidden keys may be no numbers)
                st.add(values_of(stage, g, sc, u32x2{first_bytes(left), first_bytes(left - 8)}), P, g);
            }
        }
        if constexpr (!SUMI) {
            const Source<D, kCopies> rows_src(p, own, w.b, w.hk, n_hi, lane, (wave & 1) * kCopies);
            auto issue_new = [&](int j) __attribute__((always_inline)) {
                rows_src.issue(n_lo + (wave >> 1) * 16 + j * 32, 0, room(2 * (j & 3)) + wave * kShare, room(2 * (j & 3) + 1) + wave * kShare);
            };
            if (n_new > 0) {
                meet();  // (all are done with the cached blocks' places)
                issue_new(0);
                if (n_new > 1) issue_new(1);
                if (n_new > 2) issue_new(2);
            }
            if (!again && n_clean > 0) {
                f32x16 S0[QB], S1[QB];
                bf16x8 P[QB][2];
                landed(min(n_new - 1, 2));
                meet();
                st.logits(read_k_wide<D>(room(0), lane), S0);
                st.reference(S0);
                auto step = [&](int j, int i, f32x16 (&Sc)[QB], f32x16 (&Sn)[QB]) __attribute__((always_inline)) {
                    landed(min(1, n_new - 2 - j));
                    meet();  // block j + 1 is here, and nobody reads block j - 1 any more
                    if (j + 3 < n_new)
                        rows_src.issue(n_lo + (wave >> 1) * 16 + (j + 3) * 32, 0, room(2 * ((i + 3) & 3)) + wave * kShare, room(2 * ((i + 3) & 3) + 1) + wave * kShare);
                    const KFrags<D> k = read_k_wide<D>(room(2 * ((i + 1) & 3)), lane);
                    __builtin_amdgcn_sched_barrier(0);
                    st.weights(Sc, P, 0);
                    __builtin_amdgcn_sched_barrier(0);
                    __builtin_amdgcn_s_setprio(1);
                    st.logits(k, Sn);  // (behind the last block: not used)
                    st.weights(Sc, P, 1);
                    const VFrags<D> v0 = read_v<D>(at, room(2 * i + 1)), v1 = read_v<D>(at, room(2 * i + 1) + 16 * R::kPitch);
                    __builtin_amdgcn_sched_barrier(0x40f);
                    st.add(v0, P, 0);
                    st.add(v1, P, 1);
                    __builtin_amdgcn_s_setprio(0);
                };
                for (int j = 0; j < n_clean;) {
                    step(j, 0, S0, S1);
                    if (++j == n_clean) break;
                    step(j, 1, S1, S0);
                    if (++j == n_clean) break;
                    step(j, 2, S0, S1);
                    if (++j == n_clean) break;
                    step(j, 3, S1, S0);
                    ++j;
                }
                is_far();
            }
            // blocks that not every row sees whole
#pragma unroll 1
            for (int j = again ? 0 : n_clean; j < n_new; ++j) {
                lds_u8 *const keys = room(2 * (j & 3)), *const values = room(2 * (j & 3) + 1);
                landed(min(2, n_new - 1 - j));
                if (j >= n_clean) odd |= clear_odd<kShare>(values + wave * kShare, lane);
                meet();
                if (j + 3 < n_new) issue_new(j + 3);
                const int k0 = n_lo + j * 32;
                if (k0 >= wave_hi) continue;
                f32x16 S[QB];
                bf16x8 P[QB][2];
                bool may[QB];
                st.logits(read_k_wide<D>(keys, lane), S);
#pragma unroll
                for (int qb = 0; qb < QB; ++qb) {
                    hide(S[qb], k0, hf, top[qb]);
                    may[qb] = j >= n_clean || j == 0 || far[qb];
                }
                st.reference(S, may);
                st.weights(S, P);
#pragma unroll
                for (int g = 0; g < 2; ++g) st.add(read_v<D>(at, values + g * 16 * R::kPitch), P, g);
            }
        }
        if (again || n_whole + n_clean == 0) break;
        // Weights far above the reference of the first block (or sums with them that passed the largest number): all of it again, block by
        // block.  The reference of the rows that have them may move then; the others' results are made in the same way again, and do not
        // depend on their neighbours.
        bool some = false;
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            float nothing = 0.f;  // unless an output is no finite number
#pragma unroll
            for (int db = 0; db < D / 32; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) nothing = fmaf(st.O[qb][db][i], 0.f, nothing);
            far[qb] |= !(st.l[qb] + other_half(st.l[qb]) < kFar) || !(nothing + other_half(nothing) == 0.f);
            some |= far[qb];
        }
        const int wave_far = __builtin_amdgcn_ballot_w64(some) != 0;
        if (lane == 0) flags[wave] = wave_far;
        __syncthreads();
        const bool any = (flags[0] | flags[1] | flags[2] | flags[3]) != 0;
        __syncthreads();
        if (__builtin_expect(!any, 1)) break;
        pages = first_pages, pages_next = next_pages, scales = first_scales;
        odd = false;
    }
    store_tile<D>(p, s, w, st, r_wave, rows);
    if constexpr (!SUMI) {
        if (lane == 0) flags[wave] = odd;
        __syncthreads();
        if (__builtin_expect(flags[0] | flags[1] | flags[2] | flags[3], 0))
            put_odd<D>(p, s, w, s.n + n_lo + n_clean * 32, k_hi, r_wave, min(r_wave + 32 * QB, rows), sees);
    }
}

// ---- new tokens ----------------------------------------------------------------------------------
// A wave for a block of 16 tokens of a cache head (the block-th that the sequence's new tokens touch), bound by its chain of loads: 6 us of 2200 new tokens
// of 8 users.  The scale is the least with which all of the block's tokens, those that were
// stored before too, stay within 448 of it; where it grows these are rounded again (by a power of two, so that only what lies near the
// smallest numbers changes).  Infinities become no numbers.
static __device__ __forceinline__ uint32_t wave_max(uint32_t x)
{
#pragma unroll
    for (int m = 32; m; m >>= 1) x = max(x, (uint32_t)__shfl_xor((int)x, m, 64));
    return __builtin_amdgcn_readfirstlane(x);
}

template <int D>
struct StoreBlock {
    static constexpr int kLanes = D / 8, kRows = 64 / kLanes, kLoads = 16 / kRows;  // lanes of a row, 8 values each
    bool any;
    int page, in, slot0, old, n, was[2];
    int64_t to, at;
    u32x4 x[2][kLoads];
    // what it needs of the new rows, and the scales so far
    __device__ __forceinline__ void load(const Paged8Args &p, const PagedSeq &s, int b, int hk, int block)
    {
        const int lane = threadIdx.x & 63, end = min(s.n + s.T, p.max_len);
        slot0 = ((s.n >> 4) + block) * 16;
        any = slot0 < end && s.T > 0;
        if (!any) return;
        old = min(max(s.n - slot0, 0), 16), n = min(end - slot0, 16);  // tokens [0, old) stay, [old, n) come
#pragma unroll
        for (int kv = 0; kv < 2; ++kv)
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int j = i * kRows + lane / kLanes;
                x[kv][i] = u32x4{0, 0, 0, 0};
                if (j >= old && j < n)
                    x[kv][i] = *(const u32x4 *)((kv ? p.v : p.k) + (s.row0 + slot0 + j - s.n) * p.ld_kv + (int64_t)hk * (2 * D) + (lane % kLanes) * 16);
            }
        page = p.table[(int64_t)b * p.table_ld + (slot0 >> p.page_shift)];
        any = page >= 0 && page < p.n_pages;
        if (!any) return;
        in = slot0 & ((1 << p.page_shift) - 1);
        const int64_t head = (int64_t)page * p.Hkv + hk;
        to = ((head << p.page_shift) + in) * D, at = (head << (p.page_shift - 4)) + (in >> 4);
        was[0] = old > 0 ? p.k_scale[at] : 0, was[1] = old > 0 ? p.v_scale[at] : 0;
    }
    // (nobody reads the block any more)
    __device__ __forceinline__ void write(const Paged8Args &p, const PagedSeq &s, int hk) const
    {
        if (!any) return;
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
            uint8_t *const pages = kv ? p.v_pages : p.k_pages;
            uint32_t top = 0;  // largest finite magnitude, as bits of a bf16
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t lo = x[kv][i][e] & 0x7fffu, hi = (x[kv][i][e] >> 16) & 0x7fffu;
                    top = max(top, max(lo < 0x7f80u ? lo : 0u, hi < 0x7f80u ? hi : 0u));
                }
            top = wave_max(top);
            // 1.m 2^(e - 127) <= 448 2^s = 1.75 2^(s + 8)
            const int mine = max((int)(top >> 7) - 8 + ((top & 127u) > 96u), kLeastScale), now = max(was[kv], mine);
            if (old > 0 && now > was[kv]) {
                const float down = now - was[kv] > 126 ? 0.f : __uint_as_float((uint32_t)(127 - (now - was[kv])) << 23);
#pragma unroll
                for (int i = 0; i < kLoads; ++i) {
                    const int j = i * kRows + lane / kLanes;
                    if (j >= old) continue;
                    u32x2 *const c = (u32x2 *)(pages + to + j * D + (lane % kLanes) * 8);
                    u32x2 y = *c;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const auto a = __builtin_amdgcn_cvt_pk_f32_fp8(y[e], false), b2 = __builtin_amdgcn_cvt_pk_f32_fp8(y[e], true);
                        y[e] = __builtin_amdgcn_cvt_pk_fp8_f32(b2[0] * down, b2[1] * down, __builtin_amdgcn_cvt_pk_fp8_f32(a[0] * down, a[1] * down, 0, false), true);
                    }
                    *c = y;
                }
            }
            const float up = __uint_as_float((uint32_t)(254 - now) << 23);  // 2^(127 - now)
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int j = i * kRows + lane / kLanes;
                if (j < old || j >= n) continue;
                u32x2 y;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t u = x[kv][i][2 * e], v = x[kv][i][2 * e + 1];
                    y[e] = __builtin_amdgcn_cvt_pk_fp8_f32(__uint_as_float(u << 16) * up, __uint_as_float(u & 0xffff0000u) * up, 0, false);
                    y[e] = __builtin_amdgcn_cvt_pk_fp8_f32(__uint_as_float(v << 16) * up, __uint_as_float(v & 0xffff0000u) * up, y[e], true);
                }
                *(u32x2 *)(pages + to + j * D + (lane % kLanes) * 8) = y;
            }
            if (lane == 0 && now != was[kv]) (kv ? p.v_scale : p.k_scale)[at] = (uint8_t)now;
        }
        if (hk == 0 && p.stamp && lane >= old && lane < n)
            p.stamp[((int64_t)page << p.page_shift) + in + lane] = p.stamp_new[s.row0 + slot0 + lane - s.n];
    }
};
template <int D>
static __device__ __forceinline__ void store_unit(const Paged8Args &p, unsigned group)
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t unit = (int64_t)group * 4 + wave, bh = unit / p.store_blocks;
    if (bh >= (int64_t)p.n_seqs * p.Hkv) return;
    const int b = (int)(bh / p.Hkv);
    const PagedSeq s = paged_seq(p, b);
    StoreBlock<D> block;
    block.load(p, s, b, (int)(bh % p.Hkv), (int)(unit % p.store_blocks));
    block.write(p, s, (int)(bh % p.Hkv));
}
template <int D>
__global__ __launch_bounds__(256) void paged8_store_kernel(const Paged8Args p) { store_unit<D>(p, blockIdx.x); }
// ... and the join of the parts of the keys, where there are any: nothing reads the cached tokens any more
template <int D, int GROUPS>
__global__ __launch_bounds__(256) void paged8_finish_kernel(const Paged8Args p, unsigned joins)
{
    if (blockIdx.x < joins) paged_join::combine_rows<__bf16, GROUPS>(p, blockIdx.x);
    else store_unit<D>(p, blockIdx.x - joins);
}

// ---- few rows ------------------------------------------------------------------------------------
// 32 packed rows; the waves of a workgroup take different blocks of 32 keys, each through a ring of its own, and are joined at the end.  Two
// stages, so that a CU has two workgroups: us with four stages and one / this way, all else alike, one token of 64 users 77 / 70, of one long cache
// 59 / 52.  Where a workgroup is the only one that reads its sequence's head it stores the new tokens itself, after it has read the cached ones
// (one token of 64 users in a launch of its own / this way 70 / 65).  Bound by memory: a token of each of 64 users on 500 to 4000 (8 heads of
// 128) 61 us, 291 MB at 4.8 TB/s; of one cache of 98765 40 us of 202 MB at 5.1 TB/s, and 5 for the join.  More parts of the keys: 65 / 67 to 87.
template <int D, bool SUMI>
__global__ __launch_bounds__(256, 2) void attn_paged8_few_kernel(const Paged8Args p)
{
    constexpr int kStage = 2 * 32 * D, kLoads = 4 * Rows8<D>::kLoads;  // a wave's, of a block of 32 keys
    __shared__ __attribute__((aligned(1024))) uint8_t stage0[4 * kStage], stage1[4 * kStage];
    __shared__ JoinRoom joined;
    __shared__ int odd_seen[4];
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
    int k_lo, k_hi;
    paged_part(p, w.split, sees(r_tile + 31), 128, k_lo, k_hi);
    k_lo = __builtin_amdgcn_readfirstlane(k_lo), k_hi = __builtin_amdgcn_readfirstlane(k_hi);
    const int c_lo = min(k_lo, s.n), c_hi = min(k_hi, s.n);            // the cached ones
    const int n_blk = (c_hi - c_lo + 31) / 32, mine = n_blk > wave ? (n_blk - wave + 3) / 4 : 0;  // blocks wave, wave + 4, ...

    const Source8<D> src(p, w.b, w.hk, c_hi, lane);
    lds_u8 *const at0 = (lds_u8 *)stage0 + wave * kStage, *const at1 = (lds_u8 *)stage1 + wave * kStage;
    // page numbers of 32 blocks: the lower 32 lanes have those of the first 16 keys, the upper those of the others; of the 32 after them
    const int k_mine = c_lo + wave * 32 - (lane >> 5) * (32 * 128 - 16);
    int pages = src.page_number(k_mine + lane * 128), pages_next = src.page_number(k_mine + (32 + lane) * 128);
    uint32_t scales = src.scales(k_mine + lane * 128, pages), scales_next = scales;
    auto issue = [&](int i, lds_u8 *to) __attribute__((always_inline)) {
        if ((i & 31) == 0 && i > 0) {
            pages = pages_next;
            pages_next = src.page_number(k_mine + (i + 32 + lane) * 128);
        }
        const int k0 = c_lo + (i * 4 + wave) * 32;
        src.issue(k0, __builtin_amdgcn_readlane(pages, i & 31), to, to + 32 * D);
        src.issue(k0 + 16, __builtin_amdgcn_readlane(pages, 32 + (i & 31)), to + 16 * D, to + 48 * D);
    };
    Rows8<D> at;
    at.init(lane);
    State<D, 1, true> st;
    {
        typename State<D, 1, true>::Row in;
        st.template request<SUMI>(p, 0, row, h, w.hk, hf, in);
        if (mine > 0) issue(0, at0);
        if (mine > 1) issue(1, at1);
        st.template start<SUMI>(p, 0, hf, in, w.split == 0 && wave == 0);
    }
    auto block = [&](int i, lds_u8 *keys) __attribute__((always_inline)) {
        // (rows, page numbers and scales were asked for among the copies: this waits for more than it has to, never for less)
        if (i + 1 < mine) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLoads) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if ((i & 31) == 0 && i > 0) scales = scales_next;
        if ((i & 31) == 16) scales_next = src.scales(k_mine + ((i & ~31) + 32 + lane) * 128, pages_next);
        const uint32_t s0 = __builtin_amdgcn_readlane(scales, i & 31), s1 = __builtin_amdgcn_readlane(scales, 32 + (i & 31));
        const int k0 = c_lo + (i * 4 + wave) * 32;
        f32x16 S[1];
        bf16x8 P[1][2];
        st.logits(read_k8<D>(at, keys, scale_of(l32 < 16 ? s0 : s1)), S);
        const bool whole = k0 + 32 <= c_hi;
        if (!whole) hide(S[0], k0, hf, c_hi);
        st.reference(S);
        st.weights(S, P);
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const int left = c_hi - (k0 + 16 * g + 4 * hf);  // (codes of hidden keys may be no numbers)
            st.add(read_v8<D>(at, keys + 32 * D + g * 16 * D, scale_of((g ? s1 : s0) >> 8), u32x2{first_bytes(left), first_bytes(left - 8)}), P, g);
        }
        // its place has been read
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (i + 2 < mine) issue(i + 2, keys);
    };
#pragma unroll 1
    for (int i = 0; i < mine; i += 2) {
        block(i, at0);
        if (i + 1 < mine) block(i + 1, at1);
    }

    bool odd = false;
    int n_lo = 0;
    if constexpr (!SUMI) {
        // the call's own rows: blocks of 32 from the part's first one on
        n_lo = max(k_lo - s.n, 0);
        const int n_hi = max(k_hi - s.n, 0), n_new = (n_hi - n_lo + 31) / 32;
        PagedSeq own = s;
        own.n = 0;
        const Source<D, Rows<D>::kLoads> rows_src(p, own, w.b, w.hk, n_hi, lane, 0);
        Rows<D> vat;
        vat.init(lane);
        const int lim = sees(r) - s.n, lim_lo = sees(r_tile) - s.n;
#pragma unroll 1
        for (int i = (wave - n_blk) & 3; i < n_new; i += 4) {  // (the waves that had fewer cached blocks first)
            const int k0 = n_lo + i * 32;
            lds_u8 *const keys = at0, *const values = at1;
            rows_src.issue(k0, 0, keys, values);
            rows_src.issue(k0 + 16, 0, keys + 16 * Rows<D>::kPitch, values + 16 * Rows<D>::kPitch);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            f32x16 S[1];
            bf16x8 P[1][2];
            st.logits(read_k_wide<D>(keys, lane), S);
            if (k0 + 32 > min(lim_lo, n_hi)) {
                odd |= clear_odd<32 * Rows<D>::kPitch>(values, lane);
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                hide(S[0], k0, hf, min(lim, n_hi));
            }
            st.reference(S);
            st.weights(S, P);
#pragma unroll
            for (int g = 0; g < 2; ++g) st.add(read_v<D>(vat, values + g * 16 * Rows<D>::kPitch), P, g);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        }
    }
    if (lane == 0) odd_seen[wave] = odd;
    StoreBlock<D> put;
    const bool stores = !SUMI && p.n_split == 1 && p.n_tiles == 1;  // (32 rows touch 3 blocks at most)
    if (stores && wave < p.store_blocks) put.load(p, s, w.b, w.hk, wave);
    // (each wave's outputs in units of its reference take the 2 x kStage bytes of two waves' places; all waves are done with theirs at the first barrier)
    join_few<D, true>(p, s, w, st, joined, [&](int j) { return (float *)(j < 2 ? stage0 : stage1) + (j & 1) * 32 * D; }, row, h, r_tile, rows);
    if constexpr (!SUMI) {
        if (__builtin_expect(odd_seen[0] | odd_seen[1] | odd_seen[2] | odd_seen[3], 0)) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // all waves' outputs are written
            __syncthreads();
            const int from = s.n + n_lo, clean = max(0, min(sees(r_tile), k_hi) - from) / 32 * 32;
            if (wave == 0) put_odd<D>(p, s, w, from + clean, k_hi, r_tile, min(r_tile + 32, rows), sees);
        }
        // (all of its waves have read the cached tokens, behind whose barrier they were joined)
        if (stores && wave < p.store_blocks) put.write(p, s, w.hk);
    }
}

template <int D, bool SUMI>
hipError_t launch(Paged8Args p, hipStream_t s)
{
    const int64_t rows = (int64_t)p.m_max * p.G;
    const int tile = paged8_tile_rows(D, rows, (int64_t)p.n_seqs * p.Hkv, p.max_len);
    void (*kernel)(Paged8Args) = tile == 32 ? attn_paged8_few_kernel<D, SUMI> : attn_paged8_tile_kernel<D, 1, SUMI>;
    if constexpr (D == 64)
        if (tile == 256) kernel = attn_paged8_tile_kernel<D, 2, SUMI>;
    p.n_tiles = (int)((rows + tile - 1) / tile);
    p.store_blocks = SUMI ? 0 : (int)paged8_store_blocks(p.m_max);
    const unsigned grid = paged_grid(p);
    // All at once, two to a CU: the longest sequence is to be there with the shortest (us without / with: one token of 64 users on 500 to 4000 64.7 / 61.4).
    // Over 224 shapes of 257 to 512 workgroups it takes 0.94 of the time for few rows of ragged lengths (one token of 35 users on 1668 to 13342 102 / 80; but
    // one candidate of each of 49 users on 11 to 91 6.6 / 7.7: there the ranks cost more than there is to gain), 0.98 to 1.00 for tiles (73 candidates of
    // 18 users on 258 to 2064 66 / 56; 690 of 18 on 167 to 668 24.8 / 27.3) and with parts of the keys (one token of 59 users on 2067 to 8268 26.0 / 22.7; 22 of five on 914 to 7313
    // 18.6 / 20.2), and 1.00 where lengths are equal.
    const int64_t per = (int64_t)p.Hkv * p.n_tiles * p.n_split, groups = per * p.n_seqs;
    if (p.n_seqs > 1 && p.n_seqs <= 64 && groups > 256 && groups <= 512) p.by_work = 1, p.pair = (int)((255 + per) / per);
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(256), 0, s, p);
    const unsigned stores = (unsigned)(((int64_t)p.n_seqs * p.Hkv * p.store_blocks + 3) / 4);
    if (p.n_split > 1) {
        const int64_t all = (int64_t)p.m_total * p.H;
        const unsigned joins = (unsigned)(p.n_split <= 4 ? (all + 7) / 8 : all);
        if (p.n_split <= 4) hipLaunchKernelGGL((paged8_finish_kernel<D, 1>), dim3(joins + stores), dim3(256), 0, s, p, joins);
        else hipLaunchKernelGGL((paged8_finish_kernel<D, 8>), dim3(joins + stores), dim3(256), 0, s, p, joins);
    } else if (!SUMI && (tile != 32 || p.n_tiles > 1)) {
        hipLaunchKernelGGL(paged8_store_kernel<D>, dim3(stores), dim3(256), 0, s, p);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_attn_paged8(const Paged8Args &a, hipStream_t s)
{
    if (a.d == 64) return a.sumi ? launch<64, true>(a, s) : launch<64, false>(a, s);
    return a.sumi ? launch<128, true>(a, s) : launch<128, false>(a, s);
}

}  // namespace climber
