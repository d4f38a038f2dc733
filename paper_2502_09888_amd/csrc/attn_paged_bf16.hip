// bf16 MFMA attention over the paged history cache (gfx950): a chunk of new behaviours, or candidates, of every sequence against its
// cached tokens and its own rows (Eq. (3) of Climber, arXiv 2502.09888; the mask of Sec. 3.2 for candidates).
//
// The transposed problem, S^T = K Q^T and O^T = V^T P^T with v_mfma_f32_32x32x16_bf16: a lane owns one packed row (row of the call,
// query head of the group that shares a cache head), softmax statistics are scalars of the lane, and probabilities leave the
// accumulator as the operand of the value product.  One pass over the keys.  Tiles take their reference, which a softmax subtracts, from the
// first keys and run again in the rare case that weights exceed it by 2^100; everything else has a running maximum that moves when a
// logit exceeds it by 2^8.  Logits are scaled in fp32; probabilities rounded to bf16 for the value product and summed before that in fp32
// (the sum also gives the weights per token their denominator, which rounded terms would put off by 3e-5).
//
// Keys and values are rows, in pages or of the call: they travel by global_load_lds, 16 keys of one page or of the call an instruction
// group, into LDS rows whose 16-byte pieces are permuted (Rows in paged_bf16.h) so that both the key fragments (row pieces) and the value
// fragments (LDS transpose reads) touch every bank once.
//
// Two kernels.  Tiles: 4 waves of 32 or 64 rows share the keys of a ring of four stages of 32.  Few rows (at most 32 packed rows per
// sequence and cache head, so that nothing is shared): the waves of a workgroup take different keys, each through a ring of its own and
// without a barrier, and their results are joined at the end; bound by reading the cache once.
//
// Measured: three whole histories of up to 6000 tokens, 32 heads, d_head 128: 439 to 454 us from run to run, 915 to 945 TFLOP/s, and 525 us in
// a row of 22 calls, where the clock is at 1.8 GHz; the matrix pipe is busy in 43 % of the cycles.  A library product of random matrices reaches
// 1230 to 1270 TFLOP/s on this card and of zeros 1740: power is part of the limit.  One token of each of 64 sequences of 500 to
// 4000: 108 us for 581 MB, 5.4 TB/s.
#include "paged_state_bf16.h"

#include <type_traits>

namespace climber {
namespace {

using namespace paged;

// The new tokens of packed rows r0 .. r1 - 1 go into their pages.  (No call reads them from there before this one is done.)
template <int D>
static __device__ __forceinline__ void store_new(const PagedArgs &p, const PagedSeq &s, int b, int hk, int r0, int r1)
{
    constexpr int C = D / 8;
    const int t0 = (r0 + p.G - 1) / p.G, t1 = (r1 + p.G - 1) / p.G;
    for (int i = threadIdx.x; i < (t1 - t0) * C; i += 256) {
        const int t = t0 + i / C, c = (i % C) * 16, slot = s.n + t;
        if (slot >= p.max_len) break;
        const int page = p.table[(int64_t)b * p.table_ld + (slot >> p.page_shift)];
        if (page < 0 || page >= p.n_pages) continue;
        const int64_t to = paged_row(p, page, hk, slot) + c, from = (s.row0 + t) * p.ld_kv + (int64_t)hk * (2 * D) + c;
        *(uint4 *)(p.k_pages + to) = *(const uint4 *)(p.k + from);
        *(uint4 *)(p.v_pages + to) = *(const uint4 *)(p.v + from);
        if (hk == 0 && c == 0 && p.stamp) p.stamp[((int64_t)page << p.page_shift) + (slot & ((1 << p.page_shift) - 1))] = p.stamp_new[s.row0 + t];
    }
}

// ---- tiles ---------------------------------------------------------------------------------------
// 4 waves of QB x 32 packed rows over a ring of four stages of 32 keys.  Keys that every row of the tile sees go through a pipeline: while
// the exponentials of a block are made, the matrix pipe has the logits of the next one, and two more are on their way.  The rest (the diagonal
// of the causal mask, the end of the keys) block by block.  Two waves per SIMD, so 256 registers: QB = 2 at D = 64; at D = 128, where
// outputs and queries of 64 rows would be 192 of them, QB = 1.
template <int D, int QB, bool SUMI>
__global__ __launch_bounds__(256, 2) void attn_paged_tile_kernel(const PagedArgs p)
{
    using R = Rows<D>;
    constexpr int kRows = 128 * QB, kValues = 32 * R::kPitch, kStage = 2 * kValues;  // keys, then values
    constexpr int kShare = 8 * R::kPitch, kCopies = kShare / 1024;                   // a wave's part of either; copies of it
    // (four arrays: reads of one do not wait for copies into another)
    __shared__ __attribute__((aligned(1024))) uint8_t stage0[kStage], stage1[kStage], stage2[kStage], stage3[kStage];
    __shared__ int flags[4];
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
    const int n_blocks = (k_hi - k_lo + 31) / 32, n_clean = __builtin_amdgcn_readfirstlane(max(0, min(sees(r_tile), k_hi) - k_lo) / 32);

    const Source<D, kCopies> src(p, s, w.b, w.hk, k_hi, lane, (wave & 1) * kCopies);
    auto stage = [&](int i) __attribute__((always_inline)) { return (lds_u8 *)(i == 0 ? stage0 : i == 1 ? stage1 : i == 2 ? stage2 : stage3); };
    // this wave's 8 of the 32 keys of block i
    const int k_mine = k_lo + (wave >> 1) * 16;
    // page numbers of 64 of the wave's groups of 16 keys, one in each lane, and of the 64 after them
    const int first_pages = src.page_number(k_mine + lane * 32), next_pages = src.page_number(k_mine + (64 + lane) * 32);
    int pages = first_pages, pages_next = next_pages;
    auto issue = [&](int i, lds_u8 *to) __attribute__((always_inline)) {
        if ((i & 63) == 0 && i > 0) {
            pages = pages_next;
            pages_next = src.page_number(k_mine + (i + 64 + lane) * 32);
        }
        src.issue(k_mine + i * 32, __builtin_amdgcn_readlane(pages, i & 63), to + wave * kShare, to + kValues + wave * kShare);
    };
    Rows<D> at;
    at.init(lane);
    State<D, QB> st;
    auto start = [&]() __attribute__((always_inline)) {
        typename State<D, QB>::Row in[QB];
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            const int r = min(r_wave + qb * 32 + l32, rows - 1);
            st.template request<SUMI>(p, qb, s.row0 + r / p.G, w.hk * p.G + r % p.G, w.hk, hf, in[qb]);
        }
        if (n_blocks > 0) issue(0, stage(0));
        if (n_blocks > 1) issue(1, stage(1));
        if (n_blocks > 2) issue(2, stage(2));
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) st.template start<SUMI>(p, qb, hf, in[qb], w.split == 0);
    };
    if (!SUMI && w.split == 0) store_new<D>(p, s, w.b, w.hk, r_tile, min(r_tile + kRows, rows));

    // this wave's copies have landed but for those of `later` blocks, the last ones issued
    auto landed = [&](int later) __attribute__((always_inline)) {
        static_assert(kCopies == 1 || kCopies == 2, "vmcnt immediates");
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
    int top[QB];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) top[qb] = min(sees(r_wave + qb * 32 + l32), k_hi);
    const int wave_hi = min(sees(r_wave + 32 * QB - 1), k_hi);
    bool odd = false, far[QB];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) far[qb] = false;
    // (one copy of the start's code at D = 128, where a second makes the loop spill; two at D = 64, where one costs the loop 5 %)
    if constexpr (D == 64) start();
#pragma unroll 1
    for (bool again = false;; again = true) {
        if constexpr (D != 64) start();
        if (!again && n_clean > 0) {
            f32x16 S0[QB], S1[QB];
            bf16x8 P[QB][2];
            landed(min(n_blocks - 1, 2));
            meet();
            st.logits(read_k<D>(at, stage(0)), S0);
            st.reference(S0);
            // block j: its logits in Sc, values in cur; the next one's keys in next; prev is free
            auto step = [&](int j, f32x16 (&Sc)[QB], f32x16 (&Sn)[QB], lds_u8 *prev, lds_u8 *cur, lds_u8 *next) __attribute__((always_inline)) {
                landed(min(1, n_blocks - 2 - j));
                meet();  // block j + 1 is here, and nobody reads block j - 1 any more
                if (j + 3 < n_blocks) issue(j + 3, prev);
                const KFrags<D> k = read_k<D>(at, next);
                __builtin_amdgcn_sched_barrier(0);
                st.weights(Sc, P, 0);
                __builtin_amdgcn_sched_barrier(0);
                st.logits(k, Sn);  // (behind the last block: not used)
                st.weights(Sc, P, 1);
                const VFrags<D> v0 = read_v<D>(at, cur + kValues), v1 = read_v<D>(at, cur + kValues + 16 * R::kPitch);
                __builtin_amdgcn_sched_barrier(0x40f);
                st.add(v0, P, 0);
                st.add(v1, P, 1);
            };
            for (int j = 0; j < n_clean;) {
                step(j, S0, S1, stage(3), stage(0), stage(1));
                if (++j == n_clean) break;
                step(j, S1, S0, stage(0), stage(1), stage(2));
                if (++j == n_clean) break;
                step(j, S0, S1, stage(1), stage(2), stage(3));
                if (++j == n_clean) break;
                step(j, S1, S0, stage(2), stage(3), stage(0));
                ++j;
            }
            // (now, and at the end: in the blocks to come the reference may move by more than 2^126, which makes zeros of the sums so far)
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) far[qb] = !(st.l[qb] + other_half(st.l[qb]) < kFar);
        }
        // blocks that not every row sees whole
#pragma unroll 1
        for (int j = again ? 0 : n_clean; j < n_blocks; ++j) {
            lds_u8 *cur = stage(j & 3);
            landed(min(2, n_blocks - 1 - j));
            if (j >= n_clean) odd |= clear_odd<kShare>(cur + kValues + wave * kShare, lane);
            meet();
            if (j + 3 < n_blocks) issue(j + 3, stage((j + 3) & 3));
            const int k0 = k_lo + j * 32;
            if (k0 >= wave_hi) continue;
            f32x16 S[QB];
            bf16x8 P[QB][2];
            bool may[QB];
            st.logits(read_k<D>(at, cur), S);
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) {
                hide(S[qb], k0, hf, top[qb]);
                may[qb] = j >= n_clean || j == 0 || far[qb];
            }
            st.reference(S, may);
            st.weights(S, P);
#pragma unroll
            for (int g = 0; g < 2; ++g) st.add(read_v<D>(at, cur + kValues + g * 16 * R::kPitch), P, g);
        }
        if (again || n_clean == 0) break;
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
        pages = first_pages, pages_next = next_pages;
        odd = false;
        if constexpr (D == 64) start();
    }

    store_tile<D>(p, s, w, st, r_wave, rows);
    if (lane == 0) flags[wave] = odd;
    __syncthreads();
    if (__builtin_expect(flags[0] | flags[1] | flags[2] | flags[3], 0))
        put_odd<D>(p, s, w, k_lo + n_clean * 32, k_hi, r_wave, min(r_wave + 32 * QB, rows), sees);
}

// ---- few rows ------------------------------------------------------------------------------------
// (workgroups of a CU: as many as there is LDS for)
template <int D, bool SUMI>
__global__ __launch_bounds__(256, D == 64 ? 2 : 1) void attn_paged_few_kernel(const PagedArgs p)
{
    using R = Rows<D>;
    constexpr int kStage = 2 * 32 * R::kPitch, kLoads = 4 * R::kLoads;  // a wave's
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
    const int lim = sees(r), lim_lo = sees(r_tile);
    int k_lo, k_hi;
    paged_part(p, w.split, sees(r_tile + 31), 128, k_lo, k_hi);
    k_lo = __builtin_amdgcn_readfirstlane(k_lo), k_hi = __builtin_amdgcn_readfirstlane(k_hi);
    const int n_blk = (k_hi - k_lo + 31) / 32, mine = n_blk > wave ? (n_blk - wave + 3) / 4 : 0;  // blocks wave, wave + 4, ...

    const Source<D, R::kLoads> src(p, s, w.b, w.hk, k_hi, lane, 0);
    lds_u8 *const at0 = (lds_u8 *)stage0 + wave * kStage, *const at1 = (lds_u8 *)stage1 + wave * kStage;
    // groups of 16 keys: blocks wave, wave + 4, ... of 32; the lower 32 lanes look up the first groups of 32 blocks, the upper the second
    const int k_mine = k_lo + wave * 32 - (lane >> 5) * (32 * 128 - 16);
    int pages = src.page_number(k_mine + lane * 128), pages_next = src.page_number(k_mine + (32 + lane) * 128);
    auto issue = [&](int i, lds_u8 *to) __attribute__((always_inline)) {
        if ((i & 31) == 0 && i > 0) {
            pages = pages_next;
            pages_next = src.page_number(k_mine + (i + 32 + lane) * 128);
        }
        const int k0 = k_lo + (i * 4 + wave) * 32;
        src.issue(k0, __builtin_amdgcn_readlane(pages, i & 31), to, to + 32 * R::kPitch);
        src.issue(k0 + 16, __builtin_amdgcn_readlane(pages, 32 + (i & 31)), to + 16 * R::kPitch, to + 48 * R::kPitch);
    };
    Rows<D> at;
    at.init(lane);
    State<D, 1> st;
    {
        typename State<D, 1>::Row in;
        st.template request<SUMI>(p, 0, row, h, w.hk, hf, in);
        if (mine > 0) issue(0, at0);
        if (mine > 1) issue(1, at1);
        st.template start<SUMI>(p, 0, hf, in, w.split == 0 && wave == 0);
    }
    if (!SUMI && w.split == 0) store_new<D>(p, s, w.b, w.hk, r_tile, min(r_tile + 32, rows));

    // logits for the weights per token
    float *const logits = p.logits ? p.logits + (((int64_t)w.b * p.Hkv + w.hk) * (p.m_max * p.G) + r_tile + l32) * p.logits_ld + 4 * hf : nullptr;
    auto keep = [&](const f32x16 &S, int k0) __attribute__((always_inline)) {
        if (logits && r_tile + l32 < rows) {
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *(f32x4 *)(logits + k0 + 8 * g) = f32x4{S[4 * g] * st.c[0], S[4 * g + 1] * st.c[0], S[4 * g + 2] * st.c[0], S[4 * g + 3] * st.c[0]};
        }
    };
    bool odd = false;
    auto block = [&](int i, lds_u8 *keys) __attribute__((always_inline)) {
        // (the rows and stores above were issued later than the first copies: until they are done, this waits for more than it has to)
        static_assert(kLoads == 16 || kLoads == 8, "vmcnt immediates");
        if (i + 1 < mine) {
            if constexpr (kLoads == 16) asm volatile("s_waitcnt vmcnt(16)" ::: "memory");
            else asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
        } else {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        }
        lds_u8 *const values = keys + 32 * R::kPitch;
        const int k0 = k_lo + (i * 4 + wave) * 32;
        f32x16 S[1];
        bf16x8 P[1][2];
        st.logits(read_k<D>(at, keys), S);
        if (k0 + 32 <= min(lim_lo, k_hi)) {
            keep(S[0], k0);
            st.reference(S);
            st.weights(S, P);
#pragma unroll
            for (int g = 0; g < 2; ++g) st.add(read_v<D>(at, values + g * 16 * R::kPitch), P, g);
        } else {
            odd |= clear_odd<32 * R::kPitch>(values, lane);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            hide(S[0], k0, hf, min(lim, k_hi));
            keep(S[0], k0);
            st.reference(S);
            st.weights(S, P);
#pragma unroll
            for (int g = 0; g < 2; ++g) st.add(read_v<D>(at, values + g * 16 * R::kPitch), P, g);
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

    if (lane == 0) odd_seen[wave] = odd;
    join_few<D>(p, s, w, st, joined, [&](int j) { return (float *)stage0 + j * 32 * D; }, row, h, r_tile, rows);
    if (__builtin_expect(odd_seen[0] | odd_seen[1] | odd_seen[2] | odd_seen[3], 0)) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // all waves' outputs are written
        __syncthreads();
        if (wave == 0) put_odd<D>(p, s, w, k_lo + max(0, min(lim_lo, k_hi) - k_lo) / 32 * 32, k_hi, r_tile, min(r_tile + 32, rows), sees);
    }
}

template <int D, bool SUMI>
hipError_t launch(PagedArgs p, hipStream_t s)
{
    const int64_t rows = (int64_t)p.m_max * p.G;
    const int tile = paged_tile_rows(true, D, rows, (int64_t)p.n_seqs * p.Hkv);
    void (*kernel)(PagedArgs) = tile == 32 ? attn_paged_few_kernel<D, SUMI> : attn_paged_tile_kernel<D, 1, SUMI>;
    if constexpr (D == 64)
        if (tile == 256) kernel = attn_paged_tile_kernel<D, 2, SUMI>;
    p.n_tiles = (int)((rows + tile - 1) / tile);
    hipLaunchKernelGGL(kernel, dim3(paged_grid(p)), dim3(256), 0, s, p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_attn_paged_bf16(const PagedArgs &a, hipStream_t s)
{
    if (a.d == 64) return a.sumi ? launch<64, true>(a, s) : launch<64, false>(a, s);
    return a.sumi ? launch<128, true>(a, s) : launch<128, false>(a, s);
}

}  // namespace climber
