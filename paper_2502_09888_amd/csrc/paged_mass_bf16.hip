// Attention weights per token of the paged history cache, bf16 (gfx950): how much of all softmaxes of a call falls on each cached token,
// sum over rows and query heads of p = exp2(s c - lse) with the logits made again (Eq. (3) of Climber, arXiv 2502.09888).
//
// One workgroup = 256 keys of one (sequence, cache head) and a part of its packed rows.  A wave keeps the fragments of its 64 keys
// in registers and adds up 64 sums a lane; the rows pass by in LDS, 64 at a time in a ring of two stages.  No atomics: sums are made in the
// order of the rows, then of the lanes, and a second kernel adds up cache heads and parts in theirs.
//
// Bound by the products and by what a logit costs beside them (a multiply-add, an exponential and an addition: 14 cycles of a SIMD for 64
// logits, of products 16 at d_head 64 and 32 at 128), which waves of one SIMD overlap only in part: 72 us for 2.7e8 logits of d_head 64 (512
// candidates of each of 64 users on 1024 tokens, 8 heads), beside 105 of their attention.  Logits left by the attention instead would be
// 4 bytes each, written and read, 420 us.  The next block's products beside this one's exponentials in the same wave took 4 to 9 % more (two
// waves a SIMD instead of three), stages of 128 rows the same.
#include "paged_bf16.h"

namespace climber {
namespace {

using namespace paged;

constexpr int kRowsStage = 64;

template <int D>
__global__ __launch_bounds__(256, D == 64 ? 3 : 2) void paged_mass_bf16_kernel(const PagedArgs p, float *part)
{
    using R = Rows<D>;
    constexpr int kStage = kRowsStage * R::kPitch, kLoads = kStage / 1024 / 4;  // (a wave's)
    __shared__ __attribute__((aligned(1024))) uint8_t stage0[kStage], stage1[kStage];
    const int lane = threadIdx.x & 63, l32 = lane & 31, hf = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    PagedWork w;
    PagedSeq s;
    if (!paged_work(p, w, s)) return;
    const int keys = paged_keys(p, s), k_tile = w.tile * kMassKeys, k0 = k_tile + wave * 64, rows = s.T * p.G;
    if (k_tile >= keys || rows == 0) return;
    const bool causal = !p.sumi && p.causal;
    // this part's rows, from the first one that sees a key of the tile
    const int first = causal ? max(0, k_tile - s.n) * p.G : 0, per = ((rows + p.n_split - 1) / p.n_split + kRowsStage - 1) / kRowsStage * kRowsStage;
    const int r_lo = max(w.split * per, first / kRowsStage * kRowsStage), r_hi = min((w.split + 1) * per, rows);
    const int n_stages = __builtin_amdgcn_readfirstlane(max(0, r_hi - r_lo + kRowsStage - 1) / kRowsStage);

    auto token_of = [&](int r) __attribute__((always_inline)) {  // r / G
        const int t = (int)__umulhi((unsigned)r, p.G_inv);
        return p.G == 1 ? r : t - (t * p.G > r);
    };
    // Where a row lies: of its query (this lane's piece, for each copy), and of its statistics.  From stage to stage they move by 64 rows, which
    // is next_t tokens and next_h heads; rows behind the last are read as the last.
    const int next_t = kRowsStage / p.G, next_h = kRowsStage % p.G;
    int head[kLoads], stat_head[2];
    const uint8_t *from[kLoads];
    const float2 *stat[2];
    auto place = [&](int r0) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int in = (wave * kLoads + j) * R::kPerLoad + lane / R::kPieces, r = min(r0 + in, rows - 1), t = token_of(r);
            const int c = (lane % R::kPieces) ^ R::f(in);
            head[j] = r - t * p.G;
            from[j] = p.q + (s.row0 + t) * p.ld_q + (int64_t)(w.hk * p.G + head[j]) * R::kPitch + c * 16;
        }
#pragma unroll
        for (int blk = 0; blk < 2; ++blk) {
            const int r = min(r0 + blk * 32 + l32, rows - 1), t = token_of(r);
            stat_head[blk] = r - t * p.G;
            stat[blk] = p.lse + (s.row0 + t) * p.H + w.hk * p.G + stat_head[blk];
        }
    };
    const int64_t q_step = next_t * p.ld_q + next_h * R::kPitch, q_wrap = p.ld_q - p.G * R::kPitch;
    const int stat_step = next_t * p.H + next_h, stat_wrap = p.H - p.G;
    auto advance = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            head[j] += next_h;
            const bool over = head[j] >= p.G;
            head[j] -= over ? p.G : 0;
            from[j] += q_step + (over ? q_wrap : 0);
        }
#pragma unroll
        for (int blk = 0; blk < 2; ++blk) {
            stat_head[blk] += next_h;
            const bool over = stat_head[blk] >= p.G;
            stat_head[blk] -= over ? p.G : 0;
            stat[blk] += stat_step + (over ? stat_wrap : 0);
        }
    };
    float2 next[2];
    auto issue = [&](lds_u8 *to) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) copy16((glb_u8 *)from[j], to + (wave * kLoads + j) * 1024);
#pragma unroll
        for (int blk = 0; blk < 2; ++blk) next[blk] = *stat[blk];
    };
    if (n_stages > 0) {
        place(r_lo);
        issue((lds_u8 *)stage0);
    }
    KFrags<D> k[2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
        const int j = min(k0 + kb * 32 + l32, keys - 1);
        const uint8_t *from = j < s.n ? p.k_pages + paged_row(p, paged_page(p, w.b, j), w.hk, j)
                                      : p.k + (s.row0 + j - s.n) * p.ld_kv + (int64_t)w.hk * R::kPitch;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) k[kb].a[i] = *(const bf16x8 *)(from + i * 32 + hf * 16);
    }
    // (they have arrived: else every use in the loop would wait for whatever was requested last)
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < D / 16; ++i) asm volatile("" : "+v"(k[kb].a[i]));
    Rows<D> at;
    at.init(lane);
    f32x16 sum[2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) sum[kb][i] = 0.f;

    auto stage = [&](int i, lds_u8 *cur, lds_u8 *other) __attribute__((always_inline)) {
        // this stage's copies have landed, and this wave's reads of the stage before, which is filled again behind the barrier, are done
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        float2 now[2] = {next[0], next[1]};
        asm volatile("" : "+v"(now[0].x), "+v"(now[0].y), "+v"(now[1].x), "+v"(now[1].y));
        if (i + 1 < n_stages) {
            const int r1 = r_lo + (i + 1) * kRowsStage;
            if (r1 + kRowsStage <= rows) advance();
            else place(r1);
            issue(other);
        }
#pragma unroll
        for (int blk = 0; blk < 2; ++blk) {
            const int r0 = r_lo + i * kRowsStage + blk * 32;
            if (r0 >= r_hi) break;
            const KFrags<D> q = read_k<D>(at, cur + blk * 32 * R::kPitch);
            f32x16 S[2];
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
                for (int e = 0; e < 16; ++e) S[kb][e] = 0.f;
#pragma unroll
                for (int e = 0; e < D / 16; ++e) S[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[kb].a[e], q.a[e], S[kb], 0, 0, 0);
            }
            const float c = now[blk].x, lse = now[blk].y;
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int e = 0; e < 16; ++e) S[kb][e] = __builtin_amdgcn_exp2f(fmaf(S[kb][e], c, -lse));
            if (r0 + 32 > rows || (causal && k0 + 63 > s.n + __builtin_amdgcn_readfirstlane(token_of(r0)))) {
                const int lim = (r0 + l32 >= rows ? 0 : causal ? s.n + token_of(r0 + l32) + 1 : keys) - k0 - 4 * hf;
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (kb * 32 + 8 * (e >> 2) + (e & 3) >= lim) S[kb][e] = 0.f;
            }
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int e = 0; e < 16; ++e) sum[kb][e] += S[kb][e];
        }
    };
    for (int i = 0; i < n_stages; i += 2) {
        stage(i, (lds_u8 *)stage0, (lds_u8 *)stage1);
        if (i + 1 < n_stages) stage(i + 1, (lds_u8 *)stage1, (lds_u8 *)stage0);
    }
    // over the 32 lanes that have other rows of the same keys
    float *to = part + (((int64_t)w.b * p.Hkv + w.hk) * p.n_split + w.split) * p.max_len;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            float x = row_sum16(sum[kb][e]);
            x += __shfl_xor(x, 16, 64);
            const int j = k0 + kb * 32 + 8 * (e >> 2) + 4 * hf + (e & 3);
            if (l32 == 0 && j < keys) to[j] = x;
        }
}

}  // namespace

hipError_t launch_paged_mass_bf16(const PagedArgs &a, float *part, int row_parts, hipStream_t s)
{
    PagedArgs p = a;
    p.n_split = row_parts;
    p.n_tiles = (a.max_len + kMassKeys - 1) / kMassKeys;
    if (a.d == 64) hipLaunchKernelGGL(paged_mass_bf16_kernel<64>, dim3(paged_grid(p)), dim3(256), 0, s, p, part);
    else hipLaunchKernelGGL(paged_mass_bf16_kernel<128>, dim3(paged_grid(p)), dim3(256), 0, s, p, part);
    return hipGetLastError();
}

}  // namespace climber
