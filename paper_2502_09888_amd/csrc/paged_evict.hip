// Eviction from the paged history cache by accumulated attention weight (gfx950).
//
// Every sequence keeps `keep` = min(budget, len) of its tokens: those that rank first are the ones with stamp >= keep_from, then by
// rank descending, then by slot ascending.  The cache of a sequence is a set (attention does not depend on the order of the
// cached tokens), so only what has to is moved: the kept tokens of slots >= keep go, in order, into the slots < keep whose token is
// evicted.  There are equally many of both, no slot is read and written, and a step that evicts one token moves at most one.
//
// Two launches.  select: a workgroup per sequence finds the last kept token's rank by a radix selection over the order-preserving
// bits of the ranks, 11 + 11 + 10 bits a pass, and lists holes and movers.  move: 16 bytes a thread, bound by memory.
#include "paged.h"

#include <algorithm>

namespace climber {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64, kBins = 2048;

// unsigned integers in the order of the floats; -0 is 0, a NaN ranks below everything
static __device__ __forceinline__ uint32_t order_bits(float x)
{
    if (x != x) return 0;
    const uint32_t u = __float_as_uint(x + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

static __device__ __forceinline__ int below(uint64_t mask, int lane) { return __popcll(mask & ((1ull << lane) - 1)); }

__global__ __launch_bounds__(kThreads) void evict_select_kernel(const EvictArgs p)
{
    __shared__ int hist[kBins], wave_n[2][kWaves], chosen[2];
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n = min(max(p.len[b], 0), p.max_len), keep = min(max(p.budget[b], 0), n);
    const int words = (p.max_len + 63) / 64;
    uint32_t *keys = p.keys + (int64_t)b * p.max_len;
    uint64_t *first = p.first + (int64_t)b * words;
    int32_t *holes = p.holes + (int64_t)b * (p.max_len / 2 + 1), *movers = p.movers + (int64_t)b * (p.max_len / 2 + 1);
    const int src_ld = p.table_ld << p.page_shift;
    int32_t *src = p.src ? p.src + (int64_t)b * src_ld : nullptr;
    if (p.src)
        for (int i = tid; i < src_ld; i += kThreads) src[i] = i < keep ? i : -1;
    __syncthreads();  // (len_out may be len)
    if (tid == 0) p.len_out[b] = keep;
    if (keep == n || keep == 0) {
        if (tid == 0) p.n_moves[b] = 0;
        return;
    }

    // a wave's share of the slots: whole words of 64, in order
    const int n_words = (n + 63) / 64, per = (n_words + kWaves - 1) / kWaves, w0 = min(wave * per, n_words), w1 = min(w0 + per, n_words);
    const int limit = p.keep_from ? p.keep_from[b] : 0;
    int n_first = 0;
    for (int w = w0; w < w1; ++w) {
        const int i = w * 64 + lane;
        bool is_first = false;
        if (i < n) {
            const int page = min(max(p.table[(int64_t)b * p.table_ld + (i >> p.page_shift)], 0), p.n_pages - 1);
            const int64_t at = ((int64_t)page << p.page_shift) + (i & ((1 << p.page_shift) - 1));
            keys[i] = order_bits(p.rank[at]);
            is_first = p.keep_from && p.stamp[at] >= limit;
        }
        const uint64_t m = __builtin_amdgcn_ballot_w64(is_first);
        if (lane == 0) first[w] = m;
        n_first += __popcll(m);
    }
    if (lane == 0) wave_n[0][wave] = n_first;
    __syncthreads();
    n_first = 0;
    for (int w = 0; w < kWaves; ++w) n_first += wave_n[0][w];
    // the tokens among which the cut lies, and how many of them are kept; the others are all kept, or all evicted
    const bool among_first = n_first >= keep;
    int need = among_first ? keep : keep - n_first;
    auto contested = [&](int w) { return among_first ? first[w] : ~first[w]; };

    // radix selection of the need-th largest; prefix: the bits of it that are known
    uint32_t prefix = 0, known = 0;
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
        __syncthreads();
        for (int i = tid; i < kBins; i += kThreads) hist[i] = 0;
        __syncthreads();
        for (int w = w0; w < w1; ++w) {
            const int i = w * 64 + lane;
            if (i < n && (contested(w) >> lane & 1)) {
                const uint32_t k = keys[i];
                if ((k & known) == prefix) atomicAdd(&hist[k >> shift & ((1 << bits) - 1)], 1);
            }
        }
        __syncthreads();
        if (wave == 0) {  // from the highest bin down: lane 0 has the highest 32
            int sum = 0;
            for (int j = 0; j < kBins / 64; ++j) sum += hist[kBins - 1 - (lane * (kBins / 64) + j)];
            int before = sum;  // inclusive prefix over the lanes
            for (int o = 1; o < 64; o *= 2) {
                const int x = __shfl_up(before, o, 64);
                if (lane >= o) before += x;
            }
            before -= sum;
            if (before < need && need <= before + sum) {
                for (int j = 0; j < kBins / 64; ++j) {
                    const int bin = kBins - 1 - (lane * (kBins / 64) + j);
                    if (need <= before + hist[bin]) {
                        chosen[0] = bin;
                        chosen[1] = need - before;
                        break;
                    }
                    before += hist[bin];
                }
            }
        }
        __syncthreads();
        prefix |= (uint32_t)chosen[0] << shift;
        known |= ((1u << bits) - 1) << shift;
        need = chosen[1];
    }
    // contested tokens above `prefix` are kept, and of those that equal it the first `need`
    int equal = 0;
    for (int w = w0; w < w1; ++w) {
        const int i = w * 64 + lane;
        equal += __popcll(__builtin_amdgcn_ballot_w64(i < n && (contested(w) >> lane & 1) && keys[i] == prefix));
    }
    __syncthreads();
    if (lane == 0) wave_n[0][wave] = equal;
    __syncthreads();
    int equal0 = 0;
    for (int w = 0; w < wave; ++w) equal0 += wave_n[0][w];
    auto walk = [&](auto each) {
        int eq = equal0;
        for (int w = w0; w < w1; ++w) {
            const int i = w * 64 + lane;
            const bool c = contested(w) >> lane & 1;
            const uint32_t k = i < n ? keys[i] : 0;
            const uint64_t same = __builtin_amdgcn_ballot_w64(i < n && c && k == prefix);
            const bool kept = i < n && (c ? k > prefix || (k == prefix && eq + below(same, lane) < need) : !among_first);
            eq += __popcll(same);
            each(i, __builtin_amdgcn_ballot_w64(i < keep && !kept), __builtin_amdgcn_ballot_w64(i >= keep && kept));
        }
    };
    int n_holes = 0, n_movers = 0;
    walk([&](int, uint64_t hole, uint64_t mover) {
        n_holes += __popcll(hole);
        n_movers += __popcll(mover);
    });
    __syncthreads();
    if (lane == 0) wave_n[0][wave] = n_holes, wave_n[1][wave] = n_movers;
    __syncthreads();
    int hole0 = 0, mover0 = 0, all = 0;
    for (int w = 0; w < kWaves; ++w) {
        if (w < wave) hole0 += wave_n[0][w], mover0 += wave_n[1][w];
        all += wave_n[0][w];
    }
    walk([&](int i, uint64_t hole, uint64_t mover) {
        if (hole >> lane & 1) holes[hole0 + below(hole, lane)] = i;
        if (mover >> lane & 1) movers[mover0 + below(mover, lane)] = i;
        hole0 += __popcll(hole);
        mover0 += __popcll(mover);
    });
    if (tid == 0) p.n_moves[b] = all;
    if (p.src) {
        __threadfence_block();
        __syncthreads();
        for (int i = tid; i < all; i += kThreads) src[holes[i]] = movers[i];
    }
}

__global__ __launch_bounds__(256) void evict_move_kernel(const EvictArgs p, int per_seq)
{
    const int b = blockIdx.x / per_seq, part = blockIdx.x % per_seq, n = p.n_moves[b];
    const int32_t *holes = p.holes + (int64_t)b * (p.max_len / 2 + 1), *movers = p.movers + (int64_t)b * (p.max_len / 2 + 1);
    const int32_t *table = p.table + (int64_t)b * p.table_ld;
    const int C = p.row_bytes / 16, in_page = (1 << p.page_shift) - 1;
    const int64_t items = (int64_t)n * p.Hkv * C;
    for (int64_t i = (int64_t)part * 256 + threadIdx.x; i < items; i += (int64_t)per_seq * 256) {
        const int c = (int)(i % C), h = (int)(i / C % p.Hkv), m = (int)(i / C / p.Hkv), to = holes[m], from = movers[m];
        const int tp = table[to >> p.page_shift], fp = min(max(table[from >> p.page_shift], 0), p.n_pages - 1);
        if (tp < 0 || tp >= p.n_pages) continue;
        const int64_t t = ((((int64_t)tp * p.Hkv + h) << p.page_shift) + (to & in_page)) * p.row_bytes + c * 16;
        const int64_t f = ((((int64_t)fp * p.Hkv + h) << p.page_shift) + (from & in_page)) * p.row_bytes + c * 16;
        *(uint4 *)(p.k_pages + t) = *(const uint4 *)(p.k_pages + f);
        *(uint4 *)(p.v_pages + t) = *(const uint4 *)(p.v_pages + f);
        if (h == 0 && c == 0) {
            const int64_t ts = ((int64_t)tp << p.page_shift) + (to & in_page), fs = ((int64_t)fp << p.page_shift) + (from & in_page);
            if (p.mass) p.mass[ts] = p.mass[fs];
            if (p.stamp) p.stamp[ts] = p.stamp[fs];
        }
    }
}

}  // namespace

hipError_t launch_paged_evict(const EvictArgs &a, hipStream_t s)
{
    hipLaunchKernelGGL(evict_select_kernel, dim3((unsigned)a.n_seqs), dim3(kThreads), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t items = (int64_t)(a.max_len / 2 + 1) * a.Hkv * (a.row_bytes / 16);  // the most that a sequence can have
    const int per = (int)std::max<int64_t>(1, std::min<int64_t>((items + 255) / 256, 4096 / a.n_seqs));
    hipLaunchKernelGGL(evict_move_kernel, dim3((unsigned)(per * a.n_seqs)), dim3(256), 0, s, a, per);
    return hipGetLastError();
}

}  // namespace climber
