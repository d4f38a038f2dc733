// Eviction from the paged history cache by accumulated attention weight (gfx950).
//
// Every sequence keeps `keep` = min(budget, len) of its tokens: those that rank first are the ones with stamp >= keep_from, then by
// rank descending, then by slot ascending.  The cache of a sequence is a set (attention does not depend on the order of the
// cached tokens), so only what has to is moved: the kept tokens of slots >= keep go, in order, into the slots < keep whose token is
// evicted.  There are equally many of both, no slot is read and written, and a step that evicts one token moves at most one.
//
// The last kept token is found by a radix selection over the order-preserving bits of the ranks, 11 + 11 + 10 bits a pass, among the
// tokens that the cut lies in (those with a stamp that counts, or the others); of the tokens that equal it the first are kept.
// Up to 16384 tokens a sequence: one workgroup each, whose threads keep their keys.  Longer ones: a workgroup per 4096 tokens, in four
// launches (a pass each needs the histograms of all; one workgroup for 98765 tokens took 380 us).  Then the move, 16 bytes a
// thread.  98765 tokens of 8 heads of 128 cut to 50000, 206 MB moved: 44 us for all five launches on one cache again and again, most of which then
// lies in the last-level cache, and 83 on two caches in turn, the move 40 of them (5.1 TB/s: memory) and the steps 9 to 13 each; 64 sequences
// of up to 4096 cut to 2048, 270 MB: 32 and 46, the selection 9 of them, bound by its trips to memory and the barriers of its passes.
#include "paged.h"

#include <algorithm>
#include <type_traits>

namespace climber {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64, kBins = 2048;
constexpr int kShift[3] = {21, 10, 0}, kMask[3] = {2047, 2047, 1023};
static_assert(kEvictSegInts >= 4 * kBins + 3 && kEvictMostSegments <= kBins, "a segment's histograms and counts; steps keep counts of all segments");

// unsigned integers in the order of the floats; -0 is 0, a NaN ranks below everything
static __device__ __forceinline__ uint32_t order_bits(float x)
{
    if (x != x) return 0;
    const uint32_t u = __float_as_uint(x + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
static __device__ __forceinline__ int below(uint64_t mask, int lane) { return __popcll(mask & ((1ull << lane) - 1)); }

static __device__ __forceinline__ int64_t token_at(const EvictArgs &p, int b, int slot)
{
    const int page = min(max(p.table[(int64_t)b * p.table_ld + (slot >> p.page_shift)], 0), p.n_pages - 1);
    return ((int64_t)page << p.page_shift) + (slot & ((1 << p.page_shift) - 1));
}

// inclusive sum over the lanes, by DPP: row_shr 1, 2, 4, 8, then each row's last lane to the rows behind it
static __device__ __forceinline__ int sum_to_me(int x)
{
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // lane 15 and 47 of the rows before
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // lane 31
    return x;
}

// exclusive sum over the threads of a workgroup, in their order (one barrier; `room` is free again after the next one)
static __device__ __forceinline__ int before_me(int x, int *room, int lane, int wave)
{
    const int sum = sum_to_me(x);
    if (lane == 63) room[wave] = sum;
    __syncthreads();
    int at = sum - x;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) at += w < wave ? room[w] : 0;
    return at;
}

// The bin in which the need-th largest lies (bins counted from the highest down; this thread has two) -> chosen = {bin, how many of it, of
// how many}; ends without a barrier.
static __device__ __forceinline__ void choose(int high, int low, int need, int *room, int *chosen, int tid)
{
    const int at = before_me(high + low, room, tid & 63, tid >> 6), bin = kBins - 1 - 2 * tid;
    if (at < need && need <= at + high) chosen[0] = bin, chosen[1] = need - at, chosen[2] = high;
    else if (at + high < need && need <= at + high + low) chosen[0] = bin - 1, chosen[1] = need - at - high, chosen[2] = low;
}

// ---- one workgroup per sequence, K words of 64 tokens a wave ---------------------------------------
template <int K>
__global__ __launch_bounds__(kThreads) void evict_select_kernel(const EvictArgs p)
{
    __shared__ int hist[3][kBins], room[3][kWaves], count[4][kWaves], chosen[3][3], movers_lds[K * kThreads / 2];
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n = min(max(p.len[b], 0), p.max_len), keep = min(max(p.budget[b], 0), n);
    const int limit = p.keep_from ? p.keep_from[b] : 0;
    int32_t *holes = p.holes + (int64_t)b * (p.max_len / 2 + 1), *movers = p.movers + (int64_t)b * (p.max_len / 2 + 1);
    const int src_ld = p.table_ld << p.page_shift;
    int32_t *src = p.src ? p.src + (int64_t)b * src_ld : nullptr;
    const int i0 = wave * K * 64 + lane;  // this thread's slots: i0 + 64 j
    auto write_src = [&](auto from) {
        if (!src) return;
#pragma unroll
        for (int j = 0; j < K; ++j)
            if (i0 + 64 * j < src_ld) src[i0 + 64 * j] = from(j, i0 + 64 * j);
        for (int i = K * kThreads + tid; i < src_ld; i += kThreads) src[i] = -1;
    };
    uint32_t key[K];
    uint64_t first[K];
    int n_first = 0;
#pragma unroll
    for (int j = 0; j < K; ++j) {  // (what lies behind the last token is read, before the length is known, and not used)
        const int i = i0 + 64 * j;
        const int64_t at = token_at(p, b, max(min(i, p.max_len - 1), 0));
        key[j] = order_bits(p.rank[at]);
        const int32_t stamp = p.keep_from ? p.stamp[at] : 0;
        first[j] = __builtin_amdgcn_ballot_w64(i < n && p.keep_from && stamp >= limit);
        n_first += __popcll(first[j]);
    }
    for (int i = tid; i < 3 * kBins; i += kThreads) hist[0][i] = 0;
    if (lane == 0) count[0][wave] = n_first;
    __syncthreads();  // (len_out may be len: everybody has read it)
    if (tid == 0) p.len_out[b] = keep;
    if (keep == n || keep == 0) {
        if (tid == 0) p.n_moves[b] = 0;
        write_src([&](int, int i) { return i < keep ? i : -1; });
        return;
    }
    n_first = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) n_first += count[0][w];
    // the tokens among which the cut lies, and how many of them are kept; the others are all kept, or all evicted
    const bool among_first = n_first >= keep;
    int need = among_first ? keep : keep - n_first;
    bool contested[K];
#pragma unroll
    for (int j = 0; j < K; ++j) contested[j] = i0 + 64 * j < n && ((first[j] >> lane & 1) != 0) == among_first;
    uint32_t prefix = 0, known = 0;
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
#pragma unroll
        for (int j = 0; j < K; ++j)
            if (contested[j] && (key[j] & known) == prefix) atomicAdd(&hist[pass][key[j] >> kShift[pass] & kMask[pass]], 1);
        __syncthreads();
        choose(hist[pass][kBins - 1 - 2 * tid], hist[pass][kBins - 2 - 2 * tid], need, room[pass], chosen[pass], tid);
        __syncthreads();
        prefix |= (uint32_t)chosen[pass][0] << kShift[pass];
        known |= (uint32_t)kMask[pass] << kShift[pass];
        need = chosen[pass][1];
        if (need == chosen[pass][2]) break;  // all of the bin: no matter what their other bits are
    }
#pragma unroll
    for (int j = 0; j < K; ++j) key[j] &= known;
    int equal = 0;
#pragma unroll
    for (int j = 0; j < K; ++j) equal += __popcll(__builtin_amdgcn_ballot_w64(contested[j] && key[j] == prefix));
    if (lane == 0) count[1][wave] = equal;
    __syncthreads();
    equal = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) equal += w < wave ? count[1][w] : 0;
    uint64_t hole[K], mover[K];
    int n_holes = 0, n_movers = 0;
#pragma unroll
    for (int j = 0; j < K; ++j) {
        const int i = i0 + 64 * j;
        const uint64_t same = __builtin_amdgcn_ballot_w64(contested[j] && key[j] == prefix);
        const bool kept = i < n && (contested[j] ? key[j] > prefix || (key[j] == prefix && equal + below(same, lane) < need) : !among_first);
        equal += __popcll(same);
        hole[j] = __builtin_amdgcn_ballot_w64(i < keep && !kept);
        mover[j] = __builtin_amdgcn_ballot_w64(i >= keep && kept);
        n_holes += __popcll(hole[j]);
        n_movers += __popcll(mover[j]);
    }
    if (lane == 0) count[2][wave] = n_holes, count[3][wave] = n_movers;
    __syncthreads();
    int hole0 = 0, mover0 = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        hole0 += w < wave ? count[2][w] : 0;
        mover0 += w < wave ? count[3][w] : 0;
        all += count[2][w];
    }
    if (tid == 0) p.n_moves[b] = all;
    int at_hole[K];
#pragma unroll
    for (int j = 0; j < K; ++j) {
        const int i = i0 + 64 * j;
        at_hole[j] = hole0 + below(hole[j], lane);
        if (hole[j] >> lane & 1) holes[at_hole[j]] = i;
        if (mover[j] >> lane & 1) {
            const int at = mover0 + below(mover[j], lane);
            movers[at] = i;
            movers_lds[at] = i;
        }
        hole0 += __popcll(hole[j]);
        mover0 += __popcll(mover[j]);
    }
    if (!src) return;
    __syncthreads();
    write_src([&](int j, int i) { return i >= keep ? -1 : hole[j] >> lane & 1 ? movers_lds[at_hole[j]] : i; });
}

// ---- a workgroup per 4096 tokens -------------------------------------------------------------------
// A sequence's segments: the slots below `keep`, then those from it on, each in runs of 4096; so a segment has holes or movers, not
// both, and how many follows from its histograms.
constexpr int kSegWords = kEvictSegment / kThreads;  // words of 64 a wave
struct Segment {
    int n, keep, i0, i1, low, mine, segs;  // slots i0 .. i1 - 1; segments below `keep`; this one; all
};
static __device__ __forceinline__ Segment segment_of(const EvictArgs &p, int b, int len)
{
    Segment s;
    s.n = min(max(len, 0), p.max_len);
    s.keep = min(max(p.budget[b], 0), s.n);
    s.low = (s.keep + kEvictSegment - 1) / kEvictSegment;
    s.segs = s.low + (s.n - s.keep + kEvictSegment - 1) / kEvictSegment;
    s.mine = blockIdx.x % p.segments;
    s.i0 = s.mine < s.low ? s.mine * kEvictSegment : s.keep + (s.mine - s.low) * kEvictSegment;
    s.i1 = min(s.i0 + kEvictSegment, s.mine < s.low ? s.keep : s.n);
    return s;
}

// STEP 0: keys, and histograms of their first 11 bits, of the tokens with a stamp that counts and of the others.
// STEP 1, 2: choose the bits from all segments' histograms, and the histogram of the next ones.  STEP 3: lists of holes and movers.
// Workspace of a segment: 4 histograms and {tokens with a stamp that counts, kept ones by the bits of pass 0, of pass 1}.
template <int STEP>
__global__ __launch_bounds__(kThreads) void evict_step_kernel(const EvictArgs p)
{
    __shared__ int hist[2][kBins], room[3][kWaves], count[2][kWaves], chosen[3], total[2];
    const int b = blockIdx.x / p.segments, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    // (len_out may be len: step 3 writes it, and takes what step 0 read)
    int32_t *state = p.state + (int64_t)b * 8;  // len; bits chosen by step 1, 2; of how many of those that have them the last one is kept
    const Segment s = segment_of(p, b, STEP == 0 ? p.len[b] : state[0]);
    if (STEP == 0 && s.mine == 0 && tid == 0) state[0] = s.n;
    const bool trivial = s.keep == s.n || s.keep == 0;
    if (STEP == 3) {
        const int src_ld = p.table_ld << p.page_shift;
        if (p.src) {  // (the move kernel fills in the movers)
            int32_t *src = p.src + (int64_t)b * src_ld;
            for (int i = s.mine * kThreads + tid; i < src_ld; i += p.segments * kThreads) src[i] = i < s.keep ? i : -1;
        }
        if (s.mine == 0 && tid == 0) {
            p.len_out[b] = s.keep;
            if (trivial) p.n_moves[b] = 0;
        }
    }
    if (trivial || s.mine >= s.segs) return;
    int32_t *const base = p.hists + (int64_t)b * p.segments * kEvictSegInts, *const own = base + (int64_t)s.mine * kEvictSegInts;
    uint32_t *const keys = p.keys + (int64_t)b * p.max_len;
    uint64_t *const firsts = p.first + ((int64_t)b * p.segments + s.mine) * (kEvictSegment / 64);
    const int at0 = s.i0 + wave * kSegWords * 64 + lane;  // this thread's slots: at0 + 64 j

    if (STEP < 3)
        for (int i = tid; i < 2 * kBins; i += kThreads) hist[0][i] = 0;
    uint32_t key[kSegWords];
    uint64_t first[kSegWords];
    if constexpr (STEP == 0) {
        const int limit = p.keep_from ? p.keep_from[b] : 0;
        int n_first = 0;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kSegWords; ++j) {
            const int i = at0 + 64 * j;
            const int64_t at = token_at(p, b, min(i, s.i1 - 1));
            key[j] = order_bits(p.rank[at]);
            const bool is = i < s.i1 && p.keep_from && p.stamp[at] >= limit;
            first[j] = __builtin_amdgcn_ballot_w64(is);
            n_first += __popcll(first[j]);
            if (lane == 0) firsts[wave * kSegWords + j] = first[j];
            if (i < s.i1) {
                keys[i] = key[j];
                atomicAdd(&hist[is ? 1 : 0][key[j] >> kShift[0]], 1);
            }
        }
        if (lane == 0) count[0][wave] = n_first;
        __syncthreads();
        for (int i = tid; i < 2 * kBins; i += kThreads) own[i] = hist[0][i];
        if (tid == 0) {
            n_first = 0;
            for (int w = 0; w < kWaves; ++w) n_first += count[0][w];
            own[4 * kBins] = n_first;
        }
    } else {
        // sums over the segments: this thread's two bins of the last pass's histogram, and the tokens with a stamp that counts
        int n_first = 0;
        for (int g = lane; g < s.segs; g += 64) n_first += base[(int64_t)g * kEvictSegInts + 4 * kBins];
#pragma unroll
        for (int o = 1; o < 64; o *= 2) n_first += __shfl_xor(n_first, o, 64);
        const bool among_first = n_first >= s.keep;
        const int last = STEP == 1 ? (among_first ? 1 : 0) : STEP;  // which of the four
        const int bin = kBins - 1 - 2 * tid;
        int high = 0, low = 0;
#pragma unroll 16  // (requested together: other workgroups wrote them, far away)
        for (int g = 0; g < s.segs; ++g) {
            const int2 x = *(const int2 *)(base + (int64_t)g * kEvictSegInts + last * kBins + bin - 1);
            low += x.x;
            high += x.y;
        }
        uint32_t prefix = STEP == 1 ? 0 : (uint32_t)state[1], known = STEP == 1 ? 0 : (uint32_t)kMask[0] << kShift[0];
        if (STEP == 3) prefix |= (uint32_t)state[2], known |= (uint32_t)kMask[1] << kShift[1];
        const int need_in = STEP == 1 ? (among_first ? s.keep : s.keep - n_first) : state[STEP + 1];
        choose(high, low, need_in, room[0], chosen, tid);
        __syncthreads();
        const int pick = chosen[0], need = chosen[1];
        constexpr int PASS = STEP - 1;
        prefix |= (uint32_t)pick << kShift[PASS];
        known |= (uint32_t)kMask[PASS] << kShift[PASS];
#pragma unroll
        for (int j = 0; j < kSegWords; ++j) {
            const int i = at0 + 64 * j;
            first[j] = firsts[wave * kSegWords + j];
            key[j] = i < s.i1 ? keys[i] : 0;
        }
        auto contested = [&](int j) { return at0 + 64 * j < s.i1 && ((first[j] >> lane & 1) != 0) == among_first; };
        if constexpr (STEP < 3) {
            if (s.mine == 0 && tid == 0) {
                state[STEP] = (uint32_t)pick << kShift[PASS];
                state[STEP + 2] = need;
            }
#pragma unroll
            for (int j = 0; j < kSegWords; ++j)
                if (contested(j) && (key[j] & known) == prefix) atomicAdd(&hist[0][key[j] >> kShift[STEP] & kMask[STEP]], 1);
            __syncthreads();
            for (int i = tid; i < kBins; i += kThreads) own[(STEP + 1) * kBins + i] = hist[0][i];
            // this segment's contested tokens above the chosen bits
            const int *mine = own + last * kBins;
            const int2 x = *(const int2 *)(mine + bin - 1);
            int above = (bin > pick ? x.y : 0) + (bin - 1 > pick ? x.x : 0);
#pragma unroll
            for (int o = 1; o < 64; o *= 2) above += __shfl_xor(above, o, 64);
            if (lane == 0) count[1][wave] = above;
            __syncthreads();
            if (tid == 0) {
                above = 0;
                for (int w = 0; w < kWaves; ++w) above += count[1][w];
                own[4 * kBins + STEP] = above;
            }
        } else {
            // Before this segment, and in all: kept tokens among those that equal the last kept one; holes (below `keep`) or movers.
            // A wave takes a segment at a time; its last histogram's bins above the chosen one are kept as well.
            for (int g = wave; g < s.segs; g += kWaves) {
                const int32_t *seg = base + (int64_t)g * kEvictSegInts;
                int above = 0;
#pragma unroll
                for (int i = 0; i < 1024; i += 64) {
                    const int x = seg[3 * kBins + i + lane];
                    above += i + lane > pick ? x : 0;
                }
#pragma unroll
                for (int o = 1; o < 64; o *= 2) above += __shfl_xor(above, o, 64);
                if (lane == 0) {
                    hist[0][g] = seg[3 * kBins + pick];  // equal ones
                    hist[1][g] = (among_first ? 0 : seg[4 * kBins]) + seg[4 * kBins + 1] + seg[4 * kBins + 2] + above;
                }
            }
            __syncthreads();
            if (wave == 0) {  // (64 segments at a time)
                int equal = 0, holes = 0, movers = 0;  // before them
                for (int g0 = 0; g0 < s.segs; g0 += 64) {
                    const int g = g0 + lane, eq = g < s.segs ? hist[0][g] : 0, eq_to = equal + sum_to_me(eq);
                    const int kept = g < s.segs ? hist[1][g] + min(eq, max(0, need - (eq_to - eq))) : 0;
                    const int hole = g < s.low ? min(kEvictSegment, s.keep - g * kEvictSegment) - kept : 0, mover = g < s.low ? 0 : kept;
                    const int hole_to = holes + sum_to_me(hole), mover_to = movers + sum_to_me(mover);
                    if (g == s.mine) total[0] = eq_to - eq, total[1] = g < s.low ? hole_to - hole : mover_to - mover;
                    equal = __shfl(eq_to, 63, 64), holes = __shfl(hole_to, 63, 64), movers = __shfl(mover_to, 63, 64);
                }
                if (s.mine == 0 && lane == 0) p.n_moves[b] = holes;
            }
            int equal = 0;
#pragma unroll
            for (int j = 0; j < kSegWords; ++j) equal += __popcll(__builtin_amdgcn_ballot_w64(contested(j) && key[j] == prefix));
            if (lane == 0) count[0][wave] = equal;
            __syncthreads();
            equal = total[0];
#pragma unroll
            for (int w = 0; w < kWaves; ++w) equal += w < wave ? count[0][w] : 0;
            uint64_t list[kSegWords];
            int listed = 0;
#pragma unroll
            for (int j = 0; j < kSegWords; ++j) {
                const int i = at0 + 64 * j;
                const uint64_t same = __builtin_amdgcn_ballot_w64(contested(j) && key[j] == prefix);
                const bool kept = contested(j) ? key[j] > prefix || (key[j] == prefix && equal + below(same, lane) < need) : !among_first;
                equal += __popcll(same);
                list[j] = __builtin_amdgcn_ballot_w64(i < s.i1 && kept == (s.mine >= s.low));
                listed += __popcll(list[j]);
            }
            if (lane == 0) count[1][wave] = listed;
            __syncthreads();
            int at = total[1];
#pragma unroll
            for (int w = 0; w < kWaves; ++w) at += w < wave ? count[1][w] : 0;
            int32_t *to = (s.mine < s.low ? p.holes : p.movers) + (int64_t)b * (p.max_len / 2 + 1);
#pragma unroll
            for (int j = 0; j < kSegWords; ++j) {
                if (list[j] >> lane & 1) to[at + below(list[j], lane)] = at0 + 64 * j;
                at += __popcll(list[j]);
            }
        }
    }
}

__global__ __launch_bounds__(256) void evict_move_kernel(const EvictArgs p, int per_seq)
{
    const int b = blockIdx.x / per_seq, part = blockIdx.x % per_seq, n = p.n_moves[b];
    const int32_t *holes = p.holes + (int64_t)b * (p.max_len / 2 + 1), *movers = p.movers + (int64_t)b * (p.max_len / 2 + 1);
    const int32_t *table = p.table + (int64_t)b * p.table_ld;
    const int C = p.row_bytes / 16, in_page = (1 << p.page_shift) - 1;
    const int pieces = p.Hkv * C, together = max(1, 256 / pieces);  // 16 bytes of a head of a token each; tokens that a workgroup moves at once
    for (int m0 = part * together; m0 < n; m0 += per_seq * together) {
        for (int x = threadIdx.x; x < min(together, n - m0) * pieces; x += 256) {
            const int m = m0 + x / pieces, c = x % C, h = x / C % p.Hkv, to = holes[m], from = movers[m];
            const int tp = table[to >> p.page_shift], fp = min(max(table[from >> p.page_shift], 0), p.n_pages - 1);
            if (h == 0 && c == 0 && p.segments > 0 && p.src) p.src[(int64_t)b * (p.table_ld << p.page_shift) + to] = from;
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
}

}  // namespace

hipError_t launch_paged_evict(const EvictArgs &a, hipStream_t s)
{
    if (a.segments > 0) {
        const dim3 grid((unsigned)(a.segments * a.n_seqs));
        hipLaunchKernelGGL(evict_step_kernel<0>, grid, dim3(kThreads), 0, s, a);
        hipLaunchKernelGGL(evict_step_kernel<1>, grid, dim3(kThreads), 0, s, a);
        hipLaunchKernelGGL(evict_step_kernel<2>, grid, dim3(kThreads), 0, s, a);
        hipLaunchKernelGGL(evict_step_kernel<3>, grid, dim3(kThreads), 0, s, a);
    } else {
        void (*kernel)(EvictArgs) = a.max_len <= kThreads ? evict_select_kernel<1> : a.max_len <= 4 * kThreads ? evict_select_kernel<4> : evict_select_kernel<16>;
        hipLaunchKernelGGL(kernel, dim3((unsigned)a.n_seqs), dim3(kThreads), 0, s, a);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t most = ((int64_t)(a.max_len / 2 + 1) * a.Hkv * (a.row_bytes / 16) + 255) / 256;  // workgroups that a sequence can use
    // 4096 workgroups in all (us of five cuts with 1024, 2048, 4096, 8192, 16384: 64 sequences to half 43, 34, 32, 30, 32, a long one to half 44, 44, 44,
    // 45, 47, 300 short ones to three quarters 22, 21, 22, 23, 26, eight to half 25, 26, 25, 26, 26, one token out of 32 11, 12, 12, 11, 11)
    const int per = (int)std::max<int64_t>(1, std::min<int64_t>(most, 4096 / a.n_seqs));
    hipLaunchKernelGGL(evict_move_kernel, dim3((unsigned)(per * a.n_seqs)), dim3(256), 0, s, a, per);
    return hipGetLastError();
}

}  // namespace climber
