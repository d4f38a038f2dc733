// The paged history cache: what its kernels are given, and the geometry that they share (internal).
#pragma once
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

namespace climber {

// One call on a paged cache.  Rows of the call: new behaviours (history) or candidates (SUMI) of n_seqs sequences, packed by `off`.
// The G = H / Hkv query heads that share a cache head are rows of one problem: "packed row" r of (sequence, cache head) is row r / G,
// query head r % G of the group, so that a tile of packed rows reads keys and values once for all of them.
struct PagedArgs {
    uint8_t *k_pages, *v_pages;  // [n_pages][Hkv][page][d]
    float *mass;                 // [n_pages][page] or nullptr
    int32_t *stamp;              // [n_pages][page] or nullptr
    const int32_t *table, *len;  // [n_seqs][table_ld], [n_seqs]
    const uint8_t *q, *k, *v;    // the call's rows
    int64_t ld_q, ld_kv, ld_o;   // bytes
    const int32_t *off, *scen, *beh, *stamp_new;
    const float *tau;
    uint8_t *o;
    int n_seqs, n_pages, page_shift, table_ld, max_len;
    int H, Hkv, G, d, row_bytes;  // row_bytes: of one key of one head
    uint32_t G_inv;               // ceil(2^32 / G): r / G is umulhi(r, G_inv) or one less (r, G < 2^26; G > 1)
    int n_scen, n_beh, m_total, m_max;
    int causal, sumi;
    float scale_log2e;
    // work split: tiles of packed rows, parts of the keys
    int n_tiles, n_split, bh_major, by_work;
    int pair;  // by_work: sequences from this one of their order on come in ascending order; 0: all in descending
    float *part_o, *part_ml;  // [n_split][m_total H][d], [n_split][m_total H][2] (n_split > 1)
    float *logits;            // few rows: [n_seqs Hkv][m_max G][logits_ld] logits in log2 units for paged_mass_few, or nullptr
    int logits_ld;
    float2 *lse;              // [m_total H] {scale, log of the sum of the exponentials} of a row's softmax, log2 units, or nullptr: not wanted
};

struct PagedSeq {
    int n, T;      // cached tokens, rows of the call
    int64_t row0;  // first row
};

// Lengths and offsets live in device memory: whatever they hold, nothing is read or written outside the arrays.  New tokens that a sequence of
// max_len tokens has no room for are not stored, and no row sees them.
static __device__ __forceinline__ PagedSeq paged_seq(const PagedArgs &p, int b)
{
    PagedSeq s;
    const int r0 = min(max(p.off[b], 0), p.m_total);
    s.T = min(min(max(p.off[b + 1] - r0, 0), p.m_total - r0), p.m_max);
    s.n = min(max(p.len[b], 0), p.max_len);
    s.row0 = r0;
    return s;
}
// keys of a sequence: the cached tokens, then the new ones that have a slot
static __device__ __forceinline__ int paged_keys(const PagedArgs &p, const PagedSeq &s) { return p.sumi ? s.n : min(s.n + s.T, p.max_len); }

static __device__ __forceinline__ int paged_page(const PagedArgs &p, int b, int slot)
{
    return min(max(p.table[(int64_t)b * p.table_ld + (slot >> p.page_shift)], 0), p.n_pages - 1);
}

// byte offset of a slot's row of head h in the key or value pages
static __device__ __forceinline__ int64_t paged_row(const PagedArgs &p, int page, int h, int slot)
{
    return ((((int64_t)page * p.Hkv + h) << p.page_shift) + (slot & ((1 << p.page_shift) - 1))) * p.row_bytes;
}

// Workgroup -> (sequence, cache head), tile, part of the keys.  Tiles of one head read the same keys: they follow each other on one XCD
// (workgroups are dealt to the eight in turn), where there are heads enough to have each XCD work; the last tiles, which see the
// most keys under the causal mask, first.
// With by_work the sequences of each 64 take their turns in the order of their work (each wave ranks them, one in a lane): lengths differ,
// and a long one that is begun last would be waited for.  Every second eight of them go to the XCDs the other way round, or the first XCD
// would have the most of each eight (16 users' candidates on a cache in 8 bits 159 / 144 us).
struct PagedWork {
    int b, hk, tile, split;
};
static __device__ __forceinline__ bool paged_work(const PagedArgs &p, PagedWork &w, PagedSeq &s)
{
    const int per = p.n_tiles * p.n_split, n_bh = p.n_seqs * p.Hkv;
    int bh, in;
    if (p.bh_major) {
        const int j = blockIdx.x >> 3;
        const int eight = j / per, x = blockIdx.x & 7;
        bh = eight * 8 + (p.by_work && (eight & 1) ? 7 - x : x);
        in = j % per;
    } else {
        bh = blockIdx.x / per;
        in = blockIdx.x % per;
    }
    if (bh >= n_bh) return false;
    w.b = bh / p.Hkv;
    w.hk = bh % p.Hkv;
    w.tile = p.n_tiles - 1 - in / p.n_split;
    w.split = in % p.n_split;
    if (!p.by_work) {
        s = paged_seq(p, w.b);
        return true;
    }
    const int lane = threadIdx.x & 63, b0 = w.b & ~63, n = min(p.n_seqs - b0, 64);
    const PagedSeq mine = paged_seq(p, b0 + min(lane, n - 1));
    // (work in 26 bits, and the lane: no two alike)
    const uint32_t work = lane < n ? (__float_as_uint((float)mine.T * (float)(mine.n + mine.T)) & ~63u) | (uint32_t)(63 - lane) : 0;
    int at = w.b - b0;
    if (p.pair && at >= p.pair) at = n - 1 - (at - p.pair);
    if (__builtin_amdgcn_ballot_w64(lane < n && (work >> 6) != (__builtin_amdgcn_readfirstlane(work) >> 6)) != 0) {
        int rank = 0;
        for (int j0 = 0; j0 < n; j0 += 16)
#pragma unroll
            for (int j = 0; j < 16; ++j) rank += (uint32_t)__builtin_amdgcn_readlane(work, j0 + j) > work;
        at = __ffsll((unsigned long long)__builtin_amdgcn_ballot_w64(lane < n && rank == at)) - 1;
    }
    at = __builtin_amdgcn_readfirstlane(at);
    w.b = b0 + at;
    s.n = __builtin_amdgcn_readlane(mine.n, at);
    s.T = __builtin_amdgcn_readlane(mine.T, at);
    s.row0 = __builtin_amdgcn_readlane((int)mine.row0, at);
    return true;
}
static inline unsigned paged_grid(PagedArgs &p)
{
    const int64_t bh = (int64_t)p.n_seqs * p.Hkv;
    p.bh_major = bh % 8 == 0 || bh >= 64;
    // By work: us with / without for a token of each of 64 users 107 / 117, ragged scoring of 16 users 154 / 175, sessions of eight 171 / 177 (weights
    // and all).  Where lengths are spread evenly over a factor of eight it also loses: scoring of 16 users 127 / 119, a token of each of 300
    // 81 / 73.  Fewer workgroups all run at once (256 of scoring 51 / 51, 128 38 / 41), more have small shares, and the ranks cost more than they give (4096 of
    // scoring 268 / 255, 8000 of single tokens 173 / 144).
    const int64_t all = bh * p.n_tiles * p.n_split;
    p.by_work = p.n_seqs > 1 && all >= 512 && all < 4096;
    return (unsigned)((p.bh_major ? (bh + 7) / 8 * 8 : bh) * p.n_tiles * p.n_split);
}

// the keys [lo, hi) of part `split` of the first k_end keys, in whole tiles of `unit`
static __device__ __forceinline__ void paged_part(const PagedArgs &p, int split, int k_end, int unit, int &lo, int &hi)
{
    const int tiles = (k_end + unit - 1) / unit, per = (tiles + p.n_split - 1) / p.n_split;
    lo = min(split * per * unit, k_end);
    hi = min(lo + per * unit, k_end);
}

// log2(e) qk_scale / temperature of a row
static __device__ __forceinline__ float paged_row_scale(const PagedArgs &p, int64_t row)
{
    const int sc = min(max(p.scen[row], 0), p.n_scen - 1), bh = min(max(p.beh[row], 0), p.n_beh - 1);
    return p.scale_log2e / p.tau[sc * p.n_beh + bh];
}

// Packed rows of a workgroup.  32: the kernels for few rows, whose waves share out keys.  bf16: where a sequence and cache head has no
// more of them.  fp32, which has no use for more rows per operand than 32: also where tiles of 128 rows are fewer than 96 (us few /
// tiles at d_head 64: 48 of them 30 / 46, 128 of them 76 / 70, 256 of them 156 / 127), and above d_head 64, where tiles would leave one wave
// per SIMD (788 / 1020 for chunks of 1000 of 8 users on 1000).  256 at d_head 64 in bf16: 108 / 123 with 128 for 512 candidates of
// each of 64 users on 1024.
static inline int paged_tile_rows(bool bf16, int d, int64_t rows, int64_t groups)
{
    if (rows <= 32 || (!bf16 && (d > 64 || (rows + 127) / 128 * groups < 96))) return 32;
    return bf16 && d == 64 && rows > 128 ? 256 : 128;
}

hipError_t launch_attn_paged_bf16(const PagedArgs &a, hipStream_t s);
hipError_t launch_attn_paged_f32(const PagedArgs &a, hipStream_t s);
hipError_t launch_paged_combine(const PagedArgs &a, bool bf16, hipStream_t s);
// Attention weights per cached token, in two steps: sums over the rows of one cache head into part[n_seqs][parts][max_len], the parts
// of a sequence being its cache heads (bf16: times paged_mass_parts), and those added up into the masses.
hipError_t launch_paged_mass_f32(const PagedArgs &a, float *part, hipStream_t s);
hipError_t launch_paged_mass_bf16(const PagedArgs &a, float *part, int row_parts, hipStream_t s);
// ... in one step for at most kMassFewRows packed rows of a sequence and cache head, whose attention has left its logits: keys are not
// read again.  us this way / with logits made again, chunks of 64 users on 500 to 4000, heads of 128: 4 rows 139 / 208, 8 rows 147 / 210; one long
// cache, 4 rows 72 / 98; fp32, 16 users, 4 rows 36 / 60.  With room for 16 rows 4 take 145, 8 take 154 and 16 171 / 212; for 32 rows 163, 173, 189 and
// 32 220 / 215.
constexpr int kMassFewRows = 8;
hipError_t launch_paged_mass_few(const PagedArgs &a, hipStream_t s);
hipError_t launch_paged_mass_add(const PagedArgs &a, const float *part, int n_parts, hipStream_t s);
constexpr int kMassKeys = 256, kMassGroups = 2048;  // bf16: keys of a workgroup; workgroups of a launch that parts of the rows bring it to
// bf16: parts of a cache head's rows, of 256 rows or more (us of two cases of ragged lengths with 512, 1024, 2048, 4096 workgroups:
// 184, 183, 181, 191 and 210, 196, 194, 203)
static inline int paged_mass_parts(int64_t n_seqs, int64_t Hkv, int64_t max_len, int64_t rows)
{
    const int64_t groups = n_seqs * Hkv * ((max_len + kMassKeys - 1) / kMassKeys), most = (rows + 255) / 256, want = groups > 0 ? kMassGroups / groups : 1;
    return (int)(want < 1 || most < 1 ? 1 : want < most ? want : most);
}

// Tokens of a workgroup where a sequence may be too long for one, and the integers that it leaves for the others.
constexpr int kEvictOne = 16384, kEvictSegment = 4096, kEvictSegInts = 4 * 2048 + 8, kEvictMostSegments = 1025;
static inline int64_t evict_segments(int64_t max_len) { return max_len <= kEvictOne ? 0 : (max_len + kEvictSegment - 1) / kEvictSegment + 1; }

struct EvictArgs {
    uint8_t *k_pages, *v_pages;
    float *mass;
    const float *rank;
    int32_t *stamp;
    const int32_t *table, *len, *budget, *keep_from;
    int32_t *len_out, *src;
    int n_seqs, n_pages, page_shift, table_ld, max_len, Hkv, row_bytes, segments;
    // workspace
    int32_t *holes, *movers;   // [n_seqs][max_len / 2 + 1]
    int32_t *n_moves;          // [n_seqs]
    uint32_t *keys;            // [n_seqs][max_len]                  (segments > 0, as what follows)
    uint64_t *first;           // [n_seqs][segments][64]: bit set: ranks before all others
    int32_t *hists, *state;    // [n_seqs][segments][kEvictSegInts], [n_seqs][8]
};
hipError_t launch_paged_evict(const EvictArgs &a, hipStream_t s);

}  // namespace climber
