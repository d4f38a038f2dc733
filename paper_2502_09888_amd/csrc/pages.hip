// The pages of paged caches (gfx950): tables of pages forked, extended, compacted, and the pages' data copied.
//
// refs[p] counts the table entries that hold page p (and whatever else the caller has it held by); free pages have 0.  All of it is whole
// numbers: sums by atomics do not depend on their order, and where an order decides (which free page, which of the sequences that
// write a shared page keeps it) it is that of the pages, the sequences and their places.
#include "pages.h"

#include "../../include/climber.h"

#include <algorithm>

namespace climber {
namespace {

// (values that atomics of this launch have changed: not from a line that was read before)
static __device__ __forceinline__ int fresh(const int32_t *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
static __device__ __forceinline__ int below(uint64_t bits) { return __builtin_amdgcn_mbcnt_hi((uint32_t)(bits >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)bits, 0)); }
static __device__ __forceinline__ bool in_pool(const PoolArgs &a, int page) { return page >= 0 && page < a.n_pages; }
static __device__ __forceinline__ int held_of(const PoolArgs &a, int b) { return min(max(a.held[b], 0), a.table_ld); }

// sum over the lanes before this one, and over all
static __device__ __forceinline__ int wave_before(int x, int &all)
{
    const int lane = threadIdx.x & 63;
    int y = x;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int z = __shfl_up(y, d, 64);
        if (lane >= d) y += z;
    }
    all = __builtin_amdgcn_readlane(y, 63);
    return y - x;
}
// ... over the threads of a workgroup of 1024 (scratch: 16 integers of LDS)
static __device__ __forceinline__ int group_before(int x, int &all, int *scratch)
{
    int mine;
    const int in_wave = wave_before(x, mine);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = mine;
    __syncthreads();
    int before = 0, sum = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int y = scratch[i];
        if (i < (int)(threadIdx.x >> 6)) before += y;
        sum += y;
    }
    all = sum;
    return before + in_wave;
}

// A wave looks at the pages of a unit: bits of the free ones, or of those in use, and how many of either there are.
static __device__ __forceinline__ void look(const int32_t *refs, int n_pages, int unit, bool want_free, uint64_t *bits, int32_t *n_free, int32_t *n_used)
{
    const int lane = threadIdx.x & 63;
    int r[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int64_t p = (int64_t)unit * kUnitPages + i * 64 + lane;
        r[i] = p < n_pages ? refs[p] : -1;
    }
    uint64_t mine = 0;
    int free_all = 0, used_all = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const uint64_t f = __builtin_amdgcn_ballot_w64(r[i] == 0), u = __builtin_amdgcn_ballot_w64(r[i] > 0);
        free_all += __popcll(f), used_all += __popcll(u);
        if (lane == i) mine = want_free ? f : u;
    }
    if (lane < 16) bits[(int64_t)unit * 16 + lane] = mine;
    if (lane == 0) {
        if (n_free) n_free[unit] = free_all;
        n_used[unit] = used_all;
    }
}

// ---- fork ----------------------------------------------------------------------------------------
constexpr int kForkFew = 2048;  // entries of a table that one workgroup takes (us of a whole run, in two launches / this way: 6 entries 18 / 15, 8192 entries 150 / 166)

// Waves for a row of a table: more than one where rows are long and few (us of a run that forks and moves two rows of 6173 entries and of the calls
// around it, with one / with these 173 / 46).
static int row_waves(const PoolArgs &a) { return (int)std::max<int64_t>(1, std::min<int64_t>((a.table_ld + 63) / 64, 1024 / a.n_seqs)); }

// What rows become is read before any row is written: a row's waves note it and count, another launch writes it.  Bound by its launches: 3 to 5 us
// each for 160 to 256 rows.
static __device__ __forceinline__ void fork_read(const ForkArgs &a, int b, int piece, int pieces)
{
    const int lane = threadIdx.x & 63, first = piece * 64 + lane;
    const int par = a.parent[b];
    if (par >= a.n_seqs) {  // (no sequence: the row stays)
        if (first == 0) atomicOr(a.status, CLIMBER_BAD_SEQ), a.new_held[b] = -1;
        return;
    }
    const int had = held_of(a, b);
    int n = 0, h = 0;
    if (par >= 0) {
        const int all = max(a.len[par], 0);
        n = a.keep ? min(all, max(a.keep[b], 0)) : all;
        h = min((int)(((int64_t)n + (1 << a.page_shift) - 1) >> a.page_shift), held_of(a, par));
        if (par == b && n == all && (!a.keep || h == had)) {
            if (first == 0) a.new_held[b] = -1;
            return;
        }
    }
    bool bad = false;
    for (int i = first; i < max(had, h); i += 64 * pieces) {
        const int was = i < had ? a.table[(int64_t)b * a.table_ld + i] : -1, is = i < h ? a.table[(int64_t)par * a.table_ld + i] : -1;
        a.rows[(int64_t)b * a.table_ld + i] = is;
        bad |= (i < h && !in_pool(a, is)) || (i < had && !in_pool(a, was));
        if (was == is) continue;
        if (in_pool(a, was)) atomicSub(a.refs + was, 1);
        if (in_pool(a, is)) atomicAdd(a.refs + is, 1);
    }
    if (bad) atomicOr(a.status, CLIMBER_BAD_PAGE);
    if (first == 0) a.new_len[b] = n, a.new_held[b] = h, a.entries[b] = max(had, h);
}
static __device__ __forceinline__ void fork_write(const ForkArgs &a, int b, int piece, int pieces)
{
    const int first = piece * 64 + (threadIdx.x & 63);
    const int h = a.new_held[b];
    if (h < 0) return;
    const int n = a.entries[b];  // (a.held changes here)
    for (int i = first; i < n; i += 64 * pieces) a.table[(int64_t)b * a.table_ld + i] = a.rows[(int64_t)b * a.table_ld + i];
    if (first == 0) a.len[b] = a.new_len[b], a.held[b] = h;
}
__global__ __launch_bounds__(256) void fork_read_kernel(const ForkArgs a)
{
    const int b = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (b < a.n_seqs) fork_read(a, b, blockIdx.y, gridDim.y);
}
__global__ __launch_bounds__(256) void fork_write_kernel(const ForkArgs a)
{
    const int b = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (b < a.n_seqs) fork_write(a, b, blockIdx.y, gridDim.y);
}
// ... small tables by one workgroup, a thread for each entry in turn; bound by its trips to memory, one behind the other
__global__ __launch_bounds__(1024) void fork_few_kernel(const ForkArgs a)
{
    const int all = a.n_seqs * a.table_ld;
    int bits = 0;
    for (int e0 = 0; e0 < all; e0 += 1024) {
        const int e = e0 + threadIdx.x;
        if (e >= all) continue;
        const int b = e / a.table_ld, i = e - b * a.table_ld, par = a.parent[b], had = held_of(a, b), was = a.table[e];
        int h = -1, n = 0;
        if (par < a.n_seqs) {
            h = 0;
            if (par >= 0) {
                const int there = max(a.len[par], 0);
                n = a.keep ? min(there, max(a.keep[b], 0)) : there;
                h = min((int)(((int64_t)n + (1 << a.page_shift) - 1) >> a.page_shift), held_of(a, par));
                if (par == b && n == there && (!a.keep || h == had)) h = -1;
            }
        } else {
            bits |= CLIMBER_BAD_SEQ;
        }
        if (i == 0) a.new_held[b] = h, a.new_len[b] = n;
        if (h < 0 || i >= max(had, h)) continue;
        const int is = i < h ? a.table[(int64_t)par * a.table_ld + i] : -1;
        a.rows[e] = is;
        if ((i < h && !in_pool(a, is)) || (i < had && !in_pool(a, was))) bits |= CLIMBER_BAD_PAGE;
        if (i < had && was == is) continue;
        if (i < had && in_pool(a, was)) atomicSub(a.refs + was, 1);
        if (in_pool(a, is)) atomicAdd(a.refs + is, 1);
    }
    if (bits) atomicOr(a.status, bits);
    __syncthreads();
    for (int e = threadIdx.x; e < all; e += 1024) {
        const int b = e / a.table_ld, i = e - b * a.table_ld, h = a.new_held[b];
        if (h >= 0 && i < max(held_of(a, b), h)) a.table[e] = a.rows[e];
    }
    __syncthreads();  // (what rows held before is read above)
    for (int b = threadIdx.x; b < a.n_seqs; b += 1024)
        if (a.new_held[b] >= 0) a.len[b] = a.new_len[b], a.held[b] = a.new_held[b];
}

// ---- extend --------------------------------------------------------------------------------------
constexpr int kFewSeqs = 1024, kFewUnits = 64, kFewWriters = 512, kListPages = 4096, kFewNew = 4;  // what one workgroup takes; free pages that it keeps in LDS; new ones that a thread writes
constexpr int kCompactFew = 2048;  // entries of a table that one workgroup takes (us by it / in three launches: 8192 entries 23.5 / 17.5, 50 entries 7 / 14)
constexpr int kNobody = 1 << 30;  // in last[]: a shared page that none of its writers keeps (n_seqs is less)

// Sequence b's part of the call: pages [first, shared_to) that it holds and writes, [shared_to, need) that it has to get.
struct Need {
    int first, shared_to, need, part;  // part: tokens in the first page that stay
    bool any, too_long;
};
static __device__ __forceinline__ Need need_of(const ExtendArgs &a, int b)
{
    Need x{};
    const int rows = a.rows[b], had = held_of(a, b);
    const int64_t n = max(a.len[b], 0), to = (n + max(rows, 0) + (1 << a.page_shift) - 1) >> a.page_shift;
    x.any = rows > 0;
    x.too_long = x.any && to > a.table_ld;
    x.need = x.any && !x.too_long ? (int)to : had;
    x.first = (int)min(n >> a.page_shift, (int64_t)a.table_ld);
    x.shared_to = min(had, x.need);
    x.part = (int)(n & ((1 << a.page_shift) - 1));
    if (!x.any) x.first = x.shared_to = x.need;
    return x;
}
// the shared pages that a sequence writes and does not keep
static __device__ __forceinline__ bool moves(const ExtendArgs &a, int b, int page)
{
    if (!in_pool(a, page)) return false;
    const int r = a.refs[page];
    return r > 1 && !(fresh(a.writers + page) == r && fresh(a.last + page) == b);
}

static __device__ void clear_writers(const ExtendArgs &a, int t, int n)
{
    for (int b = t; b < a.n_seqs; b += n) {
        const Need x = need_of(a, b);
        for (int i = x.first; i < x.shared_to; ++i) {
            const int page = a.table[(int64_t)b * a.table_ld + i];
            if (in_pool(a, page)) a.writers[page] = 0, a.last[page] = -1;
        }
    }
}
static __device__ void count_writers(const ExtendArgs &a, int t, int n)
{
    for (int b = t; b < a.n_seqs; b += n) {
        const Need x = need_of(a, b);
        for (int i = x.first; i < x.shared_to; ++i) {
            const int page = a.table[(int64_t)b * a.table_ld + i];
            if (!in_pool(a, page)) atomicOr(a.status, CLIMBER_BAD_PAGE);
            else if (a.refs[page] > 1) atomicAdd(a.writers + page, 1), atomicMax(a.last + page, b);
        }
    }
}
// A workgroup of 1024: who gets how many pages, whether there are enough, and which they are.
static __device__ void share_out(const ExtendArgs &a, int *scratch)
{
    const int t = threadIdx.x, lane = t & 63;
    int total = 0, n_copies = 0, bad = 0;
    for (int b0 = 0; b0 < a.n_seqs; b0 += 1024) {
        const int b = b0 + t;
        int c = 0, copy = 0;
        if (b < a.n_seqs) {
            const Need x = need_of(a, b);
            if (x.too_long) bad |= 1;
            for (int i = x.first; i < x.shared_to; ++i) {
                const int page = a.table[(int64_t)b * a.table_ld + i];
                if (!in_pool(a, page)) bad |= 2;
                if (!moves(a, b, page)) continue;
                ++c;
                copy |= i == x.first && x.part > 0;
            }
            c += max(0, x.need - max(x.shared_to, held_of(a, b)));
        }
        int all;
        // (pages of a call are fewer than 2^31: a sequence gets at most table_ld, and n_seqs table_ld is)
        const int at = group_before(c, all, scratch);
        if (b < a.n_seqs) a.first_new[b] = total + at;
        total += all;
        const int at_copy = group_before(copy, all, scratch);
        if (b < a.n_seqs) a.first_copy[b] = copy ? n_copies + at_copy : -1;
        n_copies += all;
    }
    const int units = (int)pool_units(a.n_pages);
    int n_free = 0, n_used = 0;
    for (int u0 = 0; u0 < units; u0 += 1024) {
        const int u = u0 + t;
        int all;
        const int f = u < units ? fresh(a.unit_free + u) : 0;
        const int at = group_before(f, all, scratch);
        if (u < units) a.unit_free[u] = n_free + at;  // from here on: free pages before the unit
        n_free += all;
        group_before(u < units ? fresh(a.unit_used + u) : 0, all, scratch);
        n_used += all;
    }
    int problems;
    group_before(bad & 1, problems, scratch);
    int bad_pages;
    group_before(bad >> 1, bad_pages, scratch);
    const bool full = problems > 0 || total > n_free, go = !full && bad_pages == 0;
    if (t == 0) {
        if (full) atomicOr(a.status, CLIMBER_POOL_FULL);
        a.go[0] = go;
        a.counts[0] = go ? n_copies : 0;
        a.counts[1] = n_used + (go ? total : 0);  // (a page that is given up stays with another sequence)
    }
    __syncthreads();
    if (!go) return;
    // refs change in the next launch: whether a page stays with the last of its writers is noted before
    for (int b = t; b < a.n_seqs; b += 1024) {
        const Need x = need_of(a, b);
        for (int i = x.first; i < x.shared_to; ++i) {
            const int page = a.table[(int64_t)b * a.table_ld + i];
            if (in_pool(a, page) && a.refs[page] > 1 && fresh(a.writers + page) != a.refs[page]) atomicOr(a.last + page, kNobody);
        }
    }
    for (int u = t >> 6; u < units; u += 16) {
        int at = fresh(a.unit_free + u);
        if (at >= total) break;
        const uint64_t mine = lane < 16 ? __hip_atomic_load(a.bits + (int64_t)u * 16 + lane, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0;
#pragma unroll 1
        for (int i = 0; i < 16; ++i) {
            const uint64_t w = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)mine, i) |
                               (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(mine >> 32), i) << 32;
            const int to = at + below(w);
            if (((w >> lane) & 1) && to < total) a.free_list[to] = u * kUnitPages + i * 64 + lane;
            at += __popcll(w);
        }
    }
}

__global__ __launch_bounds__(256) void extend_look_kernel(const ExtendArgs a, int unit_groups)
{
    if ((int)blockIdx.x < unit_groups) {
        const int unit = blockIdx.x * 4 + (threadIdx.x >> 6);
        if (unit < (int)pool_units(a.n_pages)) look(a.refs, a.n_pages, unit, true, a.bits, a.unit_free, a.unit_used);
        return;
    }
    clear_writers(a, (blockIdx.x - unit_groups) * 256 + threadIdx.x, (gridDim.x - unit_groups) * 256);
}
__global__ __launch_bounds__(256) void extend_writers_kernel(const ExtendArgs a) { count_writers(a, blockIdx.x * 256 + threadIdx.x, gridDim.x * 256); }
__global__ __launch_bounds__(1024) void extend_share_kernel(const ExtendArgs a)
{
    __shared__ int scratch[16];
    share_out(a, scratch);
}
// A wave for each sequence: shared pages first, then the new ones, each in order of their places.
__global__ __launch_bounds__(256) void extend_write_kernel(const ExtendArgs a)
{
    const int lane = threadIdx.x & 63, b = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (b >= a.n_seqs || !a.go[0]) return;
    const Need x = need_of(a, b);
    if (!x.any) return;
    const int had = held_of(a, b);
    int32_t *const row = a.table + (int64_t)b * a.table_ld;
    int at = a.first_new[b];
    for (int i0 = x.first; i0 < x.shared_to; i0 += 64) {
        const int i = i0 + lane, page = i < x.shared_to ? row[i] : -1, last = page >= 0 ? a.last[page] : -1;
        const bool m = last >= 0 && last != b;
        const uint64_t bits = __builtin_amdgcn_ballot_w64(m);
        if (m) {
            const int to = a.free_list[at + below(bits)];
            row[i] = to;
            a.refs[to] = 1;
            atomicSub(a.refs + page, 1);
            if (i == x.first && x.part > 0) {
                int32_t *const c = a.copies + 3 * (int64_t)a.first_copy[b];
                c[0] = page, c[1] = to, c[2] = x.part;
            }
        }
        at += __popcll(bits);
    }
    for (int i = had + lane; i < x.need; i += 64) {
        const int to = a.free_list[at + i - had];
        row[i] = to;
        a.refs[to] = 1;
    }
    if (lane == 0 && x.need > had) a.held[b] = x.need;
}

// All of it by one workgroup, a thread for each sequence; bound by its trips to memory, one behind the other: what a sequence needs, its
// pages, what their refs are (the pool's are looked through meanwhile).  Who else writes a shared page is found in LDS where that is few
// (one history forked four ways for each of 32 users, 128 writers: the call 10.5 us with counts in memory, 8.4 this way), and so are the pages handed out.
// us of a run with fork and copies, in the launches above / this way: one branch 25 / 15, four branches of 32 users 29 / 20, half of 256 users gone 153 / 150.
__global__ __launch_bounds__(1024) void extend_few_kernel(const ExtendArgs a)
{
    __shared__ int sums[3][16], list[kListPages], unit_at[kFewUnits + 1], n_listed, problems, some_long;
    // a table of shared pages that are written, at most half full: page, its writers, the last of them
    __shared__ int key[2 * kFewWriters], n_writers[2 * kFewWriters], last_writer[2 * kFewWriters];
    __shared__ uint64_t words[kFewUnits * 16];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6, units = (int)pool_units(a.n_pages), b = t;
    const bool mine = b < a.n_seqs;
    Need x{};
    int had = 0;
    if (mine) x = need_of(a, b), had = held_of(a, b);
    if (t == 0) n_listed = 0, problems = 0, some_long = 0;
    if (t < 2 * kFewWriters) key[t] = -1, n_writers[t] = 0, last_writer[t] = -1;
    int32_t *const row = a.table + (int64_t)b * a.table_ld;
    auto place = [](int page) { return (int)((uint32_t)page * 2654435769u >> 16) % (2 * kFewWriters); };
    // bits and counts of the units
    int n_used = 0;
    for (int u = wave; u < units; u += 16) {
        int r[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int64_t p = (int64_t)u * kUnitPages + i * 64 + lane;
            r[i] = p < a.n_pages ? a.refs[p] : -1;
        }
        int n_free = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const uint64_t f = __builtin_amdgcn_ballot_w64(r[i] == 0);
            n_free += __popcll(f);
            n_used += __popcll(__builtin_amdgcn_ballot_w64(r[i] > 0));
            if (lane == 0) words[u * 16 + i] = f;
        }
        if (lane == 0) unit_at[u] = n_free;
    }
    __syncthreads();
    // shared pages that are written
    bool shared = false;
    int bad = x.too_long;
    for (int i = x.first; i < x.shared_to; ++i) {
        const int page = row[i];
        if (!in_pool(a, page)) {
            bad |= 2;
        } else {
            if (a.refs[page] > 1) {
                if (atomicAdd(&n_listed, 1) < kFewWriters) {
                    int at = place(page);
                    for (int k; (k = atomicCAS(key + at, -1, page)) != -1 && k != page;) at = (at + 1) % (2 * kFewWriters);
                    atomicAdd(n_writers + at, 1);
                    atomicMax(last_writer + at, b);
                }
                shared = true;
            }
            a.writers[page] = 0, a.last[page] = -1;  // (for more of them than the list has room for)
        }
    }
    if (bad) atomicOr(&problems, bad);
    int n_free = 0;
    if (wave == 0) {
        const int f = lane < units ? unit_at[lane] : 0, before = wave_before(f, n_free);
        if (lane < units) unit_at[lane] = before;
        if (lane == 0) unit_at[units] = n_free;
    }
    __syncthreads();
    const int listed = n_listed;
    const bool in_list = listed <= kFewWriters;
    if (!in_list) {
        if (shared)
            for (int i = x.first; i < x.shared_to; ++i) {
                const int page = row[i];
                if (in_pool(a, page) && a.refs[page] > 1) atomicAdd(a.writers + page, 1), atomicMax(a.last + page, b);
            }
        __syncthreads();
    }
    // whether the sequence's page i is shared and does not stay with it
    auto goes = [&](int page) {
        if (!in_list) return moves(a, b, page);
        if (!in_pool(a, page)) return false;
        const int r = a.refs[page];
        if (r <= 1) return false;
        int at = place(page);
        while (key[at] != page) {
            if (key[at] == -1) return false;  // (not in the table: its refs were others a moment ago)
            at = (at + 1) % (2 * kFewWriters);
        }
        return !(n_writers[at] == r && last_writer[at] == b);
    };
    int c = max(0, x.need - max(x.shared_to, had)), copy = 0;
    uint64_t which = 0;  // of the first 64 pages that are written, those that go; of those behind them the entry itself says it, as ~page
    const bool some_bad = problems & 2;  // (nothing is handed out: counted all the same, for CLIMBER_POOL_FULL)
    if (shared)
        for (int i = x.first; i < x.shared_to; ++i) {
            if (!goes(row[i])) continue;
            ++c;
            if (some_bad) continue;
            copy |= i == x.first && x.part > 0;
            if (i - x.first < 64) which |= 1ull << (i - x.first);
            else row[i] = ~row[i];
        }
    int all_new, all_copies, at = wave_before(c, all_new), at_copy = wave_before(copy, all_copies);
    if (lane == 0) sums[0][wave] = all_new, sums[1][wave] = all_copies, sums[2][wave] = n_used;
    __syncthreads();
    int total = 0, n_copies = 0, in_use = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        if (i < wave) at += sums[0][i], at_copy += sums[1][i];
        total += sums[0][i], n_copies += sums[1][i], in_use += sums[2][i];
    }
    const bool full = (problems & 1) || total > unit_at[units], go = !full && !some_bad;
    if (t == 0) {
        const int found = (full ? CLIMBER_POOL_FULL : 0) | (some_bad ? CLIMBER_BAD_PAGE : 0);
        if (found) atomicOr(a.status, found);
        a.counts[0] = go ? n_copies : 0;
        a.counts[1] = in_use + (go ? total : 0);
    }
    if (!go) {
        if (shared && !some_bad)
            for (int i = x.first + 64; i < x.shared_to; ++i)
                if (row[i] < 0) row[i] = ~row[i];
        return;
    }
    for (int u = wave; u < units; u += 16) {
        int to0 = unit_at[u];
        if (to0 >= total) break;
#pragma unroll 1
        for (int i = 0; i < 16; ++i) {
            const uint64_t w = words[u * 16 + i];
            const int to = to0 + below(w);
            if (((w >> lane) & 1) && to < total) {
                const int page = u * kUnitPages + i * 64 + lane;
                if (to < kListPages) list[to] = page;
                else a.free_list[to] = page;
            }
            to0 += __popcll(w);
        }
    }
    // New pages of a sequence that gets more than a few: by all threads, each looking for the sequence of its page (eight sequences of 421 pages, half of
    // which come back: the run 129 / 41 us).  In place of the table, which nobody reads any more: the sequence's first page of the call, what makes
    // a page's place of its number, the first place.
    static_assert(2 * kFewWriters >= kFewSeqs);
    const int fresh_pages = max(0, x.need - had);
    const bool is_long = fresh_pages > kFewNew;
    key[t] = at, n_writers[t] = had - (at + c - fresh_pages), last_writer[t] = is_long ? had : 0x7fffffff;
    if (is_long) some_long = 1;
    __syncthreads();  // (and all have made up their minds: refs change from here on)
    auto take = [&](int i) { return i < kListPages ? list[i] : fresh(a.free_list + i); };
    if (shared)
        for (int i = x.first; i < x.shared_to; ++i) {
            const int e = row[i], page = e < 0 ? ~e : e;
            if (i - x.first < 64 ? !((which >> (i - x.first)) & 1) : e >= 0) continue;
            const int to = take(at++);
            row[i] = to;
            a.refs[to] = 1;
            atomicSub(a.refs + page, 1);
            if (i == x.first && x.part > 0) {
                int32_t *const o = a.copies + 3 * (int64_t)at_copy;
                o[0] = page, o[1] = to, o[2] = x.part;
            }
        }
    if (!is_long)
        for (int i = had; i < x.need; ++i) {
            const int to = take(at++);
            row[i] = to;
            a.refs[to] = 1;
        }
    if (some_long)
        for (int j = t; j < total; j += 1024) {
            int lo = 0, hi = a.n_seqs;  // (the last sequence whose first page is not behind page j)
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (key[mid] <= j) lo = mid;
                else hi = mid;
            }
            const int i = j + n_writers[lo];
            if (i < last_writer[lo]) continue;
            const int to = take(j);
            a.table[(int64_t)lo * a.table_ld + i] = to;
            a.refs[to] = 1;
        }
    if (mine && x.need > had) a.held[b] = x.need;
}

// ---- compact -------------------------------------------------------------------------------------
__global__ __launch_bounds__(256) void compact_look_kernel(const CompactArgs a)
{
    const int unit = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (unit < (int)pool_units(a.n_pages)) look(a.refs, a.n_pages, unit, false, a.bits, nullptr, a.unit_used);
}
// sum of the units' pages in use over threads of a workgroup of 256: of all units, and of those before `unit`
static __device__ __forceinline__ void used_before(const CompactArgs &a, int unit, int &all, int &before, int (*scratch)[4])
{
    const int units = (int)pool_units(a.n_pages);
    int x = 0, y = 0;
    for (int u = threadIdx.x; u < units; u += 256) {
        const int n = a.unit_used[u];
        x += n;
        y += u < unit ? n : 0;
    }
    int sx, sy;
    wave_before(x, sx), wave_before(y, sy);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) scratch[0][threadIdx.x >> 6] = sx, scratch[1][threadIdx.x >> 6] = sy;
    __syncthreads();
    all = scratch[0][0] + scratch[0][1] + scratch[0][2] + scratch[0][3];
    before = scratch[1][0] + scratch[1][1] + scratch[1][2] + scratch[1][3];
}
// A workgroup for four units: the pages in use behind the end of the compact pool, and the free ones before it, each numbered in order.
__global__ __launch_bounds__(256) void compact_list_kernel(const CompactArgs a)
{
    __shared__ int scratch[2][4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, unit0 = blockIdx.x * 4, units = (int)pool_units(a.n_pages);
    int n_used, before, x;
    used_before(a, unit0, n_used, before, scratch);
    for (int u = unit0; u < unit0 + wave && u < units; ++u) before += a.unit_used[u];
    // pages in use below the end
    const int end_unit = n_used / kUnitPages;
    int low;
    used_before(a, end_unit, x, low, scratch);
    if (end_unit < units) {
        uint64_t w = lane < 16 ? a.bits[(int64_t)end_unit * 16 + lane] : 0;
        const int rest = n_used - end_unit * kUnitPages - lane * 64;
        w &= rest >= 64 ? ~0ull : rest <= 0 ? 0ull : (1ull << rest) - 1;
        int n;
        wave_before(__popcll(w), n);
        low += n;
    }
    const int unit = unit0 + wave;
    if (unit >= units) return;
    if (unit == 0 && lane == 0) a.counts[0] = n_used - low, a.counts[1] = n_used;
    const uint64_t mine = lane < 16 ? a.bits[(int64_t)unit * 16 + lane] : 0;
#pragma unroll 1
    for (int i = 0; i < 16; ++i) {
        const uint64_t w = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)mine, i) |
                           (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(mine >> 32), i) << 32;
        const int page = unit * kUnitPages + i * 64 + lane, rank = before + below(w);
        const bool used = (w >> lane) & 1;
        if (page < a.n_pages) {
            if (page < n_used) {
                if (!used) a.holes[page - rank] = page;
            } else if (used) {
                a.to[page] = rank - low;
                a.movers[rank - low] = page;
            }
        }
        before += __popcll(w);
    }
}
// All of it by one workgroup: lists and bits in LDS but for the pages' new places.
__global__ __launch_bounds__(1024) void compact_few_kernel(const CompactArgs a)
{
    __shared__ uint64_t words[kFewUnits * 16];
    __shared__ int word_at[kFewUnits * 16], sums[16];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6, units = (int)pool_units(a.n_pages), n_words = units * 16;
    for (int u = wave; u < units; u += 16) {
        int r[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int64_t p = (int64_t)u * kUnitPages + i * 64 + lane;
            r[i] = p < a.n_pages ? a.refs[p] : -1;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const uint64_t w = __builtin_amdgcn_ballot_w64(r[i] > 0);
            if (lane == 0) words[u * 16 + i] = w;
        }
    }
    __syncthreads();
    // pages in use before each word of 64 (kFewUnits * 16 words, a thread each)
    int n_used;
    const int before = group_before(t < n_words ? __popcll(words[t]) : 0, n_used, sums);
    if (t < n_words) word_at[t] = before;
    __syncthreads();
    int low = n_used;  // pages in use below the end
    if (n_used >> 6 < n_words) {
        const int rest = n_used & 63;
        low = word_at[n_used >> 6] + (rest ? __popcll(words[n_used >> 6] & ((1ull << rest) - 1)) : 0);
    }
    if (t == 0) a.counts[0] = n_used - low, a.counts[1] = n_used;
    // pages in use behind the end, in order; free ones before it
    for (int i = wave; i < n_words; i += 16) {
        const uint64_t w = words[i];
        const int page = i * 64 + lane, rank = word_at[i] + below(w);
        const bool used = (w >> lane) & 1;
        if (page >= a.n_pages) continue;
        if (page < n_used && !used) a.holes[page - rank] = page;
        if (page >= n_used && used) a.movers[rank - low] = page;
    }
    __syncthreads();
    for (int i = t; i < n_used - low; i += 1024) {
        const int from = a.movers[i], to = a.holes[i];
        int32_t *const c = a.copies + 3 * (int64_t)i;
        c[0] = from, c[1] = to, c[2] = 1 << a.page_shift;
        a.refs[to] = a.refs[from];
        a.refs[from] = 0;
    }
    bool bad = false;
    const int all = a.n_seqs * a.table_ld;
#pragma unroll 4
    for (int e = t; e < all; e += 1024) {
        const int b = e / a.table_ld, page = a.table[e];
        if (e - b * a.table_ld >= held_of(a, b)) continue;
        const uint64_t w = in_pool(a, page) ? words[page >> 6] : 0;
        if (!((w >> (page & 63)) & 1)) bad = true;  // (no page, or one that nothing is said to hold)
        else if (page >= n_used) a.table[e] = a.holes[word_at[page >> 6] + __popcll(w & ((1ull << (page & 63)) - 1)) - low];
    }
    if (bad) atomicOr(a.status, CLIMBER_BAD_PAGE);
}
__global__ __launch_bounds__(256) void compact_move_kernel(const CompactArgs a, int pair_groups, int pieces)
{
    const int n = a.counts[0], n_used = a.counts[1];
    if ((int)blockIdx.x < pair_groups) {
        for (int i = blockIdx.x * 256 + threadIdx.x; i < n; i += pair_groups * 256) {
            const int from = a.movers[i], to = a.holes[i];
            int32_t *const c = a.copies + 3 * (int64_t)i;
            c[0] = from, c[1] = to, c[2] = 1 << a.page_shift;
            a.refs[to] = a.refs[from];
            a.refs[from] = 0;
        }
        return;
    }
    const int g = blockIdx.x - pair_groups, b = g / pieces * 4 + (threadIdx.x >> 6);
    if (b >= a.n_seqs) return;
    const int had = held_of(a, b);
    bool bad = false;
    for (int i = g % pieces * 64 + (threadIdx.x & 63); i < had; i += 64 * pieces) {
        int32_t *const e = a.table + (int64_t)b * a.table_ld + i;
        const int page = *e;
        // (a.bits: what was in use before the moves that other workgroups make meanwhile)
        if (!in_pool(a, page) || !((a.bits[page >> 6] >> (page & 63)) & 1)) bad = true;  // (no page, or one that nothing is said to hold)
        else if (page >= n_used) *e = a.holes[a.to[page]];
    }
    if (bad) atomicOr(a.status, CLIMBER_BAD_PAGE);
}

// ---- copy ----------------------------------------------------------------------------------------
// A workgroup for the keys or the values of a head of a copied page, 16 bytes a thread and pass; bound by memory: 297 MB read and written in 111 us
// (5.3 TB/s; a large copy 5.1).
__global__ __launch_bounds__(256) void pages_copy_kernel(const CopyArgs a)
{
    const int n = min(max(a.counts[0], 0), a.max_copies), per = 2 * a.Hkv, page = 1 << a.page_shift, tid = threadIdx.x;
    const int64_t units = (int64_t)n * per;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const int64_t i = u / per;
        const int hv = (int)(u % per), h = hv >> 1;
        const int from = a.copies[3 * i], to = a.copies[3 * i + 1], tokens = min(max(a.copies[3 * i + 2], 0), page);
        if (from < 0 || from >= a.n_pages || to < 0 || to >= a.n_pages || from == to) continue;
        const int64_t row = (int64_t)a.row_bytes << a.page_shift, src = ((int64_t)from * a.Hkv + h) * row, dst = ((int64_t)to * a.Hkv + h) * row;
        uint8_t *const base = hv & 1 ? a.v : a.k;
        const uint4 *const x = (const uint4 *)(base + src);
        uint4 *const y = (uint4 *)(base + dst);
        const int pieces = tokens * (a.row_bytes >> 4);
        int j = tid;
        for (; j + 768 < pieces; j += 1024) {
            const uint4 p = x[j], q = x[j + 256], r = x[j + 512], s = x[j + 768];
            y[j] = p, y[j + 256] = q, y[j + 512] = r, y[j + 768] = s;
        }
        for (; j < pieces; j += 256) y[j] = x[j];
        if (a.k_scale) {
            uint8_t *const s = hv & 1 ? a.v_scale : a.k_scale;
            const int64_t per_head = page >> 4;
            for (int e = tid; e < (tokens + 15) >> 4; e += 256) s[((int64_t)to * a.Hkv + h) * per_head + e] = s[((int64_t)from * a.Hkv + h) * per_head + e];
        }
        if (hv == 0)
            for (int e = tid; e < tokens; e += 256) {
                if (a.mass) a.mass[((int64_t)to << a.page_shift) + e] = a.mass[((int64_t)from << a.page_shift) + e];
                if (a.stamp) a.stamp[((int64_t)to << a.page_shift) + e] = a.stamp[((int64_t)from << a.page_shift) + e];
            }
    }
}

}  // namespace

hipError_t launch_pages_fork(const ForkArgs &a, hipStream_t s)
{
    if ((int64_t)a.n_seqs * a.table_ld <= kForkFew) {
        hipLaunchKernelGGL(fork_few_kernel, dim3(1), dim3(1024), 0, s, a);
        return hipGetLastError();
    }
    const dim3 grid((unsigned)((a.n_seqs + 3) / 4), (unsigned)row_waves(a));
    hipLaunchKernelGGL(fork_read_kernel, grid, dim3(256), 0, s, a);
    hipLaunchKernelGGL(fork_write_kernel, grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_pages_extend(const ExtendArgs &a, hipStream_t s)
{
    if (a.n_seqs <= kFewSeqs && pool_units(a.n_pages) <= kFewUnits) {
        hipLaunchKernelGGL(extend_few_kernel, dim3(1), dim3(1024), 0, s, a);
        return hipGetLastError();
    }
    const int unit_groups = (int)((pool_units(a.n_pages) + 3) / 4), seq_groups = std::min(1024, (a.n_seqs + 255) / 256);
    hipLaunchKernelGGL(extend_look_kernel, dim3((unsigned)(unit_groups + seq_groups)), dim3(256), 0, s, a, unit_groups);
    hipLaunchKernelGGL(extend_writers_kernel, dim3((unsigned)seq_groups), dim3(256), 0, s, a);
    hipLaunchKernelGGL(extend_share_kernel, dim3(1), dim3(1024), 0, s, a);
    hipLaunchKernelGGL(extend_write_kernel, dim3((unsigned)((a.n_seqs + 3) / 4)), dim3(256), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_pages_compact(const CompactArgs &a, hipStream_t s)
{
    if ((int64_t)a.n_seqs * a.table_ld <= kCompactFew && pool_units(a.n_pages) <= kFewUnits) {
        hipLaunchKernelGGL(compact_few_kernel, dim3(1), dim3(1024), 0, s, a);
        return hipGetLastError();
    }
    const unsigned units = (unsigned)((pool_units(a.n_pages) + 3) / 4);
    const int pair_groups = (int)std::min<int64_t>(1024, (a.n_pages / 2 + 255) / 256 + 1);
    hipLaunchKernelGGL(compact_look_kernel, dim3(units), dim3(256), 0, s, a);
    hipLaunchKernelGGL(compact_list_kernel, dim3(units), dim3(256), 0, s, a);
    hipLaunchKernelGGL(compact_move_kernel, dim3((unsigned)(pair_groups + (a.n_seqs + 3) / 4 * row_waves(a))), dim3(256), 0, s, a, pair_groups, row_waves(a));
    return hipGetLastError();
}

hipError_t launch_pages_copy(const CopyArgs &a, hipStream_t s)
{
    const int64_t units = (int64_t)a.max_copies * 2 * a.Hkv;
    hipLaunchKernelGGL(pages_copy_kernel, dim3((unsigned)std::min<int64_t>(units, 4096)), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace climber
