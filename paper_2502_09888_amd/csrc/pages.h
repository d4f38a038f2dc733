// The pages of paged caches: what the kernels that hand them out, share, move and copy them are given (internal).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace climber {

constexpr int kUnitPages = 1024;  // pages of a wave that looks for free ones: 16 words of 64 bits

struct PoolArgs {
    int32_t *refs, *table, *held, *len;  // [n_pages], [n_seqs][table_ld], [n_seqs], [n_seqs]
    int32_t n_pages, page_shift, n_seqs, table_ld;
    int32_t *status;
};

struct ForkArgs : PoolArgs {
    const int32_t *parent, *keep;
    // workspace
    int32_t *rows, *new_len, *new_held, *entries;  // [n_seqs][table_ld], [n_seqs], [n_seqs], [n_seqs]
};

struct ExtendArgs : PoolArgs {
    const int32_t *rows;
    int32_t *copies, *counts;
    // workspace
    uint64_t *bits;                         // [units][16]: page is free
    int32_t *unit_free, *unit_used;         // [units]
    int32_t *writers, *last;                // [n_pages]: sequences that write a shared page, and the last of them
    int32_t *free_list;                     // [n_pages]
    int32_t *first_new, *first_copy, *go;   // [n_seqs], [n_seqs], [1]
};

struct CompactArgs : PoolArgs {
    int32_t *copies, *counts;
    // workspace
    uint64_t *bits;                         // [units][16]: page is in use
    int32_t *unit_used;                     // [units]
    int32_t *movers, *holes, *to;           // [n_pages / 2 + 1], [n_pages / 2 + 1], [n_pages]
};

struct CopyArgs {
    uint8_t *k, *v, *k_scale, *v_scale;     // scales: nullptr but for a cache in 8 bits
    int32_t *mass, *stamp;                  // 4 bytes a token each, or nullptr
    const int32_t *copies, *counts;
    int32_t n_pages, page_shift, Hkv, row_bytes, max_copies;
};

static __host__ __device__ inline int64_t pool_units(int64_t n_pages) { return (n_pages + kUnitPages - 1) / kUnitPages; }

hipError_t launch_pages_fork(const ForkArgs &a, hipStream_t s);
hipError_t launch_pages_extend(const ExtendArgs &a, hipStream_t s);
hipError_t launch_pages_compact(const CompactArgs &a, hipStream_t s);
hipError_t launch_pages_copy(const CopyArgs &a, hipStream_t s);

}  // namespace climber
