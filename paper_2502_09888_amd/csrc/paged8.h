// The paged history cache in 8 bits: what its kernels are given beside the arguments of a paged call (internal).
#pragma once
#include "paged.h"

namespace climber {

constexpr int kScaleBlock = 16, kLeastScale = 10;  // tokens of a scale; the least one, as stored: 2^(10 - 127)

struct Paged8Args : PagedArgs {
    uint8_t *k_scale, *v_scale;  // [n_pages][Hkv][page / 16]
    int store_blocks;            // blocks of 16 tokens that a sequence's new ones can touch; 0: nothing is stored
};

// Packed rows of a workgroup.  32: the kernel for few rows, whose waves share out keys.  256 (two blocks of rows a wave, heads of 64): where that leaves a workgroup
// for each CU; us with 128 / 256: 6 users' 176 candidates 7.5 / 10.7, 257 rows of one user on 560, 64 query and 8 cache heads, 23.8 / 31.7, but 512
// of each of 64 users on 1024 108 / 103.
static inline int paged8_tile_rows(int d, int64_t rows, int64_t groups) { return rows <= 32 ? 32 : d == 64 && rows > 128 && (rows + 255) / 256 * groups >= 256 ? 256 : 128; }
static inline int64_t paged8_store_blocks(int64_t m_max) { return (m_max + 2 * kScaleBlock - 2) / kScaleBlock; }

// attention, the join of its parts, and the call's new tokens into their pages
hipError_t launch_attn_paged8(const Paged8Args &a, hipStream_t s);

}  // namespace climber
