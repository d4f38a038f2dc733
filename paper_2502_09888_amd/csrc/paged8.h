// The paged history cache in 8 bits: what its kernels are given beside the arguments of a paged call (internal).
#pragma once
#include "paged.h"

namespace climber {

constexpr int kScaleBlock = 16, kLeastScale = 10;  // tokens of a scale; the least one, as stored: 2^(10 - 127)

struct Paged8Args : PagedArgs {
    uint8_t *k_scale, *v_scale;  // [n_pages][Hkv][page / 16]
    int store_blocks;            // blocks of 16 tokens that a sequence's new ones can touch; 0: nothing is stored
};

// Packed rows of a workgroup.  256 (two blocks of rows a wave, heads of 64): where that leaves a workgroup for each CU; us with 128 / 256: 6 users' 176
// candidates 7.5 / 10.7, 257 rows of one user on 560, 64 query and 8 cache heads, 23.8 / 31.7, but 512 of each of 64 users on 1024 108 / 103.
// 32: the kernel for few rows, whose waves share out keys, also for several tiles of a head where these are soon done: it needs fewer launches
// and no parts, tiles of 128 read and widen a key for more rows.  us with 128 / 32, heads of 128 but for the last: 12 candidates of 16 users on 600 18.9 / 12.4
// (256 workgroups of 32), 200 of one on 600 20.2 / 12.3 (200), 30 of 16 on 4000 62.6 / 42.2 (512); but more of them: 64 of 16 on 600 23.2 / 27.7 (1024), long
// ones: 200 of one on 20000 91 / 115, short ones of many: 30 of 50 on 60 9.9 / 12.4 (500).  Of 64 rows and fewer a tile of 128 is half empty: 12 of 100 on 1000
// 33 / 25 (1600), heads of 64.  Over 596 shapes the rule's choice takes 1.014 times the better one's (always 128 1.16, always 32 1.05).
static inline int paged8_tile_rows(int d, int64_t rows, int64_t groups, int64_t max_len)
{
    const int64_t n32 = (rows + 31) / 32 * groups;
    if (rows <= 32 || ((n32 <= 256 || max_len >= 256) && (rows <= 64 || (n32 <= (d == 64 ? 1024 : 512) && n32 * max_len <= 3000000)))) return 32;
    return d == 64 && rows > 128 && (rows + 255) / 256 * groups >= 256 ? 256 : 128;
}
static inline int64_t paged8_store_blocks(int64_t m_max) { return (m_max + 2 * kScaleBlock - 2) / kScaleBlock; }

// attention, the join of its parts, and the call's new tokens into their pages
hipError_t launch_attn_paged8(const Paged8Args &a, hipStream_t s);

}  // namespace climber
