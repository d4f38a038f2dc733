// What the host sides of the paged caches share (internal): argument validation, the split of the keys, workspace layout.
#pragma once
#include "../../include/climber.h"

#include <algorithm>
#include <cmath>

#include "internal.h"
#include "paged.h"

namespace climber {
namespace paged_host {

static inline size_t up(size_t x) { return (x + 255) / 256 * 256; }
static inline bool aligned(const void *p, size_t a) { return ((uintptr_t)p % a) == 0; }
static inline int rt(hipError_t e) { return e == hipSuccess ? CLIMBER_OK : CLIMBER_ERR_RUNTIME; }
static inline size_t elem_of(const climber_config *cfg) { return cfg->dtype == CLIMBER_BF16 ? 2 : 4; }

// sizes of a cache and its configuration, without its pointers; `bytes`: of an element of the cache, 0: the configuration's
static inline int check_sizes(const climber_config *cfg, const climber_paged_kv *kv, int32_t bytes = 0)
{
    int e = check_config_values(cfg);
    if (e) return e;
    if (!kv) return CLIMBER_ERR_NULL;
    if (cfg->dtype == CLIMBER_BF16 ? cfg->d_head != 64 && cfg->d_head != 128 : cfg->d_head % 4 != 0 || cfg->d_head > 128)
        return CLIMBER_ERR_UNSUPPORTED;
    if (kv->n_pages < 1 || kv->n_seqs < 1 || kv->table_ld < 1 || kv->n_kv_heads < 1 || cfg->n_heads % kv->n_kv_heads != 0 || kv->page_size < 1)
        return CLIMBER_ERR_SHAPE;
    if ((kv->d_head != 0 && kv->d_head != cfg->d_head) || (kv->elem_bytes != 0 && kv->elem_bytes != (bytes ? bytes : (int32_t)elem_of(cfg)))) return CLIMBER_ERR_SHAPE;
    if (kv->page_size < 16 || kv->page_size > 4096 || (kv->page_size & (kv->page_size - 1)) != 0) return CLIMBER_ERR_ALIGN;
    if (kv->max_len < 0 || kv->max_len > (int64_t)kv->table_ld * kv->page_size) return CLIMBER_ERR_RANGE;
    // slots of a table row, rows of a launch and tokens of the pool are counted in 32 bits
    if ((int64_t)kv->table_ld * kv->page_size >= (int64_t)1 << 30 || (int64_t)kv->n_pages * kv->page_size >= (int64_t)1 << 31) return CLIMBER_ERR_RANGE;
    // a launch has less than 2^32 threads: 256 for 256 tokens of a sequence and cache head (attention weights), 1024 for 4096 of a sequence
    // (eviction)
    if ((int64_t)kv->n_seqs * kv->n_kv_heads * (((int64_t)kv->max_len + 511) / 256 * 256) >= (int64_t)1 << 32) return CLIMBER_ERR_RANGE;
    if (kv->n_seqs * std::max<int64_t>(1, evict_segments(kv->max_len)) >= (int64_t)1 << 22) return CLIMBER_ERR_RANGE;
    return CLIMBER_OK;
}

static inline int check_sizes8(const climber_config *cfg, const climber_paged_kv8 *kv8)
{
    if (!cfg || !kv8) return CLIMBER_ERR_NULL;
    const int e = check_sizes(cfg, &kv8->kv, 1);
    if (e) return e;
    return cfg->dtype != CLIMBER_BF16 || kv8->kv.mass ? CLIMBER_ERR_UNSUPPORTED : CLIMBER_OK;
}

static inline int check_rows(const climber_config *cfg, int32_t m_total, int32_t m_max)
{
    if (m_total < 0 || m_max < 0 || m_max > m_total || (m_total > 0 && m_max == 0)) return CLIMBER_ERR_SHAPE;
    if ((int64_t)m_total * cfg->d_model >= (int64_t)1 << 31) return CLIMBER_ERR_RANGE;
    return CLIMBER_OK;
}

static inline int check_pointers(const climber_paged_kv *kv)
{
    if (!kv->k || !kv->v || !kv->page_table || !kv->len) return CLIMBER_ERR_NULL;
    if (!aligned(kv->k, 16) || !aligned(kv->v, 16) || !aligned(kv->page_table, 4) || !aligned(kv->len, 4) || !aligned(kv->mass, 4) || !aligned(kv->stamp, 4))
        return CLIMBER_ERR_ALIGN;
    return CLIMBER_OK;
}

constexpr int64_t kMostGroups = 1 << 24;  // workgroups of 256 threads of a launch
// Rows x heads x parts that a call's partial results have room for at most, and parts.
static inline int64_t part_rows(const climber_paged_kv *kv) { return std::min<int64_t>(4, std::max<int64_t>(1, kv->max_len / 4096)) << 16; }
static inline int64_t most_parts(const climber_paged_kv *kv) { return std::min<int64_t>(512, std::max<int64_t>(1, kv->max_len / 32)); }

// Parts of the keys: up to two workgroups per CU (in bf16, whose parts cost less beside their keys' work, two that are expected to have
// rows), and as many as are worth it.  In us, fitted to sweeps: a workgroup needs per_key for each key and d_head's unit; a join is a launch of 3.5,
// and each part costs it 0.1 and its rows, written and read again.  One / chosen parts: 128 candidates of one user on 1000 16 / 13, three
// sessions on up to 4000 96 / 66, candidates of twelve users on up to 20000 400 / 166, one fp32 row on 1000 22 / 15; parts / one where the rows are
// many and the keys few: 18 prompts of up to 268 31 / 18, eight of up to 700 35 / 28.
static inline int parts(const climber_config *cfg, const climber_paged_kv *kv, int32_t m_total, int32_t m_max, int64_t tile)
{
    const bool bf16 = cfg->dtype == CLIMBER_BF16;
    const int64_t rows = (int64_t)m_max * (cfg->n_heads / kv->n_kv_heads), out = std::max<int64_t>(1, (int64_t)m_total * cfg->n_heads);
    const int64_t heads = (int64_t)kv->n_seqs * kv->n_kv_heads;
    const double with_rows = bf16 ? (double)m_total / ((double)kv->n_seqs * std::max(1, m_max)) : 1.0;
    const int64_t groups = std::max<int64_t>(1, (int64_t)(std::min(1.0, with_rows) * (double)((rows + tile - 1) / tile * heads)));
    const int64_t unit = bf16 && tile == 32 ? 128 : 32;  // keys that a workgroup takes at once
    const int64_t most = std::min(std::min(512 / groups, part_rows(kv) / out), std::min(most_parts(kv), kv->max_len / unit));
    if (most < 2) return 1;
    const double per_key = bf16 ? (tile == 32 ? 9e-5 : tile == 128 ? 2e-4 : 3.5e-4) : tile == 32 ? 3.5e-4 : 9e-4;
    const double one = per_key * cfg->d_head * kv->max_len, each = 0.1 + 8.0 * cfg->d_head * (double)out / 2.5e6;
    const int64_t n = std::min<int64_t>(most, (int64_t)(std::sqrt(one / each) + 0.5));
    return n > 1 && one / (double)n + 3.5 + each * (double)n < one ? (int)n : 1;
}

static inline size_t logits_pitch(const climber_paged_kv *kv) { return ((size_t)kv->max_len + 31) / 32 * 32; }

struct Layout {  // of the workspace
    size_t part_o, part_ml, lse, mass, bytes;
};
// for partial results of `part_rows` rows x heads x parts
static inline Layout layout_of(const climber_config *cfg, const climber_paged_kv *kv, int32_t m_total, size_t part_rows)
{
    Layout w{};
    w.part_o = 0;
    w.part_ml = w.part_o + up(part_rows * cfg->d_head * 4);
    w.lse = w.part_ml + up(part_rows * 8);
    w.mass = w.bytes = w.lse + (kv->mass ? up((size_t)m_total * cfg->n_heads * 8) : 0);
    if (kv->mass) {
        // sums of the rows' parts (more than one: of at most kMassGroups workgroups), or the logits of few rows (a call may have fewer rows
        // than it is asked for here)
        const size_t groups = (size_t)kv->n_seqs * kv->n_kv_heads, G = cfg->n_heads / kv->n_kv_heads;
        const size_t few = kMassFewRows / G * G * logits_pitch(kv);
        w.bytes += up(std::max(groups * kv->max_len + (size_t)kMassGroups * kMassKeys, groups * few) * 4);
    }
    return w;
}

static inline int page_shift(int page) { return __builtin_ctz((unsigned)page); }

// Two arrays of rows share an element: not if they lie apart, or are columns of the same rows that lie apart.
static inline bool overlap(const void *a, int64_t ld_a, size_t wide_a, const void *b, int64_t ld_b, size_t wide_b, int64_t rows)
{
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    const uintptr_t x1 = x + (rows - 1) * ld_a + wide_a, y1 = y + (rows - 1) * ld_b + wide_b;
    if (x1 <= y || y1 <= x) return false;
    if (ld_a != ld_b) return true;
    const uintptr_t d = x < y ? y - x : x - y, in = d % (uintptr_t)ld_a;  // the later one's columns behind the earlier one's
    const size_t first = x < y ? wide_a : wide_b, second = x < y ? wide_b : wide_a;
    return !(in >= first && in + second <= (uintptr_t)ld_a);
}

// The arguments of an attention call.
struct Call {
    const climber_config *cfg;
    const float *tau;
    const climber_paged_kv *kv;
    const void *q, *k, *v;
    int64_t ld_q, ld_kv;
    const int32_t *off;
    int32_t m_total, m_max;
    const int32_t *scen, *beh, *stamp;
    void *o;
    int64_t ld_o;
    bool sumi;
};

// ... behind check_sizes and check_rows.  `nothing`: no rows, and all is well.
static inline int check_call(const Call &c, bool &nothing)
{
    const climber_config *cfg = c.cfg;
    const climber_paged_kv *kv = c.kv;
    nothing = false;
    if (!c.sumi && cfg->sub_len != 0) return CLIMBER_ERR_UNSUPPORTED;
    const int64_t elem = (int64_t)elem_of(cfg), wide = cfg->d_model, kv_wide = (int64_t)kv->n_kv_heads * cfg->d_head;
    if (c.ld_q < wide || c.ld_o < wide || c.ld_kv < kv_wide) return CLIMBER_ERR_SHAPE;
    const int64_t most = (int64_t)1 << 24;  // (16 rows are addressed by 32 bits)
    if (c.ld_q > most || c.ld_kv > most || c.ld_o > most) return CLIMBER_ERR_RANGE;
    if (!c.tau || !c.off) return CLIMBER_ERR_NULL;
    const int e = check_pointers(kv);
    if (e) return e;
    nothing = c.m_total == 0;
    if (nothing) return CLIMBER_OK;  // their arrays are empty, their pointers free
    if (!c.q || !c.k || !c.v || !c.scen || !c.beh || !c.o || (!c.sumi && kv->stamp && !c.stamp)) return CLIMBER_ERR_NULL;
    if (!aligned(c.q, 16) || !aligned(c.k, 16) || !aligned(c.v, 16) || !aligned(c.o, 16) || c.ld_q * elem % 16 || c.ld_kv * elem % 16 || c.ld_o * elem % 16)
        return CLIMBER_ERR_ALIGN;
    if (!c.sumi && kv->max_len == 0) return CLIMBER_ERR_RANGE;
    // outputs are written while other workgroups still read rows
    if (overlap(c.o, c.ld_o * elem, wide * elem, c.k, c.ld_kv * elem, kv_wide * elem, c.m_total) ||
        overlap(c.o, c.ld_o * elem, wide * elem, c.v, c.ld_kv * elem, kv_wide * elem, c.m_total) ||
        overlap(c.o, c.ld_o * elem, wide * elem, c.q, c.ld_q * elem, wide * elem, c.m_total))
        return CLIMBER_ERR_UNSUPPORTED;
    return CLIMBER_OK;
}

// a call's arguments as its kernels get them
static inline void fill(PagedArgs &a, const Call &c, int n_split, uint8_t *ws, const Layout &w)
{
    const climber_config *cfg = c.cfg;
    const climber_paged_kv *kv = c.kv;
    const int64_t elem = (int64_t)elem_of(cfg);
    a.k_pages = (uint8_t *)kv->k;
    a.v_pages = (uint8_t *)kv->v;
    a.mass = kv->mass;
    a.stamp = kv->stamp;
    a.table = kv->page_table;
    a.len = kv->len;
    a.q = (const uint8_t *)c.q;
    a.k = (const uint8_t *)c.k;
    a.v = (const uint8_t *)c.v;
    a.ld_q = c.ld_q * elem;
    a.ld_kv = c.ld_kv * elem;
    a.ld_o = c.ld_o * elem;
    a.off = c.off;
    a.scen = c.scen;
    a.beh = c.beh;
    a.stamp_new = c.stamp;
    a.tau = c.tau;
    a.o = (uint8_t *)c.o;
    a.n_seqs = kv->n_seqs;
    a.n_pages = kv->n_pages;
    a.page_shift = page_shift(kv->page_size);
    a.table_ld = kv->table_ld;
    a.max_len = kv->max_len;
    a.H = cfg->n_heads;
    a.Hkv = kv->n_kv_heads;
    a.G = cfg->n_heads / kv->n_kv_heads;
    a.G_inv = (uint32_t)((((uint64_t)1 << 32) + a.G - 1) / a.G);
    a.d = cfg->d_head;
    a.row_bytes = (int)(cfg->d_head * elem);
    a.n_scen = cfg->n_scen;
    a.n_beh = cfg->n_beh;
    a.m_total = c.m_total;
    a.m_max = c.m_max;
    a.causal = (cfg->flags & CLIMBER_HIST_CAUSAL) ? 1 : 0;
    a.sumi = c.sumi;
    a.scale_log2e = cfg->qk_scale * 1.4426950408889634f;
    a.n_split = n_split;
    a.part_o = (float *)(ws + w.part_o);
    a.part_ml = (float *)(ws + w.part_ml);
    a.lse = kv->mass ? (float2 *)(ws + w.lse) : nullptr;
}

}  // namespace paged_host
}  // namespace climber
