// Host side of the paged history cache: argument validation, workspace layout and dispatch of its entry points (include/climber.h)
// onto the kernels.  Everything is validated before the first launch; nothing here allocates device memory.
#include "../../include/climber.h"

#include <algorithm>
#include <cmath>

#include "internal.h"
#include "paged.h"

using namespace climber;

namespace {

size_t up(size_t x) { return (x + 255) / 256 * 256; }
bool aligned(const void *p, size_t a) { return ((uintptr_t)p % a) == 0; }
int rt(hipError_t e) { return e == hipSuccess ? CLIMBER_OK : CLIMBER_ERR_RUNTIME; }
size_t elem_of(const climber_config *cfg) { return cfg->dtype == CLIMBER_BF16 ? 2 : 4; }

// sizes of a cache and its configuration, without its pointers
int check_sizes(const climber_config *cfg, const climber_paged_kv *kv)
{
    int e = check_config_values(cfg);
    if (e) return e;
    if (!kv) return CLIMBER_ERR_NULL;
    if (cfg->dtype == CLIMBER_BF16 ? cfg->d_head != 64 && cfg->d_head != 128 : cfg->d_head % 4 != 0 || cfg->d_head > 128)
        return CLIMBER_ERR_UNSUPPORTED;
    if (kv->n_pages < 1 || kv->n_seqs < 1 || kv->table_ld < 1 || kv->n_kv_heads < 1 || cfg->n_heads % kv->n_kv_heads != 0 || kv->page_size < 1)
        return CLIMBER_ERR_SHAPE;
    if ((kv->d_head != 0 && kv->d_head != cfg->d_head) || (kv->elem_bytes != 0 && kv->elem_bytes != (int32_t)elem_of(cfg))) return CLIMBER_ERR_SHAPE;
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

int check_rows(const climber_config *cfg, int32_t m_total, int32_t m_max)
{
    if (m_total < 0 || m_max < 0 || m_max > m_total || (m_total > 0 && m_max == 0)) return CLIMBER_ERR_SHAPE;
    if ((int64_t)m_total * cfg->d_model >= (int64_t)1 << 31) return CLIMBER_ERR_RANGE;
    return CLIMBER_OK;
}

int check_pointers(const climber_paged_kv *kv)
{
    if (!kv->k || !kv->v || !kv->page_table || !kv->len) return CLIMBER_ERR_NULL;
    if (!aligned(kv->k, 16) || !aligned(kv->v, 16) || !aligned(kv->page_table, 4) || !aligned(kv->len, 4) || !aligned(kv->mass, 4) || !aligned(kv->stamp, 4))
        return CLIMBER_ERR_ALIGN;
    return CLIMBER_OK;
}

constexpr int64_t kMostGroups = 1 << 24;  // workgroups of 256 threads of a launch
// Rows x heads x parts that a call's partial results have room for at most, and parts.
int64_t part_rows(const climber_paged_kv *kv) { return std::min<int64_t>(4, std::max<int64_t>(1, kv->max_len / 4096)) << 16; }
int64_t most_parts(const climber_paged_kv *kv) { return std::min<int64_t>(512, std::max<int64_t>(1, kv->max_len / 32)); }

// Parts of the keys: up to two workgroups per CU (in bf16, whose parts cost less beside their keys' work, two that are expected to have
// rows), and as many as are worth it.  In us, fitted to sweeps: a workgroup needs per_key for each key and d_head's unit; a join is a launch of 3.5,
// and each part costs it 0.1 and its rows, written and read again.  One / chosen parts: 128 candidates of one user on 1000 16 / 13, three
// sessions on up to 4000 96 / 66, candidates of twelve users on up to 20000 400 / 166, one fp32 row on 1000 22 / 15; parts / one where the rows are
// many and the keys few: 18 prompts of up to 268 31 / 18, eight of up to 700 35 / 28.
int parts(const climber_config *cfg, const climber_paged_kv *kv, int32_t m_total, int32_t m_max)
{
    const bool bf16 = cfg->dtype == CLIMBER_BF16;
    const int64_t rows = (int64_t)m_max * (cfg->n_heads / kv->n_kv_heads), out = std::max<int64_t>(1, (int64_t)m_total * cfg->n_heads);
    const int64_t heads = (int64_t)kv->n_seqs * kv->n_kv_heads, tile = paged_tile_rows(bf16, cfg->d_head, rows, heads);
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

size_t logits_pitch(const climber_paged_kv *kv) { return ((size_t)kv->max_len + 31) / 32 * 32; }

struct Layout {  // of the workspace
    size_t part_o, part_ml, lse, mass, bytes;
};
// for partial results of `part_rows` rows x heads x parts
Layout layout_of(const climber_config *cfg, const climber_paged_kv *kv, int32_t m_total, size_t part_rows)
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

struct EvictLayout {
    size_t holes, movers, n_moves, keys, first, hists, state, bytes;
};
EvictLayout evict_layout(const climber_paged_kv *kv)
{
    EvictLayout w{};
    const size_t B = kv->n_seqs, L = kv->max_len, S = evict_segments(kv->max_len);
    w.holes = 0;
    w.movers = w.holes + up(B * (L / 2 + 1) * 4);
    w.n_moves = w.movers + up(B * (L / 2 + 1) * 4);
    w.keys = w.n_moves + up(B * 4);
    w.first = w.keys + (S ? up(B * L * 4) : 0);
    w.hists = w.first + up(B * S * (kEvictSegment / 64) * 8);
    w.state = w.hists + up(B * S * kEvictSegInts * 4);
    w.bytes = w.state + up(B * 32);
    return w;
}

int page_shift(int page) { return __builtin_ctz((unsigned)page); }

// Two arrays of rows share an element: not if they lie apart, or are columns of the same rows that lie apart.
bool overlap(const void *a, int64_t ld_a, size_t wide_a, const void *b, int64_t ld_b, size_t wide_b, int64_t rows)
{
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    const uintptr_t x1 = x + (rows - 1) * ld_a + wide_a, y1 = y + (rows - 1) * ld_b + wide_b;
    if (x1 <= y || y1 <= x) return false;
    if (ld_a != ld_b) return true;
    const uintptr_t d = x < y ? y - x : x - y, in = d % (uintptr_t)ld_a;  // the later one's columns behind the earlier one's
    const size_t first = x < y ? wide_a : wide_b, second = x < y ? wide_b : wide_a;
    return !(in >= first && in + second <= (uintptr_t)ld_a);
}

int attn_paged(const climber_config *cfg, const float *tau, const climber_paged_kv *kv, const void *q, int64_t ld_q, const void *k, const void *v,
               int64_t ld_kv, const int32_t *off, int32_t m_total, int32_t m_max, const int32_t *scen, const int32_t *beh, const int32_t *stamp,
               void *o, int64_t ld_o, void *workspace, size_t ws_bytes, bool sumi, void *stream)
{
    int e = check_sizes(cfg, kv);
    if (e) return e;
    e = check_rows(cfg, m_total, m_max);
    if (e) return e;
    if (!sumi && cfg->sub_len != 0) return CLIMBER_ERR_UNSUPPORTED;
    const int64_t elem = (int64_t)elem_of(cfg), wide = cfg->d_model, kv_wide = (int64_t)kv->n_kv_heads * cfg->d_head;
    if (ld_q < wide || ld_o < wide || ld_kv < kv_wide) return CLIMBER_ERR_SHAPE;
    const int64_t most = (int64_t)1 << 24;  // (16 rows are addressed by 32 bits)
    if (ld_q > most || ld_kv > most || ld_o > most) return CLIMBER_ERR_RANGE;
    if (!tau || !off) return CLIMBER_ERR_NULL;
    e = check_pointers(kv);
    if (e) return e;
    if (m_total == 0) return CLIMBER_OK;  // no rows: their arrays are empty, their pointers free
    if (!q || !k || !v || !scen || !beh || !o || (!sumi && kv->stamp && !stamp)) return CLIMBER_ERR_NULL;
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(o, 16) || ld_q * elem % 16 || ld_kv * elem % 16 || ld_o * elem % 16)
        return CLIMBER_ERR_ALIGN;
    if (!sumi && kv->max_len == 0) return CLIMBER_ERR_RANGE;
    // outputs are written while other workgroups still read rows
    if (overlap(o, ld_o * elem, wide * elem, k, ld_kv * elem, kv_wide * elem, m_total) || overlap(o, ld_o * elem, wide * elem, v, ld_kv * elem, kv_wide * elem, m_total) ||
        overlap(o, ld_o * elem, wide * elem, q, ld_q * elem, wide * elem, m_total))
        return CLIMBER_ERR_UNSUPPORTED;
    const int n_split = parts(cfg, kv, m_total, m_max);
    const bool bf16 = cfg->dtype == CLIMBER_BF16;
    const int64_t G = cfg->n_heads / kv->n_kv_heads, heads = (int64_t)kv->n_seqs * kv->n_kv_heads, tile = paged_tile_rows(bf16, cfg->d_head, m_max * G, heads);
    if ((m_max * G + tile - 1) / tile * (heads + 7) * n_split >= kMostGroups) return CLIMBER_ERR_RANGE;
    if (kv->mass && !bf16 && heads * ((kv->max_len + 31) / 32) >= kMostGroups) return CLIMBER_ERR_RANGE;
    const Layout w = layout_of(cfg, kv, m_total, n_split > 1 ? (size_t)n_split * m_total * cfg->n_heads : 0);
    if (w.bytes > 0 && !workspace) return CLIMBER_ERR_NULL;
    if (!aligned(workspace, 256)) return CLIMBER_ERR_ALIGN;
    if (ws_bytes < w.bytes) return CLIMBER_ERR_BUFSIZE;

    uint8_t *ws = (uint8_t *)workspace;
    PagedArgs a{};
    a.k_pages = (uint8_t *)kv->k;
    a.v_pages = (uint8_t *)kv->v;
    a.mass = kv->mass;
    a.stamp = kv->stamp;
    a.table = kv->page_table;
    a.len = kv->len;
    a.q = (const uint8_t *)q;
    a.k = (const uint8_t *)k;
    a.v = (const uint8_t *)v;
    a.ld_q = ld_q * elem;
    a.ld_kv = ld_kv * elem;
    a.ld_o = ld_o * elem;
    a.off = off;
    a.scen = scen;
    a.beh = beh;
    a.stamp_new = stamp;
    a.tau = tau;
    a.o = (uint8_t *)o;
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
    a.m_total = m_total;
    a.m_max = m_max;
    a.causal = (cfg->flags & CLIMBER_HIST_CAUSAL) ? 1 : 0;
    a.sumi = sumi;
    a.scale_log2e = cfg->qk_scale * 1.4426950408889634f;
    a.n_split = n_split;
    a.part_o = (float *)(ws + w.part_o);
    a.part_ml = (float *)(ws + w.part_ml);
    a.lse = kv->mass ? (float2 *)(ws + w.lse) : nullptr;
    float *part = (float *)(ws + w.mass);
    const bool few = kv->mass && (int64_t)m_max * a.G <= kMassFewRows;
    if (few) {
        a.logits = part;
        a.logits_ld = (int)logits_pitch(kv);
    }
    const hipStream_t s = (hipStream_t)stream;
    e = rt(bf16 ? launch_attn_paged_bf16(a, s) : launch_attn_paged_f32(a, s));
    if (e) return e;
    if (a.n_split > 1) e = rt(launch_paged_combine(a, bf16, s));
    if (e || !kv->mass || kv->max_len == 0) return e;
    if (few) return rt(launch_paged_mass_few(a, s));
    const int row_parts = bf16 ? paged_mass_parts(kv->n_seqs, kv->n_kv_heads, kv->max_len, (int64_t)m_max * a.G) : 1;
    e = rt(bf16 ? launch_paged_mass_bf16(a, part, row_parts, s) : launch_paged_mass_f32(a, part, s));
    return e ? e : rt(launch_paged_mass_add(a, part, kv->n_kv_heads * row_parts, s));
}

}  // namespace

extern "C" {

size_t climber_paged_workspace_bytes(const climber_config *cfg, const climber_paged_kv *kv, int32_t m_total, int32_t m_max)
{
    if (check_sizes(cfg, kv) != CLIMBER_OK || check_rows(cfg, m_total, m_max) != CLIMBER_OK) return 0;
    // (a smaller call may have more parts: room for as many as one can have)
    const int64_t n = most_parts(kv) * m_total * cfg->n_heads;
    return std::max(layout_of(cfg, kv, m_total, most_parts(kv) > 1 ? (size_t)std::min(n, part_rows(kv)) : 0).bytes,
                    evict_segments(kv->max_len) <= kEvictMostSegments ? evict_layout(kv).bytes : 0);
}

int climber_attn_history_paged(const climber_config *cfg, const float *tau_layer, const climber_paged_kv *kv, const void *q, int64_t ld_q,
                               const void *k, const void *v, int64_t ld_kv, const int32_t *off, int32_t m_total, int32_t m_max,
                               const int32_t *scen, const int32_t *beh, const int32_t *stamp, void *o, int64_t ld_o, void *workspace,
                               size_t ws_bytes, void *stream)
{
    return attn_paged(cfg, tau_layer, kv, q, ld_q, k, v, ld_kv, off, m_total, m_max, scen, beh, stamp, o, ld_o, workspace, ws_bytes, false, stream);
}

int climber_attn_sumi_paged(const climber_config *cfg, const float *tau_layer, const climber_paged_kv *kv, const void *q_c, int64_t ld_q,
                            const void *k_c, const void *v_c, int64_t ld_kv, const int32_t *cand_off, int32_t m_total, int32_t m_max,
                            const int32_t *cand_scen, const int32_t *cand_beh, void *o_c, int64_t ld_o, void *workspace, size_t ws_bytes,
                            void *stream)
{
    return attn_paged(cfg, tau_layer, kv, q_c, ld_q, k_c, v_c, ld_kv, cand_off, m_total, m_max, cand_scen, cand_beh, nullptr, o_c, ld_o, workspace,
                      ws_bytes, true, stream);
}

int climber_paged_evict(const climber_config *cfg, const climber_paged_kv *kv, const float *rank, const int32_t *budget, const int32_t *keep_from,
                        int32_t *len_out, int32_t *src, void *workspace, size_t ws_bytes, void *stream)
{
    int e = check_sizes(cfg, kv);
    if (e) return e;
    e = check_pointers(kv);
    if (e) return e;
    if (!budget || !len_out || (!rank && !kv->mass) || (keep_from && !kv->stamp)) return CLIMBER_ERR_NULL;
    if (!aligned(rank, 4) || !aligned(budget, 4) || !aligned(keep_from, 4) || !aligned(len_out, 4) || !aligned(src, 4)) return CLIMBER_ERR_ALIGN;
    if (evict_segments(kv->max_len) > kEvictMostSegments) return CLIMBER_ERR_UNSUPPORTED;
    const EvictLayout w = evict_layout(kv);
    if (!workspace) return CLIMBER_ERR_NULL;
    if (!aligned(workspace, 256)) return CLIMBER_ERR_ALIGN;
    if (ws_bytes < w.bytes) return CLIMBER_ERR_BUFSIZE;
    uint8_t *ws = (uint8_t *)workspace;
    EvictArgs a{};
    a.k_pages = (uint8_t *)kv->k;
    a.v_pages = (uint8_t *)kv->v;
    a.mass = kv->mass;
    a.rank = rank ? rank : kv->mass;
    a.stamp = kv->stamp;
    a.table = kv->page_table;
    a.len = kv->len;
    a.budget = budget;
    a.keep_from = keep_from;
    a.len_out = len_out;
    a.src = src;
    a.n_seqs = kv->n_seqs;
    a.n_pages = kv->n_pages;
    a.page_shift = page_shift(kv->page_size);
    a.table_ld = kv->table_ld;
    a.max_len = kv->max_len;
    a.Hkv = kv->n_kv_heads;
    a.row_bytes = (int)(cfg->d_head * elem_of(cfg));
    a.segments = (int)evict_segments(kv->max_len);
    a.holes = (int32_t *)(ws + w.holes);
    a.movers = (int32_t *)(ws + w.movers);
    a.n_moves = (int32_t *)(ws + w.n_moves);
    a.keys = (uint32_t *)(ws + w.keys);
    a.first = (uint64_t *)(ws + w.first);
    a.hists = (int32_t *)(ws + w.hists);
    a.state = (int32_t *)(ws + w.state);
    return rt(launch_paged_evict(a, (hipStream_t)stream));
}

int climber_check_paged(const climber_config *cfg, const climber_paged_kv *kv, const int32_t *off, int32_t m_total, int32_t m_max, int32_t appends,
                        int32_t *status, void *stream)
{
    int e = check_sizes(cfg, kv);
    if (e) return e;
    e = check_rows(cfg, m_total, m_max);
    if (e) return e;
    if (!kv->page_table || !kv->len || !status || (appends && !off)) return CLIMBER_ERR_NULL;
    return rt(launch_check_paged(kv->page_table, kv->len, off, kv->n_seqs, kv->n_pages, page_shift(kv->page_size), kv->table_ld, kv->max_len, m_total,
                                 m_max, appends, status, (hipStream_t)stream));
}

}  // extern "C"
