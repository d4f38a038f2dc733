// Host side of the paged history cache: argument validation, workspace layout and dispatch of its entry points (include/climber.h)
// onto the kernels.  Everything is validated before the first launch; nothing here allocates device memory.
#include "paged_host.h"

using namespace climber;
using namespace climber::paged_host;

namespace {

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

int attn_paged(const Call &c, void *workspace, size_t ws_bytes, void *stream)
{
    const climber_config *cfg = c.cfg;
    const climber_paged_kv *kv = c.kv;
    int e = check_sizes(cfg, kv);
    if (e) return e;
    e = check_rows(cfg, c.m_total, c.m_max);
    if (e) return e;
    bool nothing;
    e = check_call(c, nothing);
    if (e || nothing) return e;
    const bool bf16 = cfg->dtype == CLIMBER_BF16;
    const int64_t G = cfg->n_heads / kv->n_kv_heads, heads = (int64_t)kv->n_seqs * kv->n_kv_heads, tile = paged_tile_rows(bf16, cfg->d_head, c.m_max * G, heads);
    const int n_split = parts(cfg, kv, c.m_total, c.m_max, tile);
    if ((c.m_max * G + tile - 1) / tile * (heads + 7) * n_split >= kMostGroups) return CLIMBER_ERR_RANGE;
    if (kv->mass && !bf16 && heads * ((kv->max_len + 31) / 32) >= kMostGroups) return CLIMBER_ERR_RANGE;
    const Layout w = layout_of(cfg, kv, c.m_total, n_split > 1 ? (size_t)n_split * c.m_total * cfg->n_heads : 0);
    if (w.bytes > 0 && !workspace) return CLIMBER_ERR_NULL;
    if (!aligned(workspace, 256)) return CLIMBER_ERR_ALIGN;
    if (ws_bytes < w.bytes) return CLIMBER_ERR_BUFSIZE;

    uint8_t *ws = (uint8_t *)workspace;
    PagedArgs a{};
    fill(a, c, n_split, ws, w);
    float *part = (float *)(ws + w.mass);
    const bool few = kv->mass && (int64_t)c.m_max * a.G <= kMassFewRows;
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
    const int row_parts = bf16 ? paged_mass_parts(kv->n_seqs, kv->n_kv_heads, kv->max_len, (int64_t)c.m_max * a.G) : 1;
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
    return attn_paged({cfg, tau_layer, kv, q, k, v, ld_q, ld_kv, off, m_total, m_max, scen, beh, stamp, o, ld_o, false}, workspace, ws_bytes, stream);
}

int climber_attn_sumi_paged(const climber_config *cfg, const float *tau_layer, const climber_paged_kv *kv, const void *q_c, int64_t ld_q,
                            const void *k_c, const void *v_c, int64_t ld_kv, const int32_t *cand_off, int32_t m_total, int32_t m_max,
                            const int32_t *cand_scen, const int32_t *cand_beh, void *o_c, int64_t ld_o, void *workspace, size_t ws_bytes,
                            void *stream)
{
    return attn_paged({cfg, tau_layer, kv, q_c, k_c, v_c, ld_q, ld_kv, cand_off, m_total, m_max, cand_scen, cand_beh, nullptr, o_c, ld_o, true}, workspace,
                      ws_bytes, stream);
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
    int e = check_sizes(cfg, kv, kv && kv->elem_bytes == 1 ? 1 : 0);  // (pages are not read: a cache in 8 bits is checked like the others)
    if (e) return e;
    e = check_rows(cfg, m_total, m_max);
    if (e) return e;
    if (!kv->page_table || !kv->len || !status || (appends && !off)) return CLIMBER_ERR_NULL;
    return rt(launch_check_paged(kv->page_table, kv->len, off, kv->n_seqs, kv->n_pages, page_shift(kv->page_size), kv->table_ld, kv->max_len, m_total,
                                 m_max, appends, status, (hipStream_t)stream));
}

}  // extern "C"
