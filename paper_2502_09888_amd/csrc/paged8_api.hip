// Host side of the paged history cache in 8 bits: validation, workspace and dispatch of its entry points (include/climber.h).  Everything is
// validated before the first launch; nothing here allocates device memory.
#include "paged8.h"
#include "paged_host.h"

using namespace climber;
using namespace climber::paged_host;

namespace {

int attn_paged8(const Call &c, const climber_paged_kv8 *kv8, void *workspace, size_t ws_bytes, void *stream)
{
    const climber_config *cfg = c.cfg;
    int e = check_sizes8(cfg, kv8);
    if (e) return e;
    const climber_paged_kv *kv = c.kv;
    e = check_rows(cfg, c.m_total, c.m_max);
    if (e) return e;
    if (!kv8->k_scale || !kv8->v_scale) return CLIMBER_ERR_NULL;
    bool nothing;
    e = check_call(c, nothing);
    if (e || nothing) return e;
    const int64_t G = cfg->n_heads / kv->n_kv_heads, heads = (int64_t)kv->n_seqs * kv->n_kv_heads, tile = paged8_tile_rows(cfg->d_head, c.m_max * G, heads, kv->max_len);
    const int n_split = parts(cfg, kv, c.m_total, c.m_max, tile);
    if ((c.m_max * G + tile - 1) / tile * (heads + 7) * n_split >= kMostGroups) return CLIMBER_ERR_RANGE;
    // (new tokens are stored in a launch of their own, or with the join of the parts, a workgroup for a row and head at most)
    if (!c.sumi && (heads * paged8_store_blocks(c.m_max) + 3) / 4 + (n_split > 1 ? (int64_t)c.m_total * cfg->n_heads : 0) >= kMostGroups) return CLIMBER_ERR_RANGE;
    const Layout w = layout_of(cfg, kv, c.m_total, n_split > 1 ? (size_t)n_split * c.m_total * cfg->n_heads : 0);
    if (w.bytes > 0 && !workspace) return CLIMBER_ERR_NULL;
    if (!aligned(workspace, 256)) return CLIMBER_ERR_ALIGN;
    if (ws_bytes < w.bytes) return CLIMBER_ERR_BUFSIZE;

    Paged8Args a{};
    fill(a, c, n_split, (uint8_t *)workspace, w);
    a.row_bytes = cfg->d_head;
    a.k_scale = kv8->k_scale;
    a.v_scale = kv8->v_scale;
    return rt(launch_attn_paged8(a, (hipStream_t)stream));
}

}  // namespace

extern "C" {

size_t climber_paged8_workspace_bytes(const climber_config *cfg, const climber_paged_kv8 *kv8, int32_t m_total, int32_t m_max)
{
    if (check_sizes8(cfg, kv8) != CLIMBER_OK || check_rows(cfg, m_total, m_max) != CLIMBER_OK) return 0;
    const climber_paged_kv *kv = &kv8->kv;
    // (a smaller call may have more parts: room for as many as one can have)
    const int64_t n = most_parts(kv) * m_total * cfg->n_heads;
    return layout_of(cfg, kv, m_total, most_parts(kv) > 1 ? (size_t)std::min(n, part_rows(kv)) : 0).bytes;
}

int climber_attn_history_paged8(const climber_config *cfg, const float *tau_layer, const climber_paged_kv8 *kv8, const void *q, int64_t ld_q,
                                const void *k, const void *v, int64_t ld_kv, const int32_t *off, int32_t m_total, int32_t m_max,
                                const int32_t *scen, const int32_t *beh, const int32_t *stamp, void *o, int64_t ld_o, void *workspace,
                                size_t ws_bytes, void *stream)
{
    return attn_paged8({cfg, tau_layer, kv8 ? &kv8->kv : nullptr, q, k, v, ld_q, ld_kv, off, m_total, m_max, scen, beh, stamp, o, ld_o, false}, kv8,
                       workspace, ws_bytes, stream);
}

int climber_attn_sumi_paged8(const climber_config *cfg, const float *tau_layer, const climber_paged_kv8 *kv8, const void *q_c, int64_t ld_q,
                             const void *k_c, const void *v_c, int64_t ld_kv, const int32_t *cand_off, int32_t m_total, int32_t m_max,
                             const int32_t *cand_scen, const int32_t *cand_beh, void *o_c, int64_t ld_o, void *workspace, size_t ws_bytes,
                             void *stream)
{
    return attn_paged8({cfg, tau_layer, kv8 ? &kv8->kv : nullptr, q_c, k_c, v_c, ld_q, ld_kv, cand_off, m_total, m_max, cand_scen, cand_beh, nullptr, o_c,
                        ld_o, true}, kv8, workspace, ws_bytes, stream);
}

}  // extern "C"
