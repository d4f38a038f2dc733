// The host side of the paged cache on random sizes, its launches replaced by ones that check what they are given: every array that a launch
// works in lies in the workspace, and a workspace for a call covers every smaller one.  (Built with the sanitizers; no GPU.)
#include <stdio.h>
#include <stdlib.h>

#include <algorithm>
#include <initializer_list>

#include "../../include/climber.h"
#include "../../paper_2502_09888_amd/csrc/internal.h"
#include "../../paper_2502_09888_amd/csrc/paged.h"

namespace {

uint8_t *ws;
size_t ws_bytes;
int bad = 0, launches = 0;
int64_t m_total, n_max;

void in_workspace(const char *name, const void *p, int64_t bytes)
{
    if (bytes == 0) return;
    const uint8_t *a = (const uint8_t *)p;
    if (a < ws || a + bytes > ws + ws_bytes) {
        if (bad++ < 20) printf("%s: %lld bytes at %lld of %lld\n", name, (long long)bytes, (long long)(a - ws), (long long)ws_bytes);
    }
}
void threads(const char *name, int64_t groups, int64_t each)
{
    if (groups < 1 || groups * each >= (int64_t)1 << 32) {
        if (bad++ < 20) printf("%s: %lld workgroups of %lld\n", name, (long long)groups, (long long)each);
    }
}

uint64_t state = 88172645463325252ull;
int64_t draw(int64_t lo, int64_t hi)
{
    state ^= state << 13, state ^= state >> 7, state ^= state << 17;
    return lo + (int64_t)(state % (uint64_t)(hi - lo + 1));
}
int64_t skewed(int64_t hi)  // mostly small
{
    return draw(1, std::max<int64_t>(1, hi >> draw(0, 12)));
}

}  // namespace

namespace climber {

int check_config_values(const climber_config *c) { return c->d_model == c->n_heads * c->d_head && c->n_heads > 0 ? CLIMBER_OK : CLIMBER_ERR_SHAPE; }

static hipError_t attention(const PagedArgs &a, bool bf16)
{
    ++launches;
    const int64_t out = (int64_t)a.m_total * a.H;
    if (a.n_split > 1) {
        in_workspace("part_o", a.part_o, a.n_split * out * a.d * 4);
        in_workspace("part_ml", a.part_ml, a.n_split * out * 8);
    }
    if (a.mass) in_workspace("lse", a.lse, out * 8);
    if (a.logits) in_workspace("logits", a.logits, (int64_t)a.n_seqs * a.Hkv * a.m_max * a.G * a.logits_ld * 4);
    if (a.logits && (a.logits_ld < a.max_len || a.logits_ld % 32)) ++bad;
    PagedArgs p = a;
    const int64_t rows = (int64_t)a.m_max * a.G;
    const int tile = paged_tile_rows(bf16, a.d, rows, (int64_t)a.n_seqs * a.Hkv);
    p.n_tiles = (int)((rows + tile - 1) / tile);
    threads("attention", ((int64_t)a.n_seqs * a.Hkv + 7) * p.n_tiles * a.n_split, 256);
    const int64_t bh = (int64_t)a.n_seqs * a.Hkv;
    const int64_t groups = paged_grid(p);
    if (groups < bh * p.n_tiles * a.n_split || (p.bh_major && groups % 8)) ++bad;
    return hipSuccess;
}
hipError_t launch_attn_paged_bf16(const PagedArgs &a, hipStream_t) { return attention(a, true); }
hipError_t launch_attn_paged_f32(const PagedArgs &a, hipStream_t) { return attention(a, false); }
hipError_t launch_paged_combine(const PagedArgs &a, bool, hipStream_t)
{
    if (a.n_split < 2) ++bad;
    threads("join", ((int64_t)a.m_total * a.H * (a.n_split <= 4 ? 1 : 8) + 7) / 8, 256);
    return hipSuccess;
}
hipError_t launch_paged_mass_f32(const PagedArgs &a, float *part, hipStream_t)
{
    in_workspace("part (fp32)", part, (int64_t)a.n_seqs * a.Hkv * a.max_len * 4);
    threads("weights (fp32)", (int64_t)a.n_seqs * a.Hkv * ((a.max_len + 31) / 32), 256);
    return hipSuccess;
}
hipError_t launch_paged_mass_bf16(const PagedArgs &a, float *part, int row_parts, hipStream_t)
{
    in_workspace("part (bf16)", part, (int64_t)a.n_seqs * a.Hkv * row_parts * a.max_len * 4);
    threads("weights (bf16)", ((int64_t)a.n_seqs * a.Hkv + 7) / 8 * 8 * row_parts * ((a.max_len + kMassKeys - 1) / kMassKeys), 256);
    return hipSuccess;
}
hipError_t launch_paged_mass_few(const PagedArgs &a, hipStream_t)
{
    if (!a.logits || (int64_t)a.m_max * a.G > kMassFewRows) ++bad;
    threads("weights of few", (int64_t)(a.max_len + 255) / 256 * a.n_seqs, 256);
    return hipSuccess;
}
hipError_t launch_paged_mass_add(const PagedArgs &a, const float *part, int n_parts, hipStream_t)
{
    in_workspace("parts", part, (int64_t)a.n_seqs * n_parts * a.max_len * 4);
    threads("sum of weights", (int64_t)(a.max_len + 255) / 256 * a.n_seqs, 256);
    return hipSuccess;
}
hipError_t launch_paged_evict(const EvictArgs &a, hipStream_t)
{
    ++launches;
    const int64_t B = a.n_seqs, L = a.max_len, S = a.segments;
    in_workspace("holes", a.holes, B * (L / 2 + 1) * 4);
    in_workspace("movers", a.movers, B * (L / 2 + 1) * 4);
    in_workspace("n_moves", a.n_moves, B * 4);
    if (S > 0) {
        in_workspace("keys", a.keys, B * L * 4);
        in_workspace("first", a.first, B * S * (kEvictSegment / 64) * 8);
        in_workspace("hists", a.hists, B * S * kEvictSegInts * 4);
        in_workspace("state", a.state, B * 32);
        threads("eviction", B * S, 1024);
        if (S < (L + kEvictSegment - 1) / kEvictSegment + 1) ++bad;
    } else {
        threads("eviction", B, 1024);
    }
    return hipSuccess;
}
hipError_t launch_check_paged(const int32_t *, const int32_t *, const int32_t *, int n_seqs, int, int, int, int, int, int, int, int32_t *, hipStream_t)
{
    threads("check", n_seqs, 256);
    return hipSuccess;
}

}  // namespace climber

int main()
{
    uint8_t *const far = (uint8_t *)0x7f0000000000, *const o = (uint8_t *)0x7e0000000000;  // never dereferenced
    ws = (uint8_t *)0x600000000000;
    int refused = 0, done = 0;
    for (int i = 0; i < 60000; ++i) {
        climber_config c{};
        const bool bf16 = draw(0, 1);
        c.dtype = bf16 ? CLIMBER_BF16 : CLIMBER_F32;
        c.d_head = (int32_t)(bf16 ? 64 << draw(0, 1) : 4 * draw(1, 32));
        climber_paged_kv kv{};
        kv.n_kv_heads = (int32_t)draw(1, 16);
        c.n_heads = kv.n_kv_heads * (int32_t)draw(1, 9);
        c.d_model = c.n_heads * c.d_head;
        c.n_scen = c.n_beh = 1;
        c.qk_scale = 1.f;
        kv.k = kv.v = far;
        kv.mass = draw(0, 1) ? (float *)far : nullptr;
        kv.page_table = kv.len = (const int32_t *)far;
        kv.page_size = 16 << draw(0, 8);
        kv.n_pages = 1000;
        kv.n_seqs = (int32_t)skewed(i % 7 ? 300 : 1 << 23);
        kv.max_len = (int32_t)skewed(i % 5 ? 20000 : 1 << 28);
        kv.table_ld = (kv.max_len + kv.page_size - 1) / kv.page_size;
        const int32_t most_total = (int32_t)skewed(i % 3 ? 5000 : 1 << 24), most_max = (int32_t)draw(1, most_total);
        const size_t room = climber_paged_workspace_bytes(&c, &kv, most_total, most_max);
        if (room == 0) {
            ++refused;
            continue;
        }
        ws_bytes = room;
        for (int j = 0; j < 6; ++j) {
            // the call itself, then smaller ones
            const int32_t total = j == 0 ? most_total : (int32_t)draw(1, most_total), max = j == 0 ? most_max : (int32_t)draw(1, std::min(total, most_max));
            for (bool sumi : {false, true}) {
                const int e = sumi ? climber_attn_sumi_paged(&c, (const float *)far, &kv, far, c.d_model, far, far, kv.n_kv_heads * c.d_head, (const int32_t *)far,
                                                             total, max, (const int32_t *)far, (const int32_t *)far, o, c.d_model, ws, room, nullptr)
                                   : climber_attn_history_paged(&c, (const float *)far, &kv, far, c.d_model, far, far, kv.n_kv_heads * c.d_head,
                                                                (const int32_t *)far, total, max, (const int32_t *)far, (const int32_t *)far, nullptr, o,
                                                                c.d_model, ws, room, nullptr);
                if (e != CLIMBER_OK && e != CLIMBER_ERR_RANGE && bad++ < 20) printf("attention: %d\n", e);
                done += e == CLIMBER_OK;
            }
        }
        const int e = climber_paged_evict(&c, &kv, (const float *)far, (const int32_t *)far, nullptr, (int32_t *)far, nullptr, ws, room, nullptr);
        if (e != CLIMBER_OK && e != CLIMBER_ERR_UNSUPPORTED && bad++ < 20) printf("eviction: %d\n", e);
        // to the byte: an eviction's own workspace
        const size_t own = climber_paged_workspace_bytes(&c, &kv, 0, 0);
        if (e == CLIMBER_OK && climber_paged_evict(&c, &kv, (const float *)far, (const int32_t *)far, nullptr, (int32_t *)far, nullptr, ws, own, nullptr) != CLIMBER_OK) ++bad;
    }
    printf("bad=%d launches=%d done=%d refused=%d\n", bad, launches, done, refused);
    return bad != 0;
}
