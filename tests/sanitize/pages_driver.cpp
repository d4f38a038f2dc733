// The host sides of the paged cache in 8 bits and of the page calls on random sizes, their launches replaced by ones that check what they are given:
// every array that a launch works in lies in the workspace, apart from the others, and a workspace for a call covers every smaller one.
// (Built with the sanitizers; no GPU.)
#include <stdio.h>
#include <stdlib.h>

#include <algorithm>
#include <vector>

#include "../../include/climber.h"
#include "../../paper_2502_09888_amd/csrc/internal.h"
#include "../../paper_2502_09888_amd/csrc/paged8.h"
#include "../../paper_2502_09888_amd/csrc/pages.h"

namespace {

uint8_t *ws;
size_t ws_bytes;
int bad = 0, launches = 0;

struct Part {
    const char *name;
    const uint8_t *at;
    int64_t bytes;
};
void in_workspace(std::vector<Part> parts)
{
    std::sort(parts.begin(), parts.end(), [](const Part &a, const Part &b) { return a.at < b.at; });
    const uint8_t *end = ws;
    for (const Part &p : parts) {
        if (p.at < end || p.at + p.bytes > ws + ws_bytes || (uintptr_t)p.at % 8)
            if (bad++ < 20) printf("%s: %lld bytes at %lld of %lld\n", p.name, (long long)p.bytes, (long long)(p.at - ws), (long long)ws_bytes);
        end = std::max(end, p.at + p.bytes);
    }
}
void threads(const char *name, int64_t groups, int64_t each)
{
    if (groups < 1 || groups * each >= (int64_t)1 << 32)
        if (bad++ < 20) printf("%s: %lld workgroups of %lld\n", name, (long long)groups, (long long)each);
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
template <typename T>
const uint8_t *u8(T *p) { return (const uint8_t *)p; }

}  // namespace

namespace climber {

int check_config_values(const climber_config *c) { return c->d_model == c->n_heads * c->d_head && c->n_heads > 0 ? CLIMBER_OK : CLIMBER_ERR_SHAPE; }

hipError_t launch_attn_paged8(const Paged8Args &a, hipStream_t)
{
    ++launches;
    const int64_t out = (int64_t)a.m_total * a.H, rows = (int64_t)a.m_max * a.G, bh = (int64_t)a.n_seqs * a.Hkv;
    if (a.n_split > 1) in_workspace({{"part_o", u8(a.part_o), a.n_split * out * a.d * 4}, {"part_ml", u8(a.part_ml), a.n_split * out * 8}});
    if (!a.k_scale || !a.v_scale || a.row_bytes != a.d || a.mass) ++bad;
    const int tile = paged8_tile_rows(a.d, rows, bh, a.max_len);
    threads("attention", (bh + 7) * ((rows + tile - 1) / tile) * a.n_split, 256);
    const int64_t after = (a.sumi ? 0 : (bh * paged8_store_blocks(a.m_max) + 3) / 4) + (a.n_split > 1 ? out : 0);
    if (after > 0) threads("new tokens and join", after, 256);
    return hipSuccess;
}
hipError_t launch_pages_fork(const ForkArgs &a, hipStream_t)
{
    ++launches;
    in_workspace({{"rows", u8(a.rows), (int64_t)a.n_seqs * a.table_ld * 4}, {"new_len", u8(a.new_len), a.n_seqs * 4ll}, {"new_held", u8(a.new_held), a.n_seqs * 4ll},
                  {"entries", u8(a.entries), a.n_seqs * 4ll}});
    threads("fork", (a.n_seqs + 3) / 4, 256);
    return hipSuccess;
}
hipError_t launch_pages_extend(const ExtendArgs &a, hipStream_t)
{
    ++launches;
    const int64_t units = pool_units(a.n_pages), n = a.n_pages;
    in_workspace({{"bits", u8(a.bits), units * 128}, {"unit_free", u8(a.unit_free), units * 4}, {"unit_used", u8(a.unit_used), units * 4},
                  {"writers", u8(a.writers), n * 4}, {"last", u8(a.last), n * 4}, {"free_list", u8(a.free_list), n * 4},
                  {"first_new", u8(a.first_new), a.n_seqs * 4ll}, {"first_copy", u8(a.first_copy), a.n_seqs * 4ll}, {"go", u8(a.go), 4}});
    threads("extend", (units + 3) / 4 + (a.n_seqs + 3) / 4, 256);
    return hipSuccess;
}
hipError_t launch_pages_compact(const CompactArgs &a, hipStream_t)
{
    ++launches;
    const int64_t units = pool_units(a.n_pages), n = a.n_pages;
    in_workspace({{"bits", u8(a.bits), units * 128}, {"unit_used", u8(a.unit_used), units * 4}, {"movers", u8(a.movers), (n / 2 + 1) * 4},
                  {"holes", u8(a.holes), (n / 2 + 1) * 4}, {"to", u8(a.to), n * 4}});
    threads("compact", (units + 3) / 4 + 1024 + (a.n_seqs + 3) / 4, 256);
    return hipSuccess;
}
hipError_t launch_pages_copy(const CopyArgs &a, hipStream_t)
{
    ++launches;
    if (a.max_copies < 1 || a.row_bytes % 16 || !a.k_scale != !a.v_scale) ++bad;
    return hipSuccess;
}

}  // namespace climber

int main()
{
    uint8_t *const far = (uint8_t *)0x7f0000000000, *const o = (uint8_t *)0x7e0000000000;  // never dereferenced
    ws = (uint8_t *)0x600000000000;
    int refused = 0, done = 0;
    for (int i = 0; i < 30000; ++i) {
        climber_config c{};
        c.dtype = CLIMBER_BF16;
        c.d_head = (int32_t)(64 << draw(0, 1));
        climber_paged_kv8 kv8{};
        climber_paged_kv &kv = kv8.kv;
        kv8.k_scale = kv8.v_scale = far;
        kv.n_kv_heads = (int32_t)draw(1, 16);
        c.n_heads = kv.n_kv_heads * (int32_t)draw(1, 9);
        c.d_model = c.n_heads * c.d_head;
        c.n_scen = c.n_beh = 1;
        c.qk_scale = 1.f;
        kv.k = kv.v = far;
        kv.page_table = kv.len = (const int32_t *)far;
        kv.page_size = 16 << draw(0, 8);
        kv.n_pages = 1000;
        kv.n_seqs = (int32_t)skewed(i % 7 ? 300 : 1 << 23);
        kv.max_len = (int32_t)skewed(i % 5 ? 20000 : 1 << 28);
        kv.table_ld = (kv.max_len + kv.page_size - 1) / kv.page_size;
        const int32_t most_total = (int32_t)skewed(i % 3 ? 5000 : 1 << 24), most_max = (int32_t)draw(1, most_total);
        const size_t room = climber_paged8_workspace_bytes(&c, &kv8, most_total, most_max);
        ws_bytes = room;
        for (int j = 0; j < (room ? 6 : 1); ++j) {  // (0: none is needed, or these sizes are refused)
            // the call itself, then smaller ones
            const int32_t total = j == 0 ? most_total : (int32_t)draw(1, most_total), max = j == 0 ? most_max : (int32_t)draw(1, std::min(total, most_max));
            for (bool sumi : {false, true}) {
                const int e = sumi ? climber_attn_sumi_paged8(&c, (const float *)far, &kv8, far, c.d_model, far, far, kv.n_kv_heads * c.d_head, (const int32_t *)far,
                                                              total, max, (const int32_t *)far, (const int32_t *)far, o, c.d_model, ws, room, nullptr)
                                   : climber_attn_history_paged8(&c, (const float *)far, &kv8, far, c.d_model, far, far, kv.n_kv_heads * c.d_head,
                                                                 (const int32_t *)far, total, max, (const int32_t *)far, (const int32_t *)far, nullptr, o,
                                                                 c.d_model, ws, room, nullptr);
                if (e != CLIMBER_OK && e != CLIMBER_ERR_RANGE && bad++ < 20) printf("attention: %d\n", e);
                done += e == CLIMBER_OK;
                refused += e != CLIMBER_OK;
            }
        }
        if (climber_paged8_copy(&c, &kv8, (const int32_t *)far, (const int32_t *)far, (int32_t)skewed(1 << 30), nullptr) == CLIMBER_OK) ++done;
        climber_page_pool pool{(int32_t *)far, (int32_t *)far, (int32_t *)far, (int32_t *)far, (int32_t)skewed(i % 5 ? 30000 : 1 << 27), 16 << (int)draw(0, 8),
                               (int32_t)skewed(i % 7 ? 3000 : 1 << 24), (int32_t)skewed(i % 3 ? 500 : 1 << 24)};
        const size_t pages_room = climber_pages_workspace_bytes(&pool);
        if (pages_room == 0) {
            ++refused;
            continue;
        }
        ws_bytes = pages_room;
        int32_t *const p = (int32_t *)far;
        const int e[3] = {climber_pages_fork(&pool, p, p, p, ws, pages_room, nullptr), climber_pages_extend(&pool, p, p, p, p, ws, pages_room, nullptr),
                          climber_pages_compact(&pool, p, p, p, ws, pages_room, nullptr)};
        for (int j = 0; j < 3; ++j)
            if (e[j] != CLIMBER_OK && bad++ < 20) printf("pages %d: %d\n", j, e[j]);
        done += 3;
    }
    printf("bad=%d launches=%d done=%d refused=%d\n", bad, launches, done, refused);
    return bad != 0 || launches < 100000;
}
