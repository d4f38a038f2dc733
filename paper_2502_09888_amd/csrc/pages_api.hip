// Host side of the page calls: validation, workspace layout and dispatch (include/climber.h).  Everything is validated before the first launch;
// nothing here allocates device memory.
#include "pages.h"
#include "paged_host.h"

using namespace climber;
using namespace climber::paged_host;

namespace {

int check_pool(const climber_page_pool *pool)
{
    if (!pool) return CLIMBER_ERR_NULL;
    if (pool->n_pages < 1 || pool->n_seqs < 1 || pool->table_ld < 1 || pool->page_size < 1) return CLIMBER_ERR_SHAPE;
    if (pool->page_size < 16 || pool->page_size > 4096 || (pool->page_size & (pool->page_size - 1)) != 0) return CLIMBER_ERR_ALIGN;
    // slots of a table row, tokens of the pool and entries of the table are counted in 32 bits
    if ((int64_t)pool->table_ld * pool->page_size >= (int64_t)1 << 30 || (int64_t)pool->n_pages * pool->page_size >= (int64_t)1 << 31 ||
        (int64_t)pool->n_seqs * pool->table_ld >= (int64_t)1 << 31 || pool->n_seqs >= 1 << 24)
        return CLIMBER_ERR_RANGE;
    return CLIMBER_OK;
}

struct PoolLayout {  // of the workspace, for any of the calls
    size_t a, b, c, d, e, f, bytes;
};
PoolLayout fork_layout(const climber_page_pool *p)
{
    PoolLayout w{};
    w.b = up((size_t)p->n_seqs * p->table_ld * 4);
    w.c = w.b + up((size_t)p->n_seqs * 4);
    w.d = w.c + up((size_t)p->n_seqs * 4);
    w.bytes = w.d + up((size_t)p->n_seqs * 4);
    return w;
}
PoolLayout extend_layout(const climber_page_pool *p)
{
    PoolLayout w{};
    const size_t units = pool_units(p->n_pages), pages = up((size_t)p->n_pages * 4);
    w.b = up(units * 128);                      // behind the bits: two counts of each unit
    w.c = w.b + 2 * up(units * 4);              // writers, last, free_list
    w.d = w.c + 3 * pages;                      // first_new, first_copy
    w.e = w.d + 2 * up((size_t)p->n_seqs * 4);  // go
    w.bytes = w.e + 256;
    return w;
}
PoolLayout compact_layout(const climber_page_pool *p)
{
    PoolLayout w{};
    const size_t units = pool_units(p->n_pages);
    w.b = up(units * 128);
    w.c = w.b + up(units * 4);                            // movers
    w.d = w.c + up(((size_t)p->n_pages / 2 + 1) * 4);     // holes
    w.e = w.d + up(((size_t)p->n_pages / 2 + 1) * 4);     // to
    w.bytes = w.e + up((size_t)p->n_pages * 4);
    return w;
}

// what the calls on a pool have in common; `need`: bytes of workspace
int check(const climber_page_pool *pool, const void *x, const void *y, const void *status, const void *workspace, size_t ws_bytes, size_t need)
{
    if (!pool->refs || !pool->page_table || !pool->held || !pool->len || !x || !y || !status || !workspace) return CLIMBER_ERR_NULL;
    if (!aligned(pool->refs, 4) || !aligned(pool->page_table, 4) || !aligned(pool->held, 4) || !aligned(pool->len, 4) || !aligned(x, 4) || !aligned(y, 4) ||
        !aligned(status, 4) || !aligned(workspace, 256))
        return CLIMBER_ERR_ALIGN;
    return ws_bytes < need ? CLIMBER_ERR_BUFSIZE : CLIMBER_OK;
}
void fill(PoolArgs &a, const climber_page_pool *pool, int32_t *status)
{
    a.refs = pool->refs;
    a.table = pool->page_table;
    a.held = pool->held;
    a.len = pool->len;
    a.n_pages = pool->n_pages;
    a.page_shift = page_shift(pool->page_size);
    a.n_seqs = pool->n_seqs;
    a.table_ld = pool->table_ld;
    a.status = status;
}

int copy(const climber_paged_kv *kv, uint8_t *k_scale, uint8_t *v_scale, int row_bytes, const int32_t *copies, const int32_t *counts, int32_t max_copies,
         void *stream)
{
    if (max_copies < 0) return CLIMBER_ERR_SHAPE;
    if (!kv->k || !kv->v || !copies || !counts) return CLIMBER_ERR_NULL;
    if (!aligned(kv->k, 16) || !aligned(kv->v, 16) || !aligned(kv->mass, 4) || !aligned(kv->stamp, 4) || !aligned(copies, 4) || !aligned(counts, 4))
        return CLIMBER_ERR_ALIGN;
    if (max_copies == 0) return CLIMBER_OK;
    CopyArgs a{};
    a.k = (uint8_t *)kv->k;
    a.v = (uint8_t *)kv->v;
    a.k_scale = k_scale;
    a.v_scale = v_scale;
    a.mass = (int32_t *)kv->mass;
    a.stamp = kv->stamp;
    a.copies = copies;
    a.counts = counts;
    a.n_pages = kv->n_pages;
    a.page_shift = page_shift(kv->page_size);
    a.Hkv = kv->n_kv_heads;
    a.row_bytes = row_bytes;
    a.max_copies = max_copies;
    return rt(launch_pages_copy(a, (hipStream_t)stream));
}

}  // namespace

extern "C" {

size_t climber_pages_workspace_bytes(const climber_page_pool *pool)
{
    if (check_pool(pool) != CLIMBER_OK) return 0;
    return std::max(fork_layout(pool).bytes, std::max(extend_layout(pool).bytes, compact_layout(pool).bytes));
}

int climber_pages_fork(const climber_page_pool *pool, const int32_t *parent, const int32_t *keep, int32_t *status, void *workspace, size_t ws_bytes,
                       void *stream)
{
    int e = check_pool(pool);
    if (e) return e;
    const PoolLayout w = fork_layout(pool);
    e = check(pool, parent, parent, status, workspace, ws_bytes, w.bytes);
    if (e) return e;
    if (!aligned(keep, 4)) return CLIMBER_ERR_ALIGN;
    uint8_t *ws = (uint8_t *)workspace;
    ForkArgs a{};
    fill(a, pool, status);
    a.parent = parent;
    a.keep = keep;
    a.rows = (int32_t *)ws;
    a.new_len = (int32_t *)(ws + w.b);
    a.new_held = (int32_t *)(ws + w.c);
    a.entries = (int32_t *)(ws + w.d);
    return rt(launch_pages_fork(a, (hipStream_t)stream));
}

int climber_pages_extend(const climber_page_pool *pool, const int32_t *rows, int32_t *copies, int32_t *counts, int32_t *status, void *workspace,
                         size_t ws_bytes, void *stream)
{
    int e = check_pool(pool);
    if (e) return e;
    const PoolLayout w = extend_layout(pool);
    if (!rows) return CLIMBER_ERR_NULL;
    if (!aligned(rows, 4)) return CLIMBER_ERR_ALIGN;
    e = check(pool, copies, counts, status, workspace, ws_bytes, w.bytes);
    if (e) return e;
    uint8_t *ws = (uint8_t *)workspace;
    const size_t pages = up((size_t)pool->n_pages * 4);
    ExtendArgs a{};
    fill(a, pool, status);
    a.rows = rows;
    a.copies = copies;
    a.counts = counts;
    a.bits = (uint64_t *)ws;
    a.unit_free = (int32_t *)(ws + w.b);
    a.unit_used = (int32_t *)(ws + w.b + (w.c - w.b) / 2);
    a.writers = (int32_t *)(ws + w.c);
    a.last = (int32_t *)(ws + w.c + pages);
    a.free_list = (int32_t *)(ws + w.c + 2 * pages);
    a.first_new = (int32_t *)(ws + w.d);
    a.first_copy = (int32_t *)(ws + w.d + (w.e - w.d) / 2);
    a.go = (int32_t *)(ws + w.e);
    return rt(launch_pages_extend(a, (hipStream_t)stream));
}

int climber_pages_compact(const climber_page_pool *pool, int32_t *copies, int32_t *counts, int32_t *status, void *workspace, size_t ws_bytes,
                          void *stream)
{
    int e = check_pool(pool);
    if (e) return e;
    const PoolLayout w = compact_layout(pool);
    e = check(pool, pool->n_pages < 2 && !copies ? counts : copies, counts, status, workspace, ws_bytes, w.bytes);  // (of one page there are no copies)
    if (e) return e;
    uint8_t *ws = (uint8_t *)workspace;
    CompactArgs a{};
    fill(a, pool, status);
    a.copies = copies;
    a.counts = counts;
    a.bits = (uint64_t *)ws;
    a.unit_used = (int32_t *)(ws + w.b);
    a.movers = (int32_t *)(ws + w.c);
    a.holes = (int32_t *)(ws + w.d);
    a.to = (int32_t *)(ws + w.e);
    return rt(launch_pages_compact(a, (hipStream_t)stream));
}

int climber_paged_copy(const climber_config *cfg, const climber_paged_kv *kv, const int32_t *copies, const int32_t *counts, int32_t max_copies,
                       void *stream)
{
    const int e = check_sizes(cfg, kv);
    return e ? e : copy(kv, nullptr, nullptr, (int)(cfg->d_head * elem_of(cfg)), copies, counts, max_copies, stream);
}

int climber_paged8_copy(const climber_config *cfg, const climber_paged_kv8 *kv8, const int32_t *copies, const int32_t *counts, int32_t max_copies,
                        void *stream)
{
    const int e = check_sizes8(cfg, kv8);
    if (e) return e;
    if (!kv8->k_scale || !kv8->v_scale) return CLIMBER_ERR_NULL;
    return copy(&kv8->kv, kv8->k_scale, kv8->v_scale, cfg->d_head, copies, counts, max_copies, stream);
}

}  // extern "C"
