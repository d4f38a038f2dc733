"""Pages forked, extended, compacted and copied on the GPU against their definitions (pages_ref.py)."""
import random

import numpy as np
import pytest
import torch

from paged8_ref import Case8, Device8, check8
from pages_ref import BAD_SEQ, POOL_FULL, DevicePool, Pool

pytestmark = pytest.mark.gpu

# pages, page size, sequences, entries of a table row
SIZES = [(1, 16, 1, 1), (7, 16, 3, 4), (64, 32, 5, 20), (65, 16, 70, 3), (1024, 64, 9, 200), (1025, 16, 300, 5), (5000, 4096, 40, 150), (20000, 16, 2000, 9),
         (140000, 16, 30, 6000)]


@pytest.mark.parametrize("size", SIZES, ids=str)
def test_any_calls_in_any_order(size):
    n_pages, page, n_seqs, table_ld = size
    r = random.Random(str(size))
    host = Pool.random(1, n_pages, page, n_seqs, table_ld, external=n_pages // 50)
    dev = DevicePool(host)
    for step in range(14):
        what = r.choice(["fork", "extend", "extend", "compact"])
        if what == "fork":
            parent = [r.choice([b, b, -1, -7, r.randrange(n_seqs), r.randrange(n_seqs)]) for b in range(n_seqs)]
            keep = [r.choice([10 ** 6, r.randint(-3, table_ld * page)]) for _ in range(n_seqs)] if r.random() < 0.5 else None
            host.fork(parent, keep)
            dev.fork(parent, keep)
            dev.check()
        elif what == "extend":
            most = r.choice([1, page, 3 * page])
            rows = [r.choice([0, -4, 1, r.randint(1, most)]) for _ in range(n_seqs)]
            # (sequences that a row of the table has no room for would refuse the whole call)
            rows = [min(x, table_ld * page - host.len[b]) for b, x in enumerate(rows)]
            copies = host.extend(rows)
            dev.extend(rows)
            dev.check(copies or [])
        else:
            copies = host.compact()
            dev.compact()
            dev.check(copies)


def test_a_fork_of_all_rows_at_once():
    # rows that take each other's place, twice over
    host = Pool.random(2, 60, 16, 6, 9)
    dev = DevicePool(host)
    for parent in ([1, 2, 3, 4, 5, 0], [5, 5, 5, 0, 1, 2], [0, 0, 0, 0, 0, 0], [-1, 0, -1, 3, 3, -1]):
        host.fork(parent)
        dev.fork(parent)
        dev.check()


@pytest.mark.parametrize("n", [1, 2, 5, 200])
def test_the_last_of_all_writers_keeps_a_shared_page(n):
    for tokens in (5, 16, 37, 48):
        for writers in (n, n - 1, n + 1):
            host = Pool(3 * n + 20, 16, n + 1, 6)
            host.len[0] = tokens
            host.held[0] = host.pages_of(tokens)
            for i in range(host.held[0]):
                host.table[0][i] = 2 * i + 1
                host.refs[2 * i + 1] = 1
            host.fork([0] * (n + 1))
            dev = DevicePool(host)
            rows = [1 if b < writers else 0 for b in range(n + 1)]
            copies = host.extend(rows)
            dev.extend(rows)
            dev.check(copies)
            if tokens % 16 and writers == n + 1:
                assert len(copies) == n


@pytest.mark.parametrize("n_seqs", [3, 300, 1500])
@pytest.mark.parametrize("writers", [1, 2, 3])
def test_many_shared_pages_are_written_at_once(n_seqs, writers):
    # three sequences hold the same 150 pages, and tokens are taken back by their lengths alone; hundreds of others may have one each
    for free, served in ((150 * writers + 2 * n_seqs, True), (100 * (writers - 1) + 40, False)):
        host = Pool(150 + n_seqs + free, 16, n_seqs, 160)
        for i in range(150):
            host.table[0][i] = 3 + i
            host.refs[3 + i] = 1
        host.held[0], host.len[0] = 150, 2400
        host.fork([0 if b < 3 else b for b in range(n_seqs)])
        for b in range(3, n_seqs):                        # (all share one page, in which each writes)
            host.table[b][0], host.held[b], host.len[b] = 153, 1, 5
        host.refs[153] = n_seqs - 3
        for b in range(3):
            host.len[b] = 20 + b
        rows = [2000 if b < writers else 0 if b < 3 else 1 for b in range(n_seqs)]
        dev = DevicePool(host)
        before = [list(x) for x in host.table]
        copies = host.extend(rows)
        assert (copies is not None) == served or not served and n_seqs == 3 and writers == 1
        if copies is None:
            assert host.table == before
        dev.extend(rows)
        dev.check(copies or [])


def test_a_call_that_cannot_be_served_changes_nothing():
    host = Pool.random(3, 40, 16, 5, 12)
    for rows in ([10 ** 4, 0, 0, 0, 1], [2 ** 31 - 1] * 5, [1, 1, 1, 12 * 16, 1]):
        dev = DevicePool(host)
        before, host.status = [list(x) for x in host.table], 0
        assert host.extend(rows) is None and host.table == before and host.status == POOL_FULL
        dev.extend(rows)
        dev.check([])
    # exactly all of the free pages, and one more
    free = 40 - host.used()
    host = Pool.random(3, 40, 16, 5, 60)
    free = 40 - host.used()
    for b in range(5):
        host.fork([i if i != b else -1 for i in range(5)])
    host.status = 0
    dev = DevicePool(host)
    rows = [40 * 16 + 1, 0, 0, 0, 0]
    assert host.extend(rows) is None
    dev.extend(rows)
    dev.check([])
    rows[0] -= 1
    host.status = 0
    dev = DevicePool(host)
    assert host.extend(rows) == [] and host.used() == 40
    dev.extend(rows)
    dev.check([])


def test_values_that_break_the_contract_stay_in_bounds():
    host = Pool.random(4, 50, 16, 6, 8)
    dev = DevicePool(host)
    dev.fork([6, 10 ** 9, 2, 3, 4, 5])
    torch.cuda.synchronize()
    assert dev.status.item() == BAD_SEQ and dev.table.tolist() == host.table
    dev.status.zero_()
    dev.table.copy_(torch.tensor([[10 ** 9, -5, 50, 2 ** 31 - 1, -2 ** 31, 49, 0, 99]] * 6))
    dev.held.copy_(torch.tensor([8, 10 ** 9, -3, 2, 0, 5]))
    dev.len.copy_(torch.tensor([2 ** 31 - 1, -2 ** 31, 40, 10 ** 6, 3, 30]))
    table = dev.table.clone()
    dev.extend([2 ** 31 - 1, 5, 1, 1, 1, -2 ** 31])
    torch.cuda.synchronize()
    assert dev.status.item() & POOL_FULL and torch.equal(dev.table, table)
    dev.status.zero_()
    dev.extend([0, 1, 0, 0, 0, 1])
    torch.cuda.synchronize()
    assert dev.status.item() == 32 and torch.equal(dev.table, table)
    dev.compact()
    dev.fork([1, 0, 5, 5, 5, 5], [2 ** 31 - 1, -2 ** 31, 7, 7, 7, 7])
    torch.cuda.synchronize()
    assert dev.status.item() & 32


def tensors(kind, n_pages, Hkv, page, d, g):
    dev = "cuda:0"
    if kind == "e4m3":
        t = {n: torch.randint(0, 255, (n_pages, Hkv, page, d), generator=g, device=dev, dtype=torch.uint8) for n in ("k", "v")}
        return t | {n: torch.randint(0, 255, (n_pages, Hkv, page // 16), generator=g, device=dev, dtype=torch.uint8) for n in ("k_scale", "v_scale")}
    return {n: torch.randn((n_pages, Hkv, page, d), generator=g, device=dev, dtype=torch.float32 if kind == "f32" else torch.bfloat16) for n in ("k", "v")}


@pytest.mark.parametrize("extras", [False, True])
@pytest.mark.parametrize("page", [16, 64, 1024])
@pytest.mark.parametrize("kind,d", [("bf16", 64), ("bf16", 128), ("f32", 4), ("f32", 100), ("e4m3", 64), ("e4m3", 128)])
def test_copy(kind, d, page, extras):
    import paper_2502_09888_amd as P
    g = torch.Generator(device="cuda:0").manual_seed(d)
    n_pages, Hkv = 40, 3
    t = tensors(kind, n_pages, Hkv, page, d, g)
    table, length = torch.zeros((1, 40), dtype=torch.int32, device="cuda:0"), torch.zeros(1, dtype=torch.int32, device="cuda:0")
    mass = torch.rand((n_pages, page), device="cuda:0") if extras and kind != "e4m3" else None
    stamp = torch.randint(0, 99, (n_pages, page), device="cuda:0", dtype=torch.int32) if extras else None
    cfg = P.Config(n_heads=Hkv, d_head=d, dtype=P.F32 if kind == "f32" else P.BF16)
    kv = P.paged_kv8(t["k"], t["v"], t["k_scale"], t["v_scale"], table, length, 10, stamp=stamp) if kind == "e4m3" else \
        P.paged_kv(t["k"], t["v"], table, length, 10, mass=mass, stamp=stamp)
    copy = P.climber_paged8_copy if kind == "e4m3" else P.climber_paged_copy
    pairs = [(3, 20, page), (3, 21, 1), (39, 0, page - 1), (5, 22, 17 % page), (6, 23, 0), (7, 24, page + 50), (40, 25, 1), (8, -1, 1), (9, 26, 16), (10, 27, page)]
    want = {n: x.clone() for n, x in (t | {"mass": mass, "stamp": stamp}).items() if x is not None}
    for a, b, n in pairs[:9]:                            # (the last one is behind the count)
        if a == 40 or b == -1:
            continue
        n = min(n, page)
        for name, x in want.items():
            if name in ("mass", "stamp"):
                x[b, :n] = x[a, :n]
            elif "scale" in name:
                x[b, :, :-(-n // 16)] = x[a, :, :-(-n // 16)]
            else:
                x[b, :, :n] = x[a, :, :n]
    copies, counts = torch.tensor(pairs, dtype=torch.int32, device="cuda:0"), torch.tensor([9, 0], dtype=torch.int32, device="cuda:0")
    copy(cfg, kv, copies, counts, 0)                     # room for none: none
    copy(cfg, kv, copies, counts, 100)
    torch.cuda.synchronize()
    for name, x in want.items():
        got = {"mass": mass, "stamp": stamp}.get(name, t.get(name))
        assert torch.equal(got.view(torch.uint8) if got.dtype != torch.int32 else got, x.view(torch.uint8) if x.dtype != torch.int32 else x), name


def test_copies_behind_4_gib():
    import paper_2502_09888_amd as P
    n_pages, Hkv, page, d = 300, 64, 1024, 128
    k = torch.zeros((n_pages, Hkv, page, d), dtype=torch.bfloat16, device="cuda:0")
    k[299] = torch.randn((Hkv, page, d), device="cuda:0").bfloat16()
    table, length = torch.zeros((1, 1), dtype=torch.int32, device="cuda:0"), torch.zeros(1, dtype=torch.int32, device="cuda:0")
    kv = P.paged_kv(k, torch.zeros_like(k), table, length, 10)
    P.climber_paged_copy(P.Config(n_heads=Hkv, d_head=d, dtype=P.BF16), kv, torch.tensor([[299, 290, page]], dtype=torch.int32, device="cuda:0"),
                         torch.tensor([1, 0], dtype=torch.int32, device="cuda:0"), 1)
    torch.cuda.synchronize()
    assert torch.equal(k[290], k[299]) and not k[:290].any() and not k[291:299].any()


@pytest.mark.parametrize("n_seqs,table_ld", [(5, 12), (40, 80)])
def test_pages_of_evicted_tokens_go_back(n_seqs, table_ld):
    """An eviction cuts the lengths; a fork of each row into itself, with keep, gives up the pages behind, and what stays is what was kept."""
    import paper_2502_09888_amd as P
    page, d, r = 16, 64, random.Random(n_seqs)
    host = Pool.random(8, n_seqs * table_ld, page, n_seqs, table_ld)
    dev = DevicePool(host)
    g = torch.Generator(device="cuda:0").manual_seed(3)
    k = torch.randn((host.n_pages, 2, page, d), generator=g, device="cuda:0").bfloat16()
    v, rank = k.neg(), torch.rand((host.n_pages, page), generator=g, device="cuda:0")
    cfg = P.Config(n_heads=2, d_head=d, n_scen=1, n_beh=1, dtype=P.BF16)
    kv = P.paged_kv(k, v, dev.table, dev.len, table_ld * page)
    ws = torch.empty(P.climber_paged_workspace_bytes(cfg, kv, 0, 0), dtype=torch.uint8, device="cuda:0")
    before, old = k.clone(), [list(x) for x in host.table]
    budget = [r.choice([0, 1, 16, 33, 10 ** 6]) for _ in range(n_seqs)]
    src = torch.empty((n_seqs, table_ld * page), dtype=torch.int32, device="cuda:0")
    P.climber_paged_evict(cfg, kv, rank, dev.ints(budget), None, dev.len, src, ws)
    host.len = [min(n, x) for n, x in zip(host.len, budget)]
    dev.check()
    rows = list(range(n_seqs))
    dev.fork(rows)                                        # (without keep a row stays as it is)
    dev.check()
    host.fork(rows, host.len)
    P.climber_pages_fork(dev.pool, dev.ints(rows), dev.len, dev.status, dev.ws)
    dev.check()
    assert host.held == [host.pages_of(n) for n in host.len] and host.used() == sum(host.held)
    src = src.tolist()
    for b in range(n_seqs):
        for slot in range(host.len[b]):
            was = src[b][slot]
            assert torch.equal(k[host.table[b][slot // page], :, slot % page], before[old[b][was // page], :, was % page]), (b, slot)
    more = [20] * n_seqs
    more = [min(x, table_ld * page - n) for x, n in zip(more, host.len)]
    copies = host.extend(more)
    dev.extend(more)
    dev.check(copies)


def test_captured_branches_and_streams():
    """Fork, extend and copy in a graph that is replayed, with eager work between, against the same calls made plainly; and on another stream."""
    import paper_2502_09888_amd as P
    g = torch.Generator(device="cuda:0").manual_seed(9)
    t = tensors("e4m3", 200, 2, 16, 64, g)
    cfg = P.Config(n_heads=2, d_head=64, dtype=P.BF16)

    def start():
        host = Pool.random(6, 200, 16, 12, 30, fill=0.3)
        dev = DevicePool(host)
        dev.t = {n: x.clone() for n, x in t.items()}
        dev.kv = P.paged_kv8(dev.t["k"], dev.t["v"], dev.t["k_scale"], dev.t["v_scale"], dev.table, dev.len, 480)
        dev.parent, dev.rows = dev.ints([b % 4 for b in range(12)]), dev.ints([0] * 4 + [3 * b % 17 for b in range(8)])
        return dev

    def step(dev, stream=None):
        P.climber_pages_fork(dev.pool, dev.parent, None, dev.status, dev.ws, stream)
        P.climber_pages_extend(dev.pool, dev.rows, dev.copies, dev.counts, dev.status, dev.ws, stream)
        P.climber_paged8_copy(cfg, dev.kv, dev.copies, dev.counts, 12, stream)
        if stream is None:
            dev.len += dev.rows
        else:
            with torch.cuda.stream(stream):
                dev.len += dev.rows
        P.climber_pages_compact(dev.pool, dev.copies, dev.counts, dev.status, dev.ws, stream)
        P.climber_paged8_copy(cfg, dev.kv, dev.copies, dev.counts, 100, stream)

    plain, captured, streamed, side = start(), start(), start(), torch.cuda.Stream()
    step(start())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(captured)
    for _ in range(4):
        graph.replay()
        step(plain)
        step(streamed, side)
        torch.cuda.synchronize()
        for other in (captured, streamed):
            for name in ("refs", "table", "held", "len", "copies", "counts", "status"):
                assert torch.equal(getattr(plain, name), getattr(other, name)), name
            assert all(torch.equal(plain.t[n], other.t[n]) for n in t)
        assert plain.status.item() == 0


def test_branches_of_histories_attend_as_whole_ones():
    """A cache in 8 bits in use: users' histories are forked, the branches take different behaviours and are scored, one branch becomes the
    history, the pool is compacted; every attention as if each sequence had pages of its own."""
    import paper_2502_09888_amd as P
    page, users, branches, d, Hkv, H = 16, 2, 3, 64, 2, 4
    B = users * (1 + branches)
    case = Case8([37, 64] + [0] * (B - users), [0] * B, H=H, Hkv=Hkv, d=d, page=page, seed=80, free=60, tail=1)
    case.table = torch.cat([case.table, torch.full((B, 8 - case.table.shape[1]), -1, dtype=torch.int32)], dim=1)
    host = Pool(case.n_pages, page, B, 8)
    for b in range(users):
        host.held[b], host.len[b] = host.pages_of(case.cached[b]), case.cached[b]
        for i in range(host.held[b]):
            host.table[b][i] = int(case.table[b, i])
            host.refs[host.table[b][i]] = 1
    dev = Device8(case, max_len=8 * page)
    pool = DevicePool(host)
    dev.table, dev.len = pool.table, pool.len
    dev.describe()

    def copies(list_of):
        P.climber_paged8_copy(dev.cfg, dev.kv, pool.copies, pool.counts, pool.copies.shape[0])
        for name in ("k", "v"):
            codes, scales = case.codes[name], case.scales[name]
            for a, b, n in list_of:
                codes[b, :, :n], scales[b, :, :-(-n // 16)] = codes[a, :, :n], scales[a, :, :-(-n // 16)]

    def step(chunk, seed, sumi):
        """`chunk` rows of each sequence, against the same sequences with what the host says they hold."""
        new = Case8(host.len, chunk, H=H, Hkv=Hkv, d=d, page=page, seed=seed, sumi=sumi)
        new.n_pages, new.table = case.n_pages, torch.tensor(host.table, dtype=torch.int32)
        new.codes, new.scales, new.stamp = case.codes, case.scales, case.stamp
        new.k, new.v = (torch.from_numpy(np.nan_to_num(case.held(n), posinf=0.0, neginf=0.0)).to(torch.bfloat16) for n in ("k", "v"))
        new.tau, new.scale = case.tau, case.scale
        other = Device8(new, max_len=8 * page)
        other.k, other.v, other.k_scale, other.v_scale, other.table, other.len = dev.k, dev.v, dev.k_scale, dev.v_scale, pool.table, pool.len
        other.describe()
        other.attend()
        check8(new, other)

    for turn in range(3):
        parent = list(range(users)) + [i % users for i in range(users * branches)]
        host.fork(parent), pool.fork(parent)
        rows = [0] * users + [5 + 7 * i for i in range(users * branches)]
        c = host.extend(rows)
        pool.extend(rows)
        pool.check(c)
        copies(c)
        step(rows, 81 + turn, False)
        host.len = [n + r for n, r in zip(host.len, rows)]
        pool.len.copy_(torch.tensor(host.len))
        step([9] * B, 91 + turn, True)
        # a branch of each user becomes the history, cut to 50 tokens; the others go
        parent = [users + 2 * users + u for u in range(users)] + [-1] * (users * branches)
        host.fork(parent, [50] * B), pool.fork(parent, [50] * B)
        c = host.compact()
        pool.compact()
        pool.check(c)
        copies(c)
        step([4] * users + [0] * (B - users), 95 + turn, True)
