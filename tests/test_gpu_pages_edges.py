"""Pools whose tables and counts do not agree, and calls at the ends of what the page kernels keep at hand, against their definitions."""
import random

import pytest
import torch

from pages_ref import BAD_PAGE, POOL_FULL, DevicePool, Pool

pytestmark = pytest.mark.gpu


class Checked(Pool):
    def compact(self):
        """A page that a sequence holds and that nothing is said to hold is reported, wherever it lies."""
        for b in range(self.n_seqs):
            if any(self.refs[page] == 0 for page in self.table[b][:self.held[b]]):
                self.status |= BAD_PAGE
        return super().compact()


# tables that one workgroup takes, larger ones, a pool of more pages than one workgroup looks through
@pytest.mark.parametrize("size", [(60, 16, 6, 9), (5000, 16, 300, 9), (5000, 16, 3, 1500), (70000, 16, 6, 9)], ids=str)
@pytest.mark.parametrize("side", ["none", "before", "behind", "both"])
def test_compact_reports_held_pages_without_refs(size, side):
    host, r = Checked.random(5, *size), random.Random(str(size))
    if size[0] > 60:                                      # (pages at both ends of the pool)
        host.fork([-1] + list(range(1, size[2])))
        for i, page in enumerate((0, 1, size[0] - 2, size[0] - 1)[:size[3]]):
            if host.refs[page] == 0:
                host.table[0][host.held[0]], host.refs[page] = page, 1
                host.held[0] += 1
        host.len[0] = 16 * host.held[0]
    held = [page for b in range(host.n_seqs) for page in host.table[b][:host.held[b]]]
    for before in {"none": [], "before": [True], "behind": [False], "both": [True, False]}[side]:
        # (without its refs the end of the pages in use lies one before)
        page = r.choice([p for p in held if host.refs[p] and (p < host.used() - 2) == before and abs(p - host.used()) > 3])
        host.refs[page] = 0
    dev = DevicePool(host)
    copies = host.compact()
    assert host.status == (0 if side == "none" else BAD_PAGE)
    dev.compact()
    dev.check(copies)


@pytest.mark.parametrize("n_seqs", [5, 1024, 1025])
@pytest.mark.parametrize("free", [0, 1, 2, 140, 141, 142, 300])
def test_extend_reports_all_that_it_finds(n_seqs, free):
    """A page outside the pool and too few free pages in one call: both, whatever the sizes; and nothing changes."""
    # sequences 1 and 2 share 70 pages with somebody else, that both write: 140 pages; the last one needs two more of its own
    host = Pool(70 + free, 16, n_seqs, 80)
    for b in (1, 2):
        host.table[b][:70] = range(70)
        host.held[b], host.len[b] = 70, 5
    host.refs[:70] = [3] * 70
    host.table[0][0], host.held[0], host.len[0] = 10 ** 6, 1, 3
    rows = [1, 69 * 16, 69 * 16] + [0] * (n_seqs - 4) + [20]
    dev = DevicePool(host)
    host.status = BAD_PAGE | (POOL_FULL if free < 142 else 0)
    dev.extend(rows)
    dev.check([])


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("n_seqs,most", [(60, 500), (900, 12)])
def test_extend_hands_out_more_pages_than_it_keeps_at_hand(n_seqs, most, shared):
    """One workgroup's list of free pages is 4096 long: those behind, for sequences that get many and few, and in the places of shared ones."""
    r = random.Random(n_seqs)
    host = Pool.random(6, 30000, 16, n_seqs, 600 if n_seqs < 100 else 30, fill=0.1)
    if shared:
        host.fork([b if b % 3 else (b + 1) % n_seqs for b in range(n_seqs)])
    rows = [r.choice([r.randint(1, 16), r.randint(1, 64), 16 * most, r.randint(0, 16 * most)]) for b in range(n_seqs)]
    rows[-1] = 16 * most
    rows = [min(x, host.table_ld * 16 - n) for x, n in zip(rows, host.len)]
    dev, held, used, before = DevicePool(host), list(host.held), host.used(), [list(x) for x in host.table]
    copies = host.extend(rows)
    # pages that each sequence got, in order: more than 4096, and one sequence has pages on both sides of the border
    got = [sum(x != y for x, y in zip(now[:h], was[:h])) for now, was, h in zip(host.table, before, host.held)]
    at = [sum(got[:b]) for b in range(n_seqs)]
    assert copies is not None and sum(got) > 4200 and any(a < 4096 < a + g for a, g in zip(at, got))
    assert any(a > 4096 and 0 < g <= 4 for a, g in zip(at, got)) and any(a > 4096 and g > 4 for a, g in zip(at, got))
    if shared:
        assert copies and any(host.table[b][:held[b]] != before[b][:held[b]] and at[b] > 4096 for b in range(n_seqs))
    assert host.used() == used + sum(got)
    dev.extend(rows)
    dev.check(copies)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_a_pool_of_one_page(kind):
    """Copies of exactly [n_pages / 2][3] integers, which are none."""
    import paper_2502_09888_amd as P
    host = Pool(1, 16, 2, 3)
    dev = DevicePool(host)
    dev.copies = torch.empty((2, 3), dtype=torch.int32, device="cuda:0")
    none = torch.empty((0, 3), dtype=torch.int32, device="cuda:0")
    k = torch.ones((1, 2, 16, 64), device="cuda:0").to(torch.bfloat16 if kind == "bf16" else torch.float8_e4m3fn)
    s = torch.full((1, 2, 1), 127, dtype=torch.uint8, device="cuda:0")
    kv = P.paged_kv(k, k.clone(), dev.table, dev.len, 48) if kind == "bf16" else P.paged_kv8(k, k.clone(), s, s.clone(), dev.table, dev.len, 48)
    cfg, copy = P.Config(n_heads=2, d_head=64, dtype=P.BF16), P.climber_paged_copy if kind == "bf16" else P.climber_paged8_copy
    for rows in ([16, 0], [-1, -1], [0, 3]):
        if rows[0] < 0:
            host.fork([-1, -1])
            dev.fork([-1, -1])
        else:
            host.extend(rows)
            dev.extend(rows)
        assert host.compact() == []
        P.climber_pages_compact(dev.pool, none, dev.counts, dev.status, dev.ws)
        copy(cfg, kv, none, dev.counts, 10)
        dev.check()
        assert dev.counts.tolist() == [0, host.used()] and bool((k.float() == 1).all())


@pytest.mark.parametrize("n_seqs,table_ld", [(6, 9), (300, 9), (3, 1500)])
@pytest.mark.parametrize("keep", [False, True])
def test_fork_reports_pages_outside_the_pool_that_a_row_gives_up(n_seqs, table_ld, keep):
    for page in (-1, 5000, 10 ** 9, -2 ** 31):
        for row, parent, reported in ((1, -1, True), (1, 2, True), (1, 1, keep), (2, 2, keep), (0, 0, False)):
            host = Pool.random(7, 5000, 16, n_seqs, table_ld, fill=0.5)
            for b in (1, 2):                              # rows of two pages at least
                host.fork([x if x != b else -1 for x in range(n_seqs)])
                assert host.extend([40 if x == b else 0 for x in range(n_seqs)]) == []
                host.len[b] = 40
            dev, last = DevicePool(host), host.held[row] - 1
            if row:
                dev.table[row, last] = page
                host.refs[host.table[row][last]] -= 1     # (nobody holds it any more)
                dev.refs.copy_(dev.ints(host.refs))
                host.table[row][last], host.held[row] = -1, last
            parents = [parent if b == row else b for b in range(n_seqs)]
            keeps = [20 if b == row else 10 ** 6 for b in range(n_seqs)] if keep else None
            dev.fork(parents, keeps)
            torch.cuda.synchronize()
            assert dev.status.item() == (BAD_PAGE if reported else 0), (page, row, parent)
            if reported:
                host.fork(parents, keeps)
                host.status = BAD_PAGE
                dev.check()
