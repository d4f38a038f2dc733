"""Pools whose tables and counts do not agree, and calls at the ends of what the page kernels keep at hand, against their definitions."""
import random

import pytest

from pages_ref import BAD_PAGE, DevicePool, Pool

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
