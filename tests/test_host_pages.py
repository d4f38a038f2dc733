"""Refusals of the page calls (before anything would be launched, so no GPU is needed)."""
import ctypes as C

import pytest

import paper_2502_09888_amd as P
from test_host_paged import ALIGN, BUFSIZE, FAKE, NULL, OK, RANGE, SHAPE, UNSUPPORTED, cfg, kv
from test_host_paged8 import kv8


def pool(**kw):
    return P.PagePool(*{**dict(refs=FAKE, page_table=FAKE, held=FAKE, len=FAKE, n_pages=100, page_size=64, n_seqs=4, table_ld=32), **kw}.values())


def call(name, p=None, null=(), ws=FAKE, ws_bytes=0, at=None):
    lib, p = P.load_library(), p or pool()
    n = {"fork": 3, "extend": 4, "compact": 3}[name]
    a = [FAKE] * n
    for i in null:
        a[i] = None
    if at is not None:
        a[at] = FAKE + 2
    return getattr(lib, "climber_pages_" + name)(C.byref(p), *a, ws, ws_bytes, None)


@pytest.mark.parametrize("name", ["fork", "extend", "compact"])
def test_calls_refuse(name):
    assert call(name) == BUFSIZE                          # (all right but for the workspace of 0 bytes)
    assert call(name, ws_bytes=1 << 30, ws=FAKE + 16) == ALIGN and call(name, ws=None) == NULL
    for i in range({"fork": 3, "extend": 4, "compact": 3}[name]):
        if name == "fork" and i == 1:                     # keep: all tokens
            assert call(name, null=[1]) == BUFSIZE
        else:
            assert call(name, null=[i]) == NULL, i
        assert call(name, at=i, ws_bytes=1 << 30) == ALIGN, i
    for field in ("refs", "page_table", "held", "len"):
        assert call(name, pool(**{field: None})) == NULL and call(name, pool(**{field: FAKE + 1})) == ALIGN
    for field in ("n_pages", "page_size", "n_seqs", "table_ld"):
        assert call(name, pool(**{field: 0})) == SHAPE and call(name, pool(**{field: -5})) == SHAPE
    for size in (8, 24, 8192):
        assert call(name, pool(page_size=size)) == ALIGN
    for sizes in (dict(n_pages=1 << 25), dict(table_ld=1 << 24), dict(n_seqs=1 << 24, table_ld=1), dict(n_seqs=1 << 22, table_ld=1 << 9)):
        assert call(name, pool(**sizes)) == RANGE, sizes
    lib = P.load_library()
    assert getattr(lib, "climber_pages_" + name)(None, *[FAKE] * {"fork": 3, "extend": 4, "compact": 3}[name], FAKE, 0, None) == NULL


def test_workspace():
    assert P.climber_pages_workspace_bytes(pool()) > 0 and P.climber_pages_workspace_bytes(pool(n_pages=0)) == 0
    for n_pages, n_seqs, table_ld in ((1, 1, 1), (1000, 3, 7), (100000, 500, 200)):
        need = P.climber_pages_workspace_bytes(pool(n_pages=n_pages, n_seqs=n_seqs, table_ld=table_ld, page_size=16))
        assert need >= 4 * n_seqs * table_ld and need >= 12 * n_pages


def test_copy_refuses():
    lib, c = P.load_library(), cfg()

    def copy(cache, copies=FAKE, counts=FAKE, most=0, c=c):
        f = lib.climber_paged8_copy if isinstance(cache, P.PagedKV8) else lib.climber_paged_copy
        return f(C.byref(c), C.byref(cache), copies, counts, most, None)
    for cache in (kv(), kv(mass=FAKE, stamp=FAKE), kv8(), kv8(d_head=64, elem_bytes=1)):
        assert copy(cache) == OK and copy(cache, most=-1) == SHAPE
        assert copy(cache, copies=None) == NULL and copy(cache, counts=None) == NULL
        assert copy(cache, copies=FAKE + 2) == ALIGN and copy(cache, counts=FAKE + 1) == ALIGN
    for make in (kv, kv8):
        assert copy(make(k=None)) == NULL and copy(make(v=FAKE + 8)) == ALIGN and copy(make(page_size=24)) == ALIGN and copy(make(n_pages=0)) == SHAPE
    assert copy(kv8(k_scale=None)) == NULL and copy(kv8(mass=FAKE)) == UNSUPPORTED and copy(kv8(), c=cfg(dtype=P.F32)) == UNSUPPORTED
    assert copy(kv8(elem_bytes=2)) == SHAPE
    x = kv()
    x.elem_bytes = 1                                      # a cache in 8 bits that the other call would take for one of bf16
    assert copy(x) == SHAPE


def test_pools_of_other_tensors_are_none():
    torch = pytest.importorskip("torch")
    t = dict(refs=torch.zeros(10, dtype=torch.int32), page_table=torch.zeros((3, 4), dtype=torch.int32), held=torch.zeros(3, dtype=torch.int32),
             len=torch.zeros(3, dtype=torch.int32))
    p = P.page_pool(**t, page_size=16)
    assert (p.n_pages, p.page_size, p.n_seqs, p.table_ld) == (10, 16, 3, 4)
    for name, bad in (("refs", t["refs"].long()), ("page_table", t["page_table"][:, ::2]), ("held", t["held"][:2]), ("len", t["len"].float())):
        with pytest.raises(ValueError):
            P.page_pool(**{**t, name: bad}, page_size=16)
    with pytest.raises(ValueError):                       # host memory, which no kernel can reach
        P.climber_pages_fork(p, None, None, None, None)
    # tensors elsewhere than the pool
    p._device = 0
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    other = torch.zeros(100, dtype=torch.int32)
    for f, given in ((P.climber_pages_fork, (other, None, FAKE, FAKE)), (P.climber_pages_extend, (FAKE, FAKE, other, FAKE, FAKE)),
                     (P.climber_pages_compact, (FAKE, FAKE, FAKE, ws))):
        with pytest.raises(ValueError):
            f(p, *given, stream=0)
    p._device = None
    for f, rows in ((P.climber_pages_extend, (None,)), (P.climber_pages_compact, ())):
        with pytest.raises(ValueError):                   # too short
            f(p, *rows, torch.zeros((2, 3), dtype=torch.int32), None, None, None, stream=0)


def test_copies_are_read_no_further_than_they_go():
    torch = pytest.importorskip("torch")
    from paper_2502_09888_amd.climber import _room
    assert _room(torch.zeros((7, 3), dtype=torch.int32), 100) == 7 and _room(torch.zeros((7, 3), dtype=torch.int32), 5) == 5
    assert _room(FAKE, 100) == 100 and _room(None, 100) == 100
    with pytest.raises(ValueError):
        _room(torch.zeros((3, 7), dtype=torch.int32).t(), 5)


def test_other_tensors_than_the_calls_read_are_refused():
    """Too short, of another type, not one behind the other: each argument by itself, the others in order (no workspace: nothing would be launched)."""
    torch = pytest.importorskip("torch")
    p = P.page_pool(torch.zeros(10, dtype=torch.int32), torch.zeros((6, 4), dtype=torch.int32), torch.zeros(6, dtype=torch.int32),
                    torch.zeros(6, dtype=torch.int32), 16)
    p._device = None
    for f, sizes in ((P.climber_pages_fork, (6, 6, 1)), (P.climber_pages_extend, (6, 18, 2, 1)), (P.climber_pages_compact, (15, 2, 1))):
        right = [torch.zeros(n, dtype=torch.int32) for n in sizes]
        with pytest.raises(P.ClimberError):
            f(p, *right, None, stream=0)
        for i, n in enumerate(sizes):
            for bad in (torch.zeros(n - 1, dtype=torch.int32), torch.zeros(n, dtype=torch.int64), torch.zeros(4 * n, dtype=torch.uint8),
                        torch.zeros(n, dtype=torch.float32), torch.zeros((n + 1, 2), dtype=torch.int32)[:, 0]):
                with pytest.raises(ValueError):
                    f(p, *(bad if i == j else t for j, t in enumerate(right)), None, stream=0)
    for f, cache in ((P.climber_paged_copy, kv()), (P.climber_paged8_copy, kv8())):
        for copies, counts in ((torch.zeros((4, 3), dtype=torch.int64), torch.zeros(2, dtype=torch.int32)),
                               (torch.zeros((4, 3), dtype=torch.int32), torch.zeros(2, dtype=torch.int64)),
                               (torch.zeros((4, 3), dtype=torch.int32), torch.zeros(0, dtype=torch.int32))):
            with pytest.raises(ValueError):
                f(cfg(), cache, copies, counts, 4, stream=0)
