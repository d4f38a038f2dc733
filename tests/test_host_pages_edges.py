"""Page calls at their smallest sizes, without a GPU: what comes back before anything would be launched."""
import ctypes as C

import pytest

import paper_2502_09888_amd as P
from test_host_paged import BUFSIZE, NULL, cfg, kv
from test_host_paged8 import kv8
from test_host_pages import call, pool


def test_a_pool_of_one_page_has_no_copies():
    # [n_pages / 2][3] integers: none, and an empty tensor has no address
    assert call("compact", pool(n_pages=1), null=[0]) == BUFSIZE and call("compact", pool(n_pages=1)) == BUFSIZE
    for n_pages in (2, 3):
        assert call("compact", pool(n_pages=n_pages), null=[0]) == NULL
    for i in (1, 2):                                      # counts and status are written all the same
        assert call("compact", pool(n_pages=1), null=[i]) == NULL


def test_copies_of_none():
    torch = pytest.importorskip("torch")
    p = P.page_pool(torch.zeros(1, dtype=torch.int32), torch.zeros((2, 4), dtype=torch.int32), torch.zeros(2, dtype=torch.int32),
                    torch.zeros(2, dtype=torch.int32), 16)
    p._device = None
    none, counts = torch.zeros((0, 3), dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    ws = torch.zeros(512, dtype=torch.uint8)
    ws = ws[-ws.data_ptr() % 256:][:16]                   # (aligned, and too small)
    with pytest.raises(P.ClimberError) as e:
        P.climber_pages_compact(p, none, counts, torch.zeros(1, dtype=torch.int32), ws, stream=0)
    assert e.value.code == BUFSIZE
    for f, cache in ((P.climber_paged_copy, kv()), (P.climber_paged8_copy, kv8())):
        f(cfg(), cache, none, counts, 10, stream=0)
        with pytest.raises(ValueError):
            f(cfg(), cache, none.long(), counts, 10, stream=0)
        with pytest.raises(ValueError):
            f(cfg(), cache, none, counts.long(), 10, stream=0)
        with pytest.raises(P.ClimberError):
            f(cfg(), cache, None, counts, 0, stream=0)
