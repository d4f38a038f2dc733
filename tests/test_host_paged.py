"""Refusals of the paged calls: they come back before anything would be launched, so no GPU is needed."""
import ctypes as C

import pytest

import paper_2502_09888_amd as P
from paper_2502_09888_amd.climber import PagedKV, _pitch

FAKE = 0x7F0000000000   # 256-byte aligned, never dereferenced on the host
OK, NULL, SHAPE, ALIGN, RANGE, TAU, BUFSIZE, UNSUPPORTED = 0, -1, -2, -3, -4, -5, -6, -7


def cfg(**kw):
    return P.Config(**{**dict(n_heads=8, d_head=64, n_scen=8, n_beh=4, dtype=P.BF16, qk_scale=0.125), **kw})


def kv(**kw):
    f = dict(k=FAKE, v=FAKE, mass=None, stamp=None, page_table=FAKE, len=FAKE, n_pages=100, page_size=64, n_kv_heads=2, n_seqs=4,
             table_ld=32, max_len=2048)
    f.update(kw)
    return PagedKV(*f.values())


def attend(c=None, cache=None, sumi=False, null=(), **kw):
    a = dict(tau=FAKE, q=FAKE, ld_q=512, k=FAKE + (1 << 30), v=FAKE + (2 << 30), ld_kv=128, off=FAKE, m_total=10, m_max=4, scen=FAKE, beh=FAKE,
             stamp=None, o=FAKE + (3 << 30), ld_o=512, ws=FAKE, ws_bytes=0)
    a.update(kw)
    for n in null:
        a[n] = None
    c, cache = c or cfg(), cache or kv()
    lib, ids = P.load_library(), (a["scen"], a["beh"]) + (() if sumi else (a["stamp"],))
    f = lib.climber_attn_sumi_paged if sumi else lib.climber_attn_history_paged
    return f(C.byref(c), a["tau"], C.byref(cache), a["q"], a["ld_q"], a["k"], a["v"], a["ld_kv"], a["off"], a["m_total"], a["m_max"], *ids, a["o"],
             a["ld_o"], a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("sumi", [False, True])
def test_attention_refuses(sumi):
    # (a call whose arguments are all right stops at the workspace of 0 bytes, which is too small)
    assert attend(sumi=sumi, cache=kv(mass=FAKE)) == BUFSIZE
    for name in ("tau", "q", "k", "v", "off", "scen", "beh", "o"):
        assert attend(sumi=sumi, null=[name]) == NULL, name
    assert attend(sumi=sumi, cache=kv(mass=FAKE), null=["ws"]) == NULL
    for name in ("k", "v", "page_table", "len"):
        assert attend(sumi=sumi, cache=kv(**{name: None})) == NULL, name
    assert attend(sumi=sumi, m_total=-1) == SHAPE and attend(sumi=sumi, m_max=11) == SHAPE and attend(sumi=sumi, m_max=0) == SHAPE
    assert attend(sumi=sumi, m_total=1 << 23, m_max=4) == RANGE
    for name, least in (("ld_q", 512), ("ld_o", 512), ("ld_kv", 128)):
        assert attend(sumi=sumi, **{name: least - 8}) == SHAPE, name
        assert attend(sumi=sumi, **{name: least + 4}) == ALIGN, name
        assert attend(sumi=sumi, **{name: 1 << 41}) == RANGE, name
    for name in ("q", "k", "v", "o"):
        assert attend(sumi=sumi, **{name: FAKE + (4 << 30) + 8}) == ALIGN, name
    assert attend(sumi=sumi, cache=kv(mass=FAKE), ws=FAKE + 16, ws_bytes=1 << 30) == ALIGN
    assert attend(sumi=sumi, cache=kv(k=FAKE + 8)) == ALIGN
    # no rows: nothing to do, nothing looked at
    assert attend(sumi=sumi, m_total=0, m_max=0, null=["q", "k", "v", "scen", "beh", "o", "ws"]) == OK
    # outputs on the rows that are still read; columns of the same rows are apart
    for name in ("q", "k", "v"):
        assert attend(sumi=sumi, **{name: FAKE + (3 << 30)}) == UNSUPPORTED, name
    assert attend(sumi=sumi, cache=kv(mass=FAKE), q=FAKE, k=FAKE + 1024, v=FAKE + 1280, o=FAKE + 1536, ld_q=1280, ld_kv=1280, ld_o=1280) == BUFSIZE
    assert attend(sumi=sumi, q=FAKE, k=FAKE + 1024, v=FAKE + 1280, o=FAKE + 1520, ld_q=1280, ld_kv=1280, ld_o=1280) == UNSUPPORTED


def test_history_alone_refuses():
    assert attend(cfg(sub_len=128)) == UNSUPPORTED and attend(cfg(sub_len=128), kv(mass=FAKE), sumi=True) == BUFSIZE
    assert attend(cache=kv(stamp=FAKE)) == NULL
    assert attend(cache=kv(max_len=0)) == RANGE


@pytest.mark.parametrize("call", ["history", "sumi", "evict", "check", "bytes"])
def test_caches_and_configurations_that_are_none(call):
    lib = P.load_library()

    def run(c=None, cache=None):
        c, cache = c or cfg(), cache or kv(mass=FAKE)
        if call in ("history", "sumi"):
            return attend(c, cache, sumi=call == "sumi")
        if call == "evict":
            return lib.climber_paged_evict(C.byref(c), C.byref(cache), FAKE, FAKE, None, FAKE, None, FAKE, 0, None)
        if call == "check":   # (stops at the missing status word)
            return lib.climber_check_paged(C.byref(c), C.byref(cache), FAKE, 10, 4, 1, None, None)
        return lib.climber_paged_workspace_bytes(C.byref(c), C.byref(cache), 10, 4)

    fine = run()
    assert fine > 0 if call == "bytes" else fine == (NULL if call == "check" else BUFSIZE)

    def refused(code, *args, **kw):
        got = run(*args, **kw)
        assert got == (0 if call == "bytes" else code), (got, code)

    for field in ("n_pages", "n_seqs", "table_ld", "n_kv_heads", "page_size"):
        for value in (0, -1):
            refused(SHAPE, cache=kv(mass=FAKE, **{field: value}))
    refused(SHAPE, cache=kv(mass=FAKE, n_kv_heads=3))
    for page in (8, 48, 8192):
        refused(ALIGN, cache=kv(mass=FAKE, page_size=page, max_len=64))
    refused(RANGE, cache=kv(mass=FAKE, max_len=-1))
    refused(RANGE, cache=kv(mass=FAKE, max_len=2049))
    refused(RANGE, cache=kv(mass=FAKE, table_ld=1 << 25))
    refused(RANGE, cache=kv(mass=FAKE, n_pages=1 << 26))
    refused(RANGE, cache=kv(mass=FAKE, n_seqs=1 << 26))
    for d in (32, 96, 256):
        refused(UNSUPPORTED, cfg(d_head=d))
    for d in (2, 30, 132):
        refused(UNSUPPORTED, cfg(d_head=d, dtype=P.F32))
    refused(TAU, cfg(qk_scale=0.0))
    refused(SHAPE, cfg(n_scen=0))
    refused(SHAPE, cfg(d_model=100))
    refused(SHAPE, cfg(flags=8))


def test_evict_and_check_refuse():
    lib, c = P.load_library(), cfg()

    def evict(cache=None, rank=FAKE, budget=FAKE, keep_from=None, len_out=FAKE, src=None, ws=FAKE, ws_bytes=0):
        cache = cache or kv()
        return lib.climber_paged_evict(C.byref(c), C.byref(cache), rank, budget, keep_from, len_out, src, ws, ws_bytes, None)

    assert evict() == BUFSIZE
    assert evict(budget=None) == NULL and evict(len_out=None) == NULL and evict(ws=None) == NULL
    assert evict(rank=None) == NULL and evict(kv(mass=FAKE), rank=None) == BUFSIZE
    assert evict(keep_from=FAKE) == NULL and evict(kv(stamp=FAKE), keep_from=FAKE) == BUFSIZE
    for name in ("rank", "budget", "len_out", "src"):
        assert evict(**{name: FAKE + 2}) == ALIGN, name
    assert evict(ws=FAKE + 16, ws_bytes=1 << 30) == ALIGN
    need = P.climber_paged_workspace_bytes(c, kv(), 0, 0)
    assert need > 0 and evict(ws_bytes=need - 1) == BUFSIZE
    cache = kv()
    assert lib.climber_check_paged(C.byref(c), C.byref(cache), None, 10, 4, 1, FAKE, None) == NULL
    assert lib.climber_check_paged(C.byref(c), C.byref(cache), FAKE, 10, 11, 1, FAKE, None) == SHAPE


def test_workspace_covers_every_call():
    for mass in (None, FAKE):
        small, large = (P.climber_paged_workspace_bytes(cfg(), kv(mass=mass), m, m) for m in (4, 4096))
        assert 0 < small <= large
    assert P.climber_paged_workspace_bytes(cfg(), kv(mass=FAKE), 4096, 4096) > P.climber_paged_workspace_bytes(cfg(), kv(), 4096, 4096)


def test_row_pitches_come_from_the_tensors():
    torch = pytest.importorskip("torch")
    x = torch.zeros(5, 3 * 64)
    assert _pitch(x, 64) == 192 and _pitch(x[:, :64], 64) == 192 and _pitch(x[:, 64:].unflatten(1, (2, 64)), 128) == 192
    assert _pitch(x[:1, :64], 64) == 64 and _pitch(FAKE, 64) == 64 and _pitch(x[:0], 192) == 192
    for bad in (x.t(), x.view(5, 3, 64).transpose(1, 2), x.view(5, 3, 64)[:, :, ::2]):
        with pytest.raises(ValueError):
            _pitch(bad, 64)
    pages, table, n = torch.zeros(10, 2, 16, 64), torch.zeros(3, 4, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    made = P.paged_kv(pages, pages.clone(), table, n, 64, mass=torch.zeros(10, 16))
    assert (made.n_pages, made.n_kv_heads, made.page_size, made.n_seqs, made.table_ld, made.max_len) == (10, 2, 16, 3, 4, 64)
    for args in ((pages, pages[:5], table, n), (pages, pages, table[:2], n), (pages.transpose(0, 1), pages, table, n)):
        with pytest.raises(ValueError):
            P.paged_kv(*args, 64)
    with pytest.raises(ValueError):
        P.paged_kv(pages, pages, table, n, 64, mass=torch.zeros(10, 8))
