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


def test_launches_that_would_be_too_large():
    # a launch has fewer than 2^32 threads: 2^24 workgroups of 256, of 1024 for an eviction
    c = cfg()
    lib = P.load_library()
    assert attend(cache=kv(n_seqs=1 << 20)) == RANGE      # 2^20 sequences x 2 heads x 2304 (2048 and up to 256 more) tokens: 1.1 x 2^32
    assert attend(cache=kv(n_seqs=1 << 22, max_len=16)) == RANGE
    assert attend(cache=kv(n_seqs=1 << 16), m_total=1 << 18, m_max=1 << 17) == RANGE   # rows of 2^16 sequences with 2^17 each
    assert P.climber_paged_workspace_bytes(c, kv(n_seqs=1 << 22, max_len=16), 4, 4) == 0
    cache = kv(n_seqs=1 << 13, max_len=1 << 21, table_ld=1 << 15, n_kv_heads=1)
    assert lib.climber_paged_evict(C.byref(c), C.byref(cache), FAKE, FAKE, None, FAKE, None, FAKE, 1 << 40, None) == RANGE
    f32 = cfg(dtype=P.F32)
    assert attend(f32, kv(n_seqs=1 << 16, max_len=1 << 12, table_ld=64, mass=FAKE)) == RANGE
    assert attend(f32, kv(n_seqs=1 << 12, max_len=1 << 12, table_ld=64, mass=FAKE)) == BUFSIZE


def test_caches_and_streams_of_other_devices(monkeypatch):
    torch = pytest.importorskip("torch")
    pages, table, n = torch.zeros(10, 2, 16, 64), torch.zeros(3, 4, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        P.paged_kv(pages, pages, table.to("meta"), n, 64)
    cache = kv()
    cache._device = 1                                   # a cache of cuda:1 while cuda:0 is the current device
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    other = type("Stream", (), {"cuda_stream": 5, "device_index": 0})()
    for stream in (None, other):
        with pytest.raises(ValueError):
            P.climber_attn_history_paged(cfg(), FAKE, cache, FAKE, FAKE, FAKE, FAKE, 4, 4, FAKE, FAKE, None, FAKE, None, stream)
        with pytest.raises(ValueError):
            P.climber_attn_sumi_paged(cfg(), FAKE, cache, FAKE, FAKE, FAKE, FAKE, 4, 4, FAKE, FAKE, FAKE, None, stream)
        with pytest.raises(ValueError):
            P.climber_paged_evict(cfg(), cache, FAKE, FAKE, None, FAKE, None, None, stream)
    other.device_index = 1                              # its own device: the call goes on, and stops at its arguments
    with pytest.raises(P.ClimberError) as e:
        P.climber_paged_evict(cfg(), cache, FAKE, None, None, FAKE, None, None, other)
    assert e.value.code == NULL


@pytest.mark.parametrize("name", ["climber_attn_history_paged", "climber_attn_sumi_paged", "climber_paged_evict"])
def test_native_binding_passes_every_argument_in_its_place(name, monkeypatch):
    # the binding's entry point is replaced by one that records what arrives; what it does not convert goes to ctypes, which does or refuses
    torch = pytest.importorskip("torch")
    from paper_2502_09888_amd import _native, climber as mod
    lib = P.load_library()
    real, args = getattr(lib, name), getattr(lib, name).argtypes
    seen = []
    structs = [hasattr(t, "_type_") and hasattr(t._type_, "_fields_") for t in args]

    def record(*a):
        seen.append([C.string_at(x, C.sizeof(t._type_)) if s else x for x, t, s in zip(a, args, structs)])
        return -5
    call = C.CFUNCTYPE(C.c_int, *(C.c_void_p if s else t for t, s in zip(args, structs)))(record)

    def bind(which):
        def address(n):
            return C.cast(call if n == which else getattr(lib, n), C.c_void_p).value
        _native.bind(*(address(n) for n in ("climber_attn_history", "climber_attn_sumi", "climber_attn_history_bias", "climber_attn_sumi_bias")),
                     P.Config, P.RelBias, torch.cuda.current_device, torch._C._cuda_getCurrentRawStream,
                     *(address(n) for n in ("climber_attn_history_paged", "climber_attn_sumi_paged", "climber_paged_evict")), PagedKV)
    c, cache = cfg(), kv()
    rows = torch.zeros(6, 12 * 64, dtype=torch.bfloat16)                        # one projection's output: 8 + 2 + 2 heads
    q, k, v = rows[:, :512], rows[:, 512:640], rows[:, 640:].unflatten(1, (2, 64))
    o, t, ws = torch.zeros(6, 8, 64, dtype=torch.bfloat16), [torch.zeros(4) for _ in range(8)], torch.zeros(300, dtype=torch.uint8)
    raw = [C.string_at(C.byref(x), C.sizeof(x)) for x in (c, cache)]
    ptr = [x.data_ptr() for x in t]
    if name == "climber_paged_evict":
        given = [c, cache, t[0], t[1], None, t[2], FAKE, ws]
        arrives = [*raw, ptr[0], ptr[1], None, ptr[2], FAKE, ws.data_ptr(), 300]
    elif name == "climber_attn_sumi_paged":
        given = [c, t[0], cache, q, k, v, t[1], 70000, 2**31 - 1, t[2], t[3], o, ws]
        arrives = [raw[0], ptr[0], raw[1], q.data_ptr(), 768, k.data_ptr(), v.data_ptr(), 768, ptr[1], 70000, 2**31 - 1, ptr[2], ptr[3],
                   o.data_ptr(), 512, ws.data_ptr(), 300]
    else:
        given = [c, t[0], cache, FAKE, q[:1, :128], k[1:2], t[1], 1, 1, t[2], t[3], t[4], o, None]
        arrives = [raw[0], ptr[0], raw[1], FAKE, 512, q.data_ptr(), k[1:2].data_ptr(), 128, ptr[1], 1, 1, ptr[2], ptr[3], ptr[4], o.data_ptr(), 512,
                   None, 0]
    try:
        bind(name)
        for stream, handle in ((0x55AA, 0x55AA), (type("S", (), {"cuda_stream": 77})(), 77), (0, None)):
            with pytest.raises(P.ClimberError) as e:
                getattr(P, name)(*given, stream=stream)
            assert e.value.code == -5 and seen.pop() == arrives + [handle]
        for at in range(len(given)):
            bad = list(given)
            bad[at] = type("Wrong", (), {})()
            with pytest.raises((AttributeError, TypeError, C.ArgumentError)):
                getattr(P, name)(*bad, stream=0)
        if name == "climber_attn_sumi_paged":           # rows that no pitch describes
            for at, bad in ((3, rows.t()), (4, rows.view(6, 12, 64).transpose(1, 2)), (5, torch.zeros(6, 128)), (11, rows[:, ::2])):
                wrong = list(given)
                wrong[at] = bad
                with pytest.raises(ValueError):
                    getattr(P, name)(*wrong, stream=0)
        assert not seen and mod._native is _native and real.argtypes == args
    finally:
        bind(None)


def test_a_cache_of_other_types_is_none():
    torch = pytest.importorskip("torch")
    parts = dict(k=torch.zeros(10, 2, 16, 64), v=torch.zeros(10, 2, 16, 64), page_table=torch.zeros(3, 4, dtype=torch.int32),
                 len=torch.zeros(3, dtype=torch.int32), mass=torch.zeros(10, 16), stamp=torch.zeros(10, 16, dtype=torch.int32))
    P.paged_kv(**parts, max_len=64)
    P.paged_kv(**{**parts, "k": parts["k"].bfloat16(), "v": parts["v"].bfloat16(), "mass": None}, max_len=64)
    for name, to in (("k", torch.bfloat16), ("v", torch.float64), ("page_table", torch.int64), ("len", torch.int64), ("mass", torch.float64),
                     ("stamp", torch.float32)):
        with pytest.raises(ValueError):
            P.paged_kv(**{**parts, name: parts[name].to(to)}, max_len=64)
    with pytest.raises(ValueError):
        P.paged_kv(**{**parts, "k": parts["k"].half(), "v": parts["v"].half()}, max_len=64)
