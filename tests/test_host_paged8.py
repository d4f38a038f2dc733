"""Refusals of the calls on the paged cache in 8 bits: they come back before anything would be launched, so no GPU is needed.  And the host's
definition of its rounding, which the GPU tests go by."""
import ctypes as C

import numpy as np
import pytest

import paper_2502_09888_amd as P
from paged8_ref import POSITIVE, decode, encode, scale_for
from test_host_paged import ALIGN, BUFSIZE, FAKE, NULL, OK, RANGE, SHAPE, UNSUPPORTED, cfg, kv


def kv8(k_scale=FAKE, v_scale=FAKE, d_head=0, elem_bytes=0, **kw):
    x = kv(**kw)
    x.d_head, x.elem_bytes = d_head, elem_bytes
    return P.PagedKV8(x, k_scale, v_scale)


def attend(c=None, cache=None, sumi=False, null=(), **kw):
    a = dict(tau=FAKE, q=FAKE, ld_q=512, k=FAKE + (1 << 30), v=FAKE + (2 << 30), ld_kv=128, off=FAKE, m_total=10, m_max=4, scen=FAKE, beh=FAKE,
             stamp=None, o=FAKE + (3 << 30), ld_o=512, ws=FAKE, ws_bytes=0)
    a.update(kw)
    for n in null:
        a[n] = None
    c, cache = c or cfg(), cache or kv8()
    lib, ids = P.load_library(), (a["scen"], a["beh"]) + (() if sumi else (a["stamp"],))
    f = lib.climber_attn_sumi_paged8 if sumi else lib.climber_attn_history_paged8
    return f(C.byref(c), a["tau"], C.byref(cache), a["q"], a["ld_q"], a["k"], a["v"], a["ld_kv"], a["off"], a["m_total"], a["m_max"], *ids, a["o"],
             a["ld_o"], a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("sumi", [False, True])
def test_attention_refuses(sumi):
    # (a call whose arguments are all right stops at the workspace of 0 bytes, which is too small where the keys are shared out)
    assert attend(sumi=sumi) == BUFSIZE and attend(sumi=sumi, cache=kv8(elem_bytes=1, d_head=64)) == BUFSIZE
    for name in ("tau", "q", "k", "v", "off", "scen", "beh", "o", "ws"):
        assert attend(sumi=sumi, null=[name]) == NULL, name
    for name in ("k", "v", "page_table", "len", "k_scale", "v_scale"):
        assert attend(sumi=sumi, cache=kv8(**{name: None})) == NULL, name
    assert attend(sumi=sumi, m_total=-1) == SHAPE and attend(sumi=sumi, m_max=11) == SHAPE and attend(sumi=sumi, m_max=0) == SHAPE
    assert attend(sumi=sumi, m_total=1 << 23, m_max=4) == RANGE
    for name, least in (("ld_q", 512), ("ld_o", 512), ("ld_kv", 128)):
        assert attend(sumi=sumi, **{name: least - 8}) == SHAPE, name
        assert attend(sumi=sumi, **{name: least + 4}) == ALIGN, name
        assert attend(sumi=sumi, **{name: 1 << 41}) == RANGE, name
    for name in ("q", "k", "v", "o"):
        assert attend(sumi=sumi, **{name: FAKE + (4 << 30) + 8}) == ALIGN, name
        if name != "o":
            assert attend(sumi=sumi, **{name: FAKE + (3 << 30)}) == UNSUPPORTED, name
    assert attend(sumi=sumi, ws=FAKE + 16, ws_bytes=1 << 30) == ALIGN
    assert attend(sumi=sumi, cache=kv8(k=FAKE + 8)) == ALIGN
    assert attend(sumi=sumi, m_total=0, m_max=0, null=["q", "k", "v", "scen", "beh", "o", "ws"]) == OK
    # not bf16, weights, sizes that are none
    assert attend(cfg(dtype=P.F32), sumi=sumi) == UNSUPPORTED
    assert attend(sumi=sumi, cache=kv8(mass=FAKE)) == UNSUPPORTED
    assert attend(cfg(d_head=96), sumi=sumi, ld_q=768, ld_o=768, ld_kv=192) == UNSUPPORTED
    assert attend(sumi=sumi, cache=kv8(elem_bytes=2)) == SHAPE and attend(sumi=sumi, cache=kv8(d_head=128)) == SHAPE
    assert attend(sumi=sumi, cache=kv8(n_kv_heads=3)) == SHAPE and attend(sumi=sumi, cache=kv8(page_size=24)) == ALIGN
    assert attend(sumi=sumi, cache=kv8(page_size=8)) == ALIGN and attend(sumi=sumi, cache=kv8(max_len=2049)) == RANGE
    if not sumi:
        assert attend(cfg(sub_len=128)) == UNSUPPORTED and attend(cache=kv8(stamp=FAKE)) == NULL and attend(cache=kv8(max_len=0)) == RANGE


def test_workspace_and_other_calls():
    lib, c = P.load_library(), cfg()
    assert P.climber_paged8_workspace_bytes(c, kv8(), 10, 4) > 0
    assert P.climber_paged8_workspace_bytes(c, kv8(mass=FAKE), 10, 4) == 0 and P.climber_paged8_workspace_bytes(cfg(dtype=P.F32), kv8(), 10, 4) == 0
    assert P.climber_paged8_workspace_bytes(c, kv8(), 4, 10) == 0
    cache = kv8(elem_bytes=1, d_head=64)
    # the other calls on a paged cache do not take one whose elements are bytes; the check of its table and lengths does
    assert lib.climber_paged_evict(C.byref(c), C.byref(cache.kv), FAKE, FAKE, None, FAKE, None, FAKE, 1 << 30, None) == SHAPE
    assert lib.climber_check_paged(C.byref(c), C.byref(cache.kv), None, 0, 0, 0, None, None) == NULL
    # a smaller call's workspace is never larger
    for m_total, m_max in ((1000, 100), (64, 1), (1, 1)):
        most = P.climber_paged8_workspace_bytes(c, kv8(), m_total, m_max)
        assert all(P.climber_paged8_workspace_bytes(c, kv8(), m, min(m, m_max)) <= most for m in range(1, m_total, 37))


def test_a_cache_of_other_types_is_none():
    torch = pytest.importorskip("torch")
    parts = dict(k=torch.zeros(10, 2, 32, 64, dtype=torch.uint8), v=torch.zeros(10, 2, 32, 64, dtype=torch.uint8).view(torch.float8_e4m3fn),
                 k_scale=torch.zeros(10, 2, 2, dtype=torch.uint8), v_scale=torch.zeros(10, 2, 2, dtype=torch.uint8),
                 page_table=torch.zeros(3, 4, dtype=torch.int32), len=torch.zeros(3, dtype=torch.int32), stamp=torch.zeros(10, 32, dtype=torch.int32))
    cache = P.paged_kv8(**parts, max_len=64)
    assert (cache.kv.elem_bytes, cache.kv.d_head, cache.kv.page_size, cache.kv.table_ld) == (1, 64, 32, 4)
    for name, to in (("k", torch.int8), ("v", torch.bfloat16), ("k_scale", torch.float32), ("page_table", torch.int64), ("len", torch.int64),
                     ("stamp", torch.float32)):
        with pytest.raises(ValueError):
            P.paged_kv8(**{**parts, name: parts[name].to(to)}, max_len=64)
    for name, x in (("k", parts["k"][:, :, :, :32]), ("k_scale", parts["k_scale"][:, :, :1]), ("v_scale", parts["v_scale"][:5]), ("len", parts["len"][:2])):
        with pytest.raises(ValueError):
            P.paged_kv8(**{**parts, name: x.contiguous()}, max_len=64)
    # tensors in host memory, which no kernel can reach, are noticed by the call
    with pytest.raises(ValueError):
        P.climber_attn_sumi_paged8(cfg(), None, cache, None, None, None, None, 0, 0, None, None, None, None)


def test_rounding_as_torch_has_it():
    torch = pytest.importorskip("torch")
    g = torch.Generator().manual_seed(1)
    x = torch.cat([torch.randn(4000, generator=g) * s for s in (1e-3, 0.01, 1.0, 50.0)]).clamp(-448, 448)
    mid = torch.from_numpy((POSITIVE[1:] + POSITIVE[:-1]) / 2).float()
    x = torch.cat([x, mid, -mid, torch.tensor([0.0, -0.0, 448.0, float("inf"), float("nan")])])
    ours, theirs = decode(encode(x.numpy())), x.to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(ours, theirs, equal_nan=True)
    for s in range(10, 248, 13):
        top = 448 * 2.0 ** (s - 127)
        assert scale_for([top, -0.5 * top]) == s and (scale_for([top * (1 + 2.0 ** -7)]) == s + 1 or s == 247)
    assert scale_for([0.0]) == scale_for([float("nan"), float("inf")]) == 10


@pytest.mark.parametrize("name", ["climber_attn_history_paged8", "climber_attn_sumi_paged8"])
def test_native_binding_marshals_as_ctypes_does(name):
    torch = pytest.importorskip("torch")
    from paper_2502_09888_amd import _native
    lib = P.load_library()
    args = getattr(lib, name).argtypes
    structs = [hasattr(t, "_type_") and hasattr(t._type_, "_fields_") for t in args]
    seen = []

    def record(*a):
        seen.append([C.string_at(x, C.sizeof(t._type_)) if s else x for x, t, s in zip(a, args, structs)])
        return -5
    call = C.CFUNCTYPE(C.c_int, *(C.c_void_p if s else t for t, s in zip(args, structs)))(record)

    def bind(which):
        def address(n):
            return C.cast(call if n == which else getattr(lib, n), C.c_void_p).value
        _native.bind(*(address(n) for n in ("climber_attn_history", "climber_attn_sumi", "climber_attn_history_bias", "climber_attn_sumi_bias")),
                     P.Config, P.RelBias, torch.cuda.current_device, torch._C._cuda_getCurrentRawStream,
                     *(address(n) for n in ("climber_attn_history_paged", "climber_attn_sumi_paged", "climber_paged_evict")), P.PagedKV,
                     *(address(n) for n in ("climber_attn_history_paged8", "climber_attn_sumi_paged8")), P.PagedKV8)
    c, cache = cfg(), kv8(stamp=FAKE)
    rows = torch.zeros(6, 12 * 64, dtype=torch.bfloat16)
    q, k, v = rows[:, :512], rows[:, 512:640], rows[:, 640:].unflatten(1, (2, 64))
    o, t, ws = torch.zeros(6, 8, 64, dtype=torch.bfloat16), [torch.zeros(4) for _ in range(5)], torch.zeros(300, dtype=torch.uint8)
    raw, ptr = [C.string_at(C.byref(x), C.sizeof(x)) for x in (c, cache)], [x.data_ptr() for x in t]
    stamp = [] if "sumi" in name else [t[4]]
    given = [c, t[0], cache, q, k, v, t[1], 7, 5, t[2], t[3], *stamp, o, ws]
    arrives = [raw[0], ptr[0], raw[1], q.data_ptr(), 768, k.data_ptr(), v.data_ptr(), 768, ptr[1], 7, 5, ptr[2], ptr[3], *(x.data_ptr() for x in stamp),
               o.data_ptr(), 512, ws.data_ptr(), 300]
    try:
        bind(name)
        for stream, handle in ((0x55AA, 0x55AA), (0, None)):
            with pytest.raises(P.ClimberError) as e:
                getattr(P, name)(*given, stream=stream)
            assert e.value.code == -5 and seen.pop() == arrives + [handle]
        for at in range(len(given)):
            bad = list(given)
            bad[at] = type("Wrong", (), {})()
            with pytest.raises((AttributeError, TypeError, C.ArgumentError)):
                getattr(P, name)(*bad, stream=0)
        assert not seen
    finally:
        bind(None)
