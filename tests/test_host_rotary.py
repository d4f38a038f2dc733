"""Rotary positions: frequencies, and refusals (before anything would be launched, so no GPU is needed)."""
import ctypes as C
import math

import pytest

import paper_2502_09888_amd as P
from test_host_paged import ALIGN, FAKE, NULL, OK, RANGE, SHAPE, UNSUPPORTED, cfg


def test_frequencies():
    close = lambda a, b: all(abs(x - y) <= 1e-14 * abs(y) for x, y in zip(a, b))  # noqa: E731
    plain, one = P.climber_rotary_frequencies(64)
    assert one == 1.0 and len(plain) == 32 and close(plain, [10000.0 ** (-i / 32) for i in range(32)])
    linear, one = P.climber_rotary_frequencies(64, 10000.0, P.ROTARY_LINEAR, 4.0)
    assert one == 1.0 and close(linear, [f / 4 for f in plain])
    based, one = P.climber_rotary_frequencies(64, 10000.0, P.ROTARY_BASE, 4.0)
    assert one == 1.0 and based[0] == 1.0 and abs(based[-1] - plain[-1] / 4) < 1e-18
    parts, scale = P.climber_rotary_frequencies(64, 10000.0, P.ROTARY_PARTS, 16.0, 4096.0, 32.0, 1.0)
    assert abs(scale - (0.1 * math.log(16) + 1)) < 1e-7
    for f, was in zip(parts, plain):
        turns = 4096 * was / (2 * math.pi)
        r = min(1.0, max(0.0, (turns - 1) / 31))
        assert abs(f - (r * was + (1 - r) * was / 16)) < 1e-14
    assert parts[0] == plain[0] and abs(parts[-1] - plain[-1] / 16) < 1e-18
    assert P.climber_rotary_frequencies(2)[0] == [1.0]


def test_frequencies_refuse():
    def code(*a):
        with pytest.raises(P.ClimberError) as e:
            P.climber_rotary_frequencies(*a)
        return e.value.code
    assert code(0) == code(-2) == code(3) == code(514) == SHAPE
    for base in (0.0, -1.0, math.inf, math.nan):
        assert code(64, base) == RANGE
    for factor in (0.0, -2.0, math.nan, math.inf):
        for kind in (P.ROTARY_LINEAR, P.ROTARY_BASE, P.ROTARY_PARTS):
            assert code(64, 1e4, kind, factor, 4096.0) == RANGE
    assert code(2, 1e4, P.ROTARY_BASE, 2.0) == SHAPE and code(64, 1e4, 4) == code(64, 1e4, -1) == UNSUPPORTED
    for bad in ((0.0, 32.0, 1.0), (4096.0, 1.0, 1.0), (4096.0, 32.0, -1.0), (math.nan, 32.0, 1.0), (4096.0, math.inf, 1.0)):
        assert code(64, 1e4, P.ROTARY_PARTS, 2.0, *bad) == RANGE
    lib, s = P.load_library(), C.c_float()
    assert lib.climber_rotary_frequencies(64, 1e4, 0, 1.0, 0.0, 0.0, 0.0, None, C.byref(s)) == NULL


def call(c=None, null=(), freq=FAKE, rot=64, scale=1.0, **kw):
    a = dict(pos=FAKE, m=0, n_kv=2, q=FAKE, ld_q=512, k=FAKE + (1 << 30), ld_k=128, q_out=FAKE + (2 << 30), ld_qo=512, k_out=FAKE + (3 << 30), ld_ko=128)
    a.update(kw)
    for n in null:
        a[n] = None
    plan = P.RotaryPlan(freq, rot, 0, 0, scale)
    return P.load_library().climber_rotary(C.byref(c or cfg()), C.byref(plan), *a.values(), None)


def test_calls_refuse():
    assert call() == OK and call(null=["pos", "q", "k", "q_out", "k_out"]) == OK              # no rows: nothing is looked at
    assert call(freq=None) == NULL and call(freq=FAKE + 4) == ALIGN
    for rot in (0, -2, 3, 66):
        assert call(rot=rot) == SHAPE
    assert call(scale=math.nan) == SHAPE and call(cfg(d_head=600), rot=514, ld_q=4800, ld_qo=4800, ld_k=1200, ld_ko=1200) == UNSUPPORTED
    assert call(m=-1) == SHAPE and call(n_kv=-1) == SHAPE and call(cfg(dtype=7)) == UNSUPPORTED and call(cfg(d_model=100)) == SHAPE
    for name in ("ld_q", "ld_qo"):
        assert call(**{name: 511}) == SHAPE and call(**{name: 1 << 25}) == RANGE
    for name in ("ld_k", "ld_ko"):
        assert call(**{name: 127}) == SHAPE and call(**{name: 1 << 25}) == RANGE and call(n_kv=0, **{name: 0}) == OK
    for name in ("pos", "q", "k", "q_out", "k_out"):
        assert call(m=5, null=[name]) == NULL, name
        assert call(m=5, **{name: FAKE + (5 << 30) + 1}) == ALIGN, name
    # in place, or apart: not on other rows, not on the other's, not at another pitch
    for name, other in (("q_out", "k"), ("k_out", "q"), ("q_out", "k_out")):
        assert call(m=5, **{name: FAKE + (6 << 30), other: FAKE + (6 << 30)}) == UNSUPPORTED, (name, other)
    assert call(m=5, q_out=FAKE + 2) == UNSUPPORTED and call(m=5, q_out=FAKE, ld_qo=520) == UNSUPPORTED
    assert call(m=5, k_out=FAKE + (1 << 30) + 128) == UNSUPPORTED
    assert P.load_library().climber_rotary(None, None, *[None, 0, 0] + [None, 0] * 4, None) == NULL


def test_tensors_of_other_kinds_are_refused():
    torch = pytest.importorskip("torch")
    with pytest.raises(ValueError):
        P.rotary(torch.zeros(32), 64)
    with pytest.raises(ValueError):
        P.rotary(torch.zeros(31, dtype=torch.float64), 64)
    plan = P.rotary(torch.zeros(32, dtype=torch.float64), 64)
    q, pos = torch.zeros(3, 8, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):                       # frequencies in host memory, which no kernel can reach
        P.climber_rotary(cfg(), plan, pos, 0, q, None, q, None)
    plan._device = 3                                      # ... and rows elsewhere than these
    with pytest.raises(ValueError):
        P.climber_rotary(cfg(), plan, pos, 0, q, None, q, None, stream=0)
    plan._device = None
    for bad in (dict(q=q[:2]), dict(q_out=q.float()), dict(pos=pos.long()), dict(pos=pos[:2]), dict(q=q.transpose(1, 2).contiguous().transpose(1, 2))):
        a = {**dict(pos=pos, q=q, q_out=q), **bad}
        with pytest.raises(ValueError):
            P.climber_rotary(cfg(), plan, a["pos"], 0, a["q"], None, a["q_out"], None, stream=0)
