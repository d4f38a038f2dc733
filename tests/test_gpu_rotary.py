"""Rotary positions on the GPU against rotations in 64 bits."""
import math

import pytest
import torch

import paper_2502_09888_amd as P

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
KINDS = {"plain": P.ROTARY_PLAIN, "linear": P.ROTARY_LINEAR, "base": P.ROTARY_BASE, "parts": P.ROTARY_PARTS}


def reference(x, pos, freq, rot, interleaved, scale, inverse):
    """(turned rows, bound) in 64 bits; x [m, heads, d] on the CPU."""
    y = x.double()
    a, b = (y[..., 0:rot:2], y[..., 1:rot:2]) if interleaved else (y[..., :rot // 2], y[..., rot // 2:rot])
    t = pos.double()[:, None] * torch.tensor(freq, dtype=torch.float64)
    c, s = (f(t)[:, None] * scale for f in (torch.cos, torch.sin))
    if inverse:
        s = -s
    u, v = a * c - b * s, a * s + b * c
    out, tol = y.clone(), torch.zeros_like(y)
    # An angle is off by the three roundings of position * frequency / (2 pi) in 64 bits and by those of pi / 2 and of the eighth of a turn in
    # 32, sines and cosines by five more half steps of 32 bits (and 2e-9, less than one), the products and their sum by two.
    e = (abs(scale) * (a.abs() + b.abs())) * (9 * 2.0 ** -24 + 4 * 2.0 ** -53 * t.abs()[:, None])
    half = 2.0 ** -8 if x.dtype == torch.bfloat16 else 2.0 ** -24
    if interleaved:
        out[..., 0:rot:2], out[..., 1:rot:2] = u, v
        tol[..., 0:rot:2] = tol[..., 1:rot:2] = e
    else:
        out[..., :rot // 2], out[..., rot // 2:rot] = u, v
        tol[..., :rot // 2] = tol[..., rot // 2:rot] = e
    tol[..., :rot] += (out[..., :rot].abs() + tol[..., :rot]) * half
    return out, tol


def turned(m, H, Hkv, d, rot, dtype, *, interleaved=False, kind="plain", inverse=False, place="out", pad=0, pos=None, seed=0):
    """Runs the call on rows laid out as `place` says and checks it; returns the turned rows on the GPU."""
    g = torch.Generator().manual_seed(seed)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    q, k = (torch.randn(m, h, d, generator=g).to(dt) for h in (H, Hkv))
    pos = torch.randint(0, 4096, (m,), generator=g, dtype=torch.int32) if pos is None else pos
    freq, scale = P.climber_rotary_frequencies(rot, 10000.0, KINDS[kind], 8.0, 2048.0, 32.0, 1.0)
    plan = P.rotary(torch.tensor(freq, dtype=torch.float64, device=DEV), rot, interleaved=interleaved, scale=scale, inverse=inverse)
    cfg = P.Config(n_heads=H, d_head=d, dtype=P.F32 if dtype == "f32" else P.BF16)
    w = (H + 2 * Hkv) * d
    rows = torch.full((m, w + pad), 3.0, dtype=dt, device=DEV)
    dq, dk = rows[:, :H * d], rows[:, H * d:(H + Hkv) * d]
    dq.copy_(q.view(m, -1)), dk.copy_(k.view(m, -1))
    if place == "in":                                     # columns of one projection's output, turned where they are
        oq, ok = dq, dk
    else:
        oq, ok = (torch.full((m, h, d), 5.0, dtype=dt, device=DEV) for h in (H, Hkv))
    P.climber_rotary(cfg, plan, pos.to(DEV), Hkv, dq, dk if Hkv else None, oq, ok if Hkv else None)
    torch.cuda.synchronize()
    for x, y in ((q, oq), (k, ok)):
        if x.numel():
            want, tol = reference(x, pos, freq, rot, interleaved, scale, inverse)
            got = y.double().cpu().view(x.shape)
            assert ((got - want).abs() <= tol).all(), float(((got - want).abs() - tol).max())
    assert (rows[:, (H + Hkv) * d:] == 3.0).all()         # the values' columns
    if place != "in":
        assert torch.equal(dq.cpu(), q.view(m, -1))
    return oq, ok


@pytest.mark.parametrize("place", ["out", "in"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,rot", [(64, 64), (128, 128), (128, 64), (64, 48), (64, 2), (80, 26), (32, 10), (7, 4), (2, 2), (256, 256), (512, 512), (600, 512),
                                   (256, 114), (256, 26), (128, 78), (72, 66), (41, 18), (40, 34), (23, 16), (19, 18)])
def test_widths(d, rot, dtype, interleaved, place):
    turned(37, 4, 2, d, rot, dtype, interleaved=interleaved, place=place, seed=d + rot)


@pytest.mark.parametrize("m", [1, 2, 255, 4095, 4096, 4099, 20001])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows(m, dtype):
    turned(m, 3, 1, 64, 64, dtype, place="in", pad=8, seed=m)


@pytest.mark.parametrize("H,Hkv", [(1, 1), (5, 0), (40, 8), (1, 7)])
def test_heads(H, Hkv):
    turned(9, H, Hkv, 128, 96, "bf16", seed=H)
    turned(9, H, Hkv, 64, 64, "f32", interleaved=True, place="in", pad=3, seed=H)   # (a pitch that is no multiple of 16 bytes)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("inverse", [False, True])
def test_kinds_and_inverses(kind, inverse):
    turned(50, 2, 2, 64, 64, "f32", kind=kind, inverse=inverse)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_far_and_negative_positions(dtype):
    pos = torch.tensor([0, 1, -1, 5, -4096, 10 ** 6, 10 ** 9, 2 ** 31 - 1, -2 ** 31, 2 ** 24 + 1, 314159265, 355, 103993, 710], dtype=torch.int32)
    for interleaved in (False, True):
        turned(14, 2, 1, 128, 128, dtype, interleaved=interleaved, pos=pos)


def test_odd_numbers_stay_in_their_pair():
    q = torch.randn(3, 1, 16, device=DEV)
    q[1, 0, 2], q[2, 0, 15] = math.nan, math.inf
    cfg, pos = P.Config(n_heads=1, d_head=16, dtype=P.F32), torch.tensor([3, 4, 5], dtype=torch.int32, device=DEV)
    freq, _ = P.climber_rotary_frequencies(8)
    out = torch.empty_like(q)
    P.climber_rotary(cfg, P.rotary(torch.tensor(freq, dtype=torch.float64, device=DEV), 8), pos, 0, q, None, out, None)
    bad = ~torch.isfinite(out)
    assert bad.nonzero().tolist() == [[1, 0, 2], [1, 0, 6], [2, 0, 15]]


@pytest.mark.parametrize("interleaved", [False, True])
def test_the_inverse_is_the_gradient_and_turns_back(interleaved):
    m, H, d, rot = 6, 2, 12, 8
    cfg = P.Config(n_heads=H, d_head=d, dtype=P.F32)
    freq, _ = P.climber_rotary_frequencies(rot)
    f = torch.tensor(freq, dtype=torch.float64, device=DEV)
    g = torch.Generator().manual_seed(3)
    x, dy = (torch.randn(m, H, d, generator=g).to(DEV) for _ in range(2))
    pos = torch.tensor([0, 1, 7, 100, 5000, 123456], dtype=torch.int32, device=DEV)
    scale = 1.25

    def call(v, inverse):
        out = torch.empty_like(v)
        P.climber_rotary(cfg, P.rotary(f, rot, interleaved=interleaved, scale=scale, inverse=inverse), pos, 0, v, None, out, None)
        return out
    dx = call(dy, True).double()
    # sum(y dy) is linear in x: its differences are exact but for the roundings of y, 12 half steps of |y| < 4 in 16 terms a row
    for r in range(m):
        for e in range(d):
            step = torch.zeros_like(x)
            step[r, 1, e] = 1.0
            up = (call(x + step, False).double() * dy.double()).sum()
            down = (call(x - step, False).double() * dy.double()).sum()
            assert abs((up - down).item() / 2 - dx[r, 1, e].item()) <= 2e-4
    # there and back: scale^2 on what is turned
    back = call(call(x, False), True)
    assert torch.allclose(back[..., :rot], x[..., :rot] * scale ** 2, rtol=0, atol=40 * 2.0 ** -24 * 8) and torch.equal(back[..., rot:], x[..., rot:])


def test_captured_and_on_another_stream():
    m, H, d = 5, 4, 64
    cfg = P.Config(n_heads=H, d_head=d, dtype=P.BF16)
    freq, scale = P.climber_rotary_frequencies(64)
    plan = P.rotary(torch.tensor(freq, dtype=torch.float64, device=DEV), 64)
    q, k = (torch.randn(m, h, d, device=DEV).bfloat16() for h in (H, 2))
    pos, oq, ok = torch.arange(m, dtype=torch.int32, device=DEV), torch.empty_like(q), torch.empty_like(k)
    P.climber_rotary(cfg, plan, pos, 2, q, k, oq, ok)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph):
        P.climber_rotary(cfg, plan, pos, 2, q, k, oq, ok)
    for i in range(4):
        pos += 1000 * i
        q.copy_(torch.randn(m, H, d, device=DEV))
        eq, ek = torch.empty_like(q), torch.empty_like(k)
        torch.cuda.synchronize()
        graph.replay()
        P.climber_rotary(cfg, plan, pos, 2, q, k, eq, ek, side)
        torch.cuda.synchronize()
        assert torch.equal(oq, eq) and torch.equal(ok, ek)


@pytest.mark.parametrize("interleaved", [False, True])
def test_logits_of_turned_rows_depend_on_distances_alone(interleaved):
    """In use: turned rows appended to a paged history in 8 bits and scored, at positions shifted by any number: the same outputs."""
    from paged8_ref import Case8, Device8, check8
    outs = []
    for shift in (0, 77777):
        case = Case8([0], [90], H=4, Hkv=2, seed=12, page=32)
        freq, scale = P.climber_rotary_frequencies(64, 10000.0, P.ROTARY_PARTS, 4.0, 64.0, 32.0, 1.0)
        plan = P.rotary(torch.tensor(freq, dtype=torch.float64, device=DEV), 64, interleaved=interleaved, scale=scale)
        pos = torch.arange(90, dtype=torch.int32, device=DEV) + shift
        dev = Device8(case)
        P.climber_rotary(dev.cfg, plan, pos, 2, dev.q, dev.kn, dev.q, dev.kn)
        case.q, case.kn = dev.q.cpu(), dev.kn.cpu()
        dev.attend()
        check8(case, dev)
        outs.append(dev.out())
    # rows are rounded to bf16 behind the turn: logits differ by two half steps of 2^-8 each of sum |q||k| d^-0.5 / tau < 60, in the mean far less
    assert (outs[0] - outs[1]).abs().max() < 0.25 and (outs[0] - outs[1]).square().mean().sqrt() < 0.02
