"""The paged cache in 8 bits on the host: its rounding and its append by their definitions, on top of paged_ref.py."""
import math

import numpy as np
import torch

from paged_ref import Case, Device

POSITIVE = np.array([(m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)) for e in range(16) for m in range(8)][:127])
NAN = 0x7F


def decode(codes):
    """Values of e4m3 codes, in 64 bits (numpy)."""
    codes = np.asarray(codes)
    mag = np.append(POSITIVE, math.nan)[codes & 127]
    return np.where(codes & 128, -mag, mag)


def encode(x):
    """The nearest e4m3 number's code, ties to the even one; |x| <= 448, or not finite: NaN."""
    x = np.asarray(x, dtype=np.float64)
    a = np.where(np.isfinite(x), np.abs(x), 0)
    hi = np.clip(np.searchsorted(POSITIVE, a), 1, 126)
    lo = hi - 1
    up, down = POSITIVE[hi] - a, a - POSITIVE[lo]
    code = np.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
    code = np.where(np.isfinite(x), code | np.where(np.signbit(x), 128, 0), NAN)
    return code.astype(np.uint8)


def scale_for(values):
    """The least stored scale, from 10 on, with which the finite ones stay within 448."""
    a = np.abs(np.asarray(values, dtype=np.float64))
    top = a[np.isfinite(a)].max(initial=0.0)
    s = 10
    while top > 448 * 2.0 ** (s - 127):
        s += 1
    return s


class Case8(Case):
    """A Case whose cached tokens are held in 8 bits: `k`, `v` are the values that they stand for, `codes` and `scales` what the cache holds."""

    def __init__(self, *args, **kw):
        super().__init__(*args, **kw)
        self.quantise()

    def quantise(self):
        n, H, P, d = self.k.shape
        self.codes, self.scales = {}, {}
        for name in ("k", "v"):
            codes, scales = np.full((n, H, P, d), NAN, np.uint8), np.full((n, H, P // 16), 255, np.uint8)
            x = getattr(self, name).double().numpy()
            for b, c in enumerate(self.cached):
                for j in range(0, c, 16):
                    pg, s = self.at(b, j)
                    m = min(16, c - j)
                    for h in range(H):
                        scales[pg, h, s // 16] = e = scale_for(x[pg, h, s:s + m])
                        codes[pg, h, s:s + m] = encode(x[pg, h, s:s + m] * 2.0 ** (127 - e))
            self.codes[name], self.scales[name] = codes, scales
            setattr(self, name, torch.from_numpy(self.held(name)).to(torch.bfloat16))

    def held(self, name):
        return decode(self.codes[name]) * 2.0 ** (np.repeat(self.scales[name].astype(np.float64), 16, axis=2)[..., None] - 127)

    def append(self, limit=None):
        """The chunk joins the cache (codes, scales, stamps); slots from `limit` on and tokens without a page are left out."""
        for b, (n, t) in enumerate(zip(self.cached, self.chunk)):
            r0, end = int(self.off[b]), min(n + t, limit if limit is not None else n + t)
            for j in range(n // 16 * 16, end, 16):
                pg, s = self.at(b, j)
                if pg < 0 or pg >= self.n_pages or t == 0:
                    continue
                old, m = max(0, n - j), min(16, end - j)
                for i in range(old, m):
                    self.stamp[pg, s + i] = self.stamp_new[r0 + j + i - n]
                for name, rows in (("k", self.kn), ("v", self.vn)):
                    codes, scales = self.codes[name], self.scales[name]
                    for h in range(self.Hkv):
                        x = rows[r0 + j + old - n:r0 + j + m - n, h].double().numpy()
                        was = int(scales[pg, h, s // 16]) if old else 0
                        now = max(was, scale_for(x))
                        if old and now > was:
                            codes[pg, h, s:s + old] = encode(decode(codes[pg, h, s:s + old]) * 2.0 ** (was - now))
                        codes[pg, h, s + old:s + m] = encode(x * 2.0 ** (127 - now))
                        scales[pg, h, s // 16] = now


class Device8(Device):
    more = 0  # sequences without tokens and rows behind the case's own: the same problem in a launch for many

    def describe(self):
        P, dev = self.P, "cuda:0"
        if self.more and self.len.numel() == len(self.c.cached):
            self.table = torch.cat([self.table, self.table.new_full((self.more, self.table.shape[1]), -1)])
            self.len = torch.cat([self.len, self.len.new_zeros(self.more)])
            self.off = torch.cat([self.off, self.off[-1:].expand(self.more)])
        if not hasattr(self, "k_scale"):
            self.k, self.v = (torch.from_numpy(self.c.codes[n]).to(dev) for n in ("k", "v"))
            self.k_scale, self.v_scale = (torch.from_numpy(self.c.scales[n]).to(dev) for n in ("k", "v"))
        self.kv = P.paged_kv8(self.k, self.v, self.k_scale, self.v_scale, self.table, self.len, self.max_len, stamp=self.stamp)
        self.ws = torch.full((max(256, P.climber_paged8_workspace_bytes(self.cfg, self.kv, self.c.m, self.m_max)),), 0xFF, dtype=torch.uint8, device=dev)

    def history(self, stream=None):
        self.P.climber_attn_history_paged8(self.cfg, self.tau, self.kv, self.q, self.kn, self.vn, self.off, self.c.m, self.m_max, self.scen, self.beh,
                                           self.stamp_new if self.stamp is not None else None, self.o, self.ws, stream)

    def sumi(self, stream=None):
        self.P.climber_attn_sumi_paged8(self.cfg, self.tau, self.kv, self.q, self.kn, self.vn, self.off, self.c.m, self.m_max, self.scen, self.beh,
                                        self.o, self.ws, stream)


def check8(case, dev, limit=None):
    """o and what the cache holds after a call; the case takes the chunk."""
    o, tol, _, _ = case.expect()
    got = dev.out()
    rows = sum(case.chunk)
    assert torch.isfinite(got[:rows]).all()
    off = (got[:rows] - o[:rows]).abs() - tol[:rows]
    assert off.max() <= 0 if rows else True, f"max over the bound {off.max():.3e}, error {(got[:rows] - o[:rows]).abs().max():.3e}"
    assert (got[rows:] == 77.0).all()           # rows of no sequence
    if not case.sumi:
        case.append(limit)
    check_cache(case, dev)


def check_cache(case, dev):
    torch.cuda.synchronize()
    for name in ("k", "v"):
        scales, codes = getattr(dev, name + "_scale").cpu().numpy(), getattr(dev, name).cpu().numpy()
        assert np.array_equal(scales, case.scales[name]), name
        # (which of the two codes of NaN is not said, nor are two zeros told apart by their values)
        assert np.array_equal(decode(codes), decode(case.codes[name]), equal_nan=True), name
    if dev.stamp is not None:
        assert torch.equal(dev.stamp.cpu(), case.stamp)
