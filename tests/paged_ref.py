"""A paged cache on the host and its operators in 64 bits, by their definitions, token by token (used by the tests of the paged calls)."""
import math

import torch

LOG2E = 1.4426950408889634
HALF_BF16, HALF_F32 = 2.0 ** -8, 2.0 ** -24   # half a step of a rounding, relative


class Case:
    """One call's inputs on the CPU: values as the device gets them."""

    def __init__(self, cached, chunk, H=4, Hkv=2, d=64, page=16, dtype="bf16", causal=True, n_scen=3, n_beh=2, seed=0, free=2, std=1.0,
                 sumi=False, tail=0, scale=None):
        self.g = g = torch.Generator().manual_seed(seed)
        self.cached, self.chunk, self.H, self.Hkv, self.d, self.page = list(cached), list(chunk), H, Hkv, d, page
        self.dtype, self.causal, self.sumi = dtype, causal, sumi
        self.dt = torch.float32 if dtype == "f32" else torch.bfloat16
        self.scale = d ** -0.5 if scale is None else scale
        B = len(self.cached)
        need = [-(-(c + (0 if sumi else t)) // page) for c, t in zip(cached, chunk)]
        self.n_pages = sum(need) + free
        order = torch.randperm(self.n_pages, generator=g)
        self.table = torch.full((B, max(1, max(need))), -1, dtype=torch.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n].int()
            at += n
        # unused slots hold NaN: nothing may read them
        self.k = torch.full((self.n_pages, Hkv, page, d), math.nan, dtype=self.dt)
        self.v = self.k.clone()
        self.mass = torch.full((self.n_pages, page), math.nan)
        self.stamp = torch.full((self.n_pages, page), -7, dtype=torch.int32)
        for b, n in enumerate(self.cached):
            for j in range(n):
                pg, s = self.at(b, j)
                self.k[pg, :, s] = self.normal(Hkv, d) * std
                self.v[pg, :, s] = self.normal(Hkv, d)
                self.mass[pg, s] = torch.rand(1, generator=g)[0]
                self.stamp[pg, s] = j
        m = sum(chunk) + tail     # rows behind the last sequence
        self.q, self.kn, self.vn = self.normal(m, H, d) * std, self.normal(m, Hkv, d) * std, self.normal(m, Hkv, d)
        self.off = torch.tensor([sum(self.chunk[:b]) for b in range(B + 1)], dtype=torch.int32)
        self.scen = torch.randint(0, n_scen, (m,), generator=g, dtype=torch.int32)
        self.beh = torch.randint(0, n_beh, (m,), generator=g, dtype=torch.int32)
        self.tau = torch.rand(n_scen, n_beh, generator=g) * 1.5 + 0.5
        self.stamp_new = torch.arange(m, dtype=torch.int32) + 1000
        self.m, self.len = m, torch.tensor(self.cached, dtype=torch.int32)

    def normal(self, *shape):
        return torch.randn(*shape, generator=self.g).to(self.dt)

    def at(self, b, j):
        return int(self.table[b, j // self.page]), j % self.page

    def rows(self, pages, b, n):
        """[n, ...] of the first n tokens of b."""
        return torch.stack([pages[pg, :, s] if pages.dim() == 4 else pages[pg, s] for pg, s in (self.at(b, j) for j in range(n))]) \
            if n else pages.new_zeros((0,) + ((pages.shape[1], pages.shape[3]) if pages.dim() == 4 else ()))

    def expect(self):
        """o [m, H, d], its bound, weights {b: [keys]}, their bounds: 64 bits."""
        G, d = self.H // self.Hkv, self.d
        o, tol = torch.zeros(self.m, self.H, d, dtype=torch.float64), torch.zeros(self.m, self.H, d, dtype=torch.float64)
        weight, wtol = {}, {}
        for b, (n, t) in enumerate(zip(self.cached, self.chunk)):
            r = slice(int(self.off[b]), int(self.off[b]) + t)
            ks = torch.cat([self.rows(self.k, b, n), self.kn[r]]).double()
            vs = torch.cat([self.rows(self.v, b, n), self.vn[r]]).double()
            sees = torch.ones(t, n + t, dtype=torch.bool)
            if self.sumi:
                sees[:, n:] = torch.eye(t, dtype=torch.bool)
            elif self.causal:
                sees = sees.tril(diagonal=n)
            c = self.scale / self.tau.double()[self.scen[r].long(), self.beh[r].long()]
            w, wt = torch.zeros(n + t, dtype=torch.float64), torch.zeros(n + t, dtype=torch.float64)
            for h in range(self.H):
                q, k, v = self.q[r, h].double(), ks[:, h // G], vs[:, h // G]
                logits = torch.where(sees, (q @ k.t()) * c[:, None], -math.inf)
                p = torch.where(sees, torch.softmax(logits, dim=1), 0.0)
                # keys that a row does not see have no part in it, whatever they hold
                o[r, h] = torch.stack([p[i, sees[i]] @ v[sees[i]] for i in range(t)]) if t else o[r, h]
                # A logit is off by the roundings of d products and sums, of its scale and of the reference subtracted from it:
                # (d + 4) half steps of sum |q||k| c.  A probability by twice that (its own and the sum's), by the 3 half steps that
                # exp2 and the division have each, and by those of adding n terms.  In bf16 each is also rounded once, as is the
                # output.
                mag = torch.where(sees, (q.abs() @ k.abs().t()) * c[:, None], 0.0)
                worst = torch.nan_to_num(mag, 0, 0, 0).amax(1) if n + t else torch.zeros(t, dtype=torch.float64)
                rel = 2 * (d + 4) * HALF_F32 * worst + (n + t + 12) * HALF_F32
                a = torch.stack([p[i, sees[i]] @ v[sees[i]].abs() for i in range(t)]) if t else o[r, h]
                tol[r, h] = a * rel[:, None] * 1.01 + a * (HALF_BF16 if self.dtype == "bf16" else 0) * 1.01
                tol[r, h] += (o[r, h].abs() + tol[r, h]) * (HALF_BF16 if self.dtype == "bf16" else HALF_F32)
                w += p.sum(0)
                # (a weight below the smallest normal number, 2^-126, may be flushed to 0: a weight in each of t rows)
                wt += t * 2.0 ** -126 + (p * (rel[:, None] + (t * G + 40) * HALF_F32)).sum(0) * 1.01
            weight[b], wtol[b] = w, wt
        return o, tol, weight, wtol


class Device:
    """The case on the GPU, and the calls."""

    def __init__(self, case, mass=False, stamp=False, packed=False, max_len=None, pad_o=0):
        import paper_2502_09888_amd as P
        self.P, self.c = P, case
        dev = "cuda:0"
        self.k, self.v, self.table, self.len = case.k.to(dev), case.v.to(dev), case.table.to(dev), case.len.to(dev)
        self.mass, self.stamp = case.mass.to(dev) if mass else None, case.stamp.to(dev) if stamp else None
        H, Hkv, d, m = case.H, case.Hkv, case.d, case.m
        if packed:
            w = (H + 2 * Hkv) * d
            rows = torch.empty(m, w + 16, dtype=case.dt, device=dev)
            self.q, self.kn, self.vn = (rows[:, a:z].unflatten(1, (-1, d)) for a, z in ((0, H * d), (H * d, (H + Hkv) * d), ((H + Hkv) * d, w)))
            self.q.copy_(case.q), self.kn.copy_(case.kn), self.vn.copy_(case.vn)
        else:
            self.q, self.kn, self.vn = case.q.to(dev), case.kn.to(dev), case.vn.to(dev)
        self.off, self.scen, self.beh, self.tau, self.stamp_new = (x.to(dev) for x in (case.off, case.scen, case.beh, case.tau, case.stamp_new))
        self.o = torch.full((m, H * d + pad_o), 77.0, dtype=case.dt, device=dev)[:, :H * d]
        self.max_len = max_len or max(1, max(c + (0 if case.sumi else t) for c, t in zip(case.cached, case.chunk)))
        self.cfg = P.Config(n_heads=H, d_head=d, n_scen=case.tau.shape[0], n_beh=case.tau.shape[1], dtype=P.F32 if case.dtype == "f32" else P.BF16,
                            flags=P.HIST_CAUSAL if case.causal else 0, qk_scale=case.scale)
        self.m_max = max(case.chunk)
        self.describe()

    def describe(self):
        P = self.P
        self.kv = P.paged_kv(self.k, self.v, self.table, self.len, self.max_len, mass=self.mass, stamp=self.stamp)
        self.ws = torch.full((max(256, P.climber_paged_workspace_bytes(self.cfg, self.kv, self.c.m, self.m_max)),), 0xFF, dtype=torch.uint8, device="cuda:0")

    def history(self, stream=None):
        self.P.climber_attn_history_paged(self.cfg, self.tau, self.kv, self.q, self.kn, self.vn, self.off, self.c.m, self.m_max, self.scen, self.beh,
                                          self.stamp_new if self.stamp is not None else None, self.o, self.ws, stream)

    def sumi(self, stream=None):
        self.P.climber_attn_sumi_paged(self.cfg, self.tau, self.kv, self.q, self.kn, self.vn, self.off, self.c.m, self.m_max, self.scen, self.beh,
                                       self.o, self.ws, stream)

    def attend(self, stream=None):
        (self.sumi if self.c.sumi else self.history)(stream)

    def out(self):
        torch.cuda.synchronize()
        return self.o.double().cpu().view(self.c.m, self.c.H, self.c.d)


def evict_ref(table, page, n, budget, rank, stamp=None, keep_from=None):
    """Per sequence (new length, src list): ranks by (protected, rank, slot)."""
    out = []
    for b in range(len(n)):
        at = [(int(table[b, j // page]), j % page) for j in range(n[b])]
        keep = min(max(int(budget[b]), 0), n[b])

        def key(j):
            r = float(rank[at[j]])
            first = keep_from is not None and int(stamp[at[j]]) >= int(keep_from[b])
            return (not first, r != r, -r if r == r else 0.0, j)

        kept = set(sorted(range(n[b]), key=key)[:keep])
        src = list(range(keep))
        for hole, mover in zip([j for j in range(keep) if j not in kept], [j for j in range(keep, n[b]) if j in kept]):
            src[hole] = mover
        out.append((keep, src))
    return out
