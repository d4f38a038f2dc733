"""Performance cases of the paged history cache: what a server that keeps users' histories in pages does between two
encodes of them.

A case is a dict of plain values.  `path` selects the call:

  history  a chunk of new behaviours per user is stored into the user's pages and attends to the cached history and to itself
           (`causal`: to itself up to each row); `cached` = 0 makes it whole histories ("prompts") of different lengths
  score    candidates attend to the cached history and to themselves
  evict    each user's cache is cut to `budget` tokens by accumulated attention weight

`users` sequences; `cached` / `chunk`: tokens in the cache and new rows of the longest user, *_min those of the shortest.  `heads`
query heads share `kv_heads` heads of the cache.  `mass`: attention weights are accumulated per cached token.  `packed`: the
rows are columns of one q | k | v matrix, as a projection writes them.  Lengths follow from `layout` and so belong to the case; tensor
contents and the order of the pages follow from the seed.
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
N_SCEN, N_BEH = 8, 4   # scenarios x behaviours of the temperature table


def _attention(name, path, users, cached, chunk, heads, kv_heads, d_head, page, *, cached_min=None, chunk_min=None, dtype="bf16",
               causal=False, mass=False, packed=False, layout=0):
    return dict(name=name, path=path, dtype=dtype, users=users, cached=cached, cached_min=cached if cached_min is None else cached_min,
                chunk=chunk, chunk_min=chunk if chunk_min is None else chunk_min, heads=heads, kv_heads=kv_heads, d_head=d_head,
                page=page, causal=causal, mass=mass, packed=packed, layout=layout)


def _evict(name, users, cached, budget, kv_heads, d_head, page, *, cached_min=None, dtype="bf16", recent=0, layout=0):
    return dict(name=name, path="evict", dtype=dtype, users=users, cached=cached, cached_min=cached if cached_min is None else cached_min,
                budget=budget, kv_heads=kv_heads, d_head=d_head, page=page, recent=recent, layout=layout)


def listed():
    return [
        # The smallest call: one user of the small fp32 configuration does one thing.
        _attention("one behaviour, fp32", "history", 1, 64, 1, 2, 2, 32, 16, dtype="f32"),
        # 64 users do one thing each, histories of 500 to 4000: a decode step, bound by reading the cache once.
        _attention("one token of 64", "history", 64, 4000, 1, 32, 8, 128, 64, cached_min=500, causal=True, layout=1),
        # One lifelong history, one new token: its keys have to be shared out over the whole card.
        _attention("one token, long cache", "history", 1, 98765, 1, 32, 8, 128, 256, causal=True),
        # Sessions of 60 to 500 behaviours join histories of 1000 to 4000, weights accumulated for a later eviction.
        _attention("sessions, weights", "history", 8, 4000, 500, 32, 8, 128, 64, cached_min=1000, chunk_min=60, causal=True, mass=True,
                   layout=2),
        # Whole histories, new to the cache, of very different lengths.
        _attention("whole histories", "history", 3, 0, 6000, 32, 8, 128, 64, chunk_min=1500, causal=True, packed=True, layout=3),
        # The reference precision: a few users' sessions, each seen as a whole.
        _attention("sessions, fp32", "history", 4, 1000, 130, 8, 4, 64, 32, cached_min=300, chunk_min=37, dtype="f32", layout=4),
        # The benchmark's candidate pass (64 users, histories of 1024, 512 candidates each, 8 heads of 64) from pages.
        _attention("scoring", "score", 64, 1024, 512, 8, 8, 64, 128),
        # Heavy users with grouped heads and very different lengths, weights accumulated.
        _attention("scoring, ragged, weights", "score", 16, 4096, 1024, 8, 2, 64, 16, cached_min=512, chunk_min=256, mass=True, layout=5),
        # One request's candidates: latency.
        _attention("scoring of one user", "score", 1, 1000, 128, 8, 8, 64, 64),
        # A nightly cut of many histories to half, the last 256 behaviours kept.
        _evict("cut to half", 64, 4096, 2048, 8, 128, 64, cached_min=1500, recent=256, layout=6),
        # A full cache that takes one token and gives one up, every step.
        _evict("one out", 32, 1025, 1024, 8, 64, 64, recent=64),
        # A lifelong history cut to half.
        _evict("long cache to half", 1, 98765, 50000, 8, 128, 256, recent=1000),
    ]


def _log(rng, lo, hi):
    """An integer whose logarithm is uniform over [lo, hi]."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        path, f32, layout, ragged = rng.choice(["step", "history", "prompt", "score", "evict"]), rng.random() < 0.2, rng.randrange(1 << 20), rng.random() < 0.6
        page, kv_heads, d_head = 16 << rng.randint(0, 4), rng.choice([1, 2, 4, 8]), rng.choice([32, 64, 128] if f32 else [64, 128])
        heads, dtype = kv_heads * rng.choice([1, 2, 4, 5, 8]), "f32" if f32 else "bf16"
        cached = _log(rng, 1, 4096 if f32 else 65536)
        if path == "evict":
            case = _evict("", _log(rng, 1, 64), cached, max(1, int(cached * rng.uniform(0.3, 1.1))), kv_heads, d_head, page,
                          cached_min=max(1, cached // 4) if ragged else None, dtype=dtype, recent=rng.choice([0, cached // 16]), layout=layout)
        else:
            if path == "prompt":
                cached = 0
            chunk = rng.randint(1, 4) if path == "step" else _log(rng, 2, 256 if f32 else 4096)
            case = _attention("", "score" if path == "score" else "history", _log(rng, 1, 64), cached, chunk, heads, kv_heads, d_head, page,
                              cached_min=cached // 4 if ragged else None, chunk_min=max(1, chunk // 4) if ragged else None, dtype=dtype,
                              causal=rng.random() < 0.7, mass=rng.random() < 0.4, packed=rng.random() < 0.3, layout=layout)
        del case["name"]
        # no more than the largest listed cases: whole histories; a tenth of that in fp32; logits of the plain form in memory
        w, n = work(case), case["cached"] + case.get("chunk", 0)
        if w["flops"] > (1e10 if f32 else 4e11) or w["bytes"] > 1.5e9 or case["users"] * n * kv_heads * d_head > 3e8:
            continue
        if case["users"] * case.get("heads", 1) * case.get("chunk", 1) * n > 2.5e9:
            continue
        return case


def _lengths(case, what):
    hi, lo = case[what], case[what + "_min"]
    rng = random.Random("%s %d" % (what, case["layout"]))
    ls = [rng.randint(lo, hi) for _ in range(case["users"])]
    ls[0] = hi
    if len(ls) > 1:
        ls[-1] = lo
    return ls


def _pages(case, g, tokens):
    """A cache whose users have the tokens' pages in any order, and one page in eight free: (table, pages)."""
    P = case["page"]
    need = [-(-t // P) for t in tokens]
    total = sum(need)
    pages = total + total // 8 + 1
    order = torch.randperm(pages, generator=g, device=DEV)
    width = max(1, max(need))
    start = torch.tensor([sum(need[:b]) for b in range(len(need))], device=DEV)
    col = torch.arange(width, device=DEV)
    has = col < torch.tensor(need, device=DEV)[:, None]
    table = torch.where(has, order[(start[:, None] + col).clamp(max=pages - 1)], -1)
    return table.to(torch.int32), pages


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    B, P, Hkv, D = case["users"], case["page"], case["kv_heads"], case["d_head"]
    cached, chunk = _lengths(case, "cached"), [0] * B
    s = {"case": case}
    if case["path"] != "evict":
        chunk = _lengths(case, "chunk")
    appends = case["path"] == "history"
    table, n_pages = _pages(case, g, [c + (t if appends else 0) for c, t in zip(cached, chunk)])

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV, dtype=dt)

    def ids(n, hi):
        return torch.randint(0, hi, (n,), generator=g, device=DEV, dtype=torch.int32)

    s["table"], s["len"] = table, torch.tensor(cached, dtype=torch.int32, device=DEV)
    s["k_pages"], s["v_pages"] = normal(n_pages, Hkv, P, D), normal(n_pages, Hkv, P, D)
    s["mass"] = s["stamp"] = None
    if case["path"] == "evict":
        # weights as they accumulate: a few tokens hold most of it, and some none
        w = torch.exp(2 * torch.randn((n_pages, P), generator=g, device=DEV))
        s["rank"] = torch.where(torch.rand((n_pages, P), generator=g, device=DEV) < 0.02, 0.0, w)
        s["mass"] = s["rank"].clone()
        slot = torch.arange(table.shape[1] * P, device=DEV)
        stamp = torch.zeros((n_pages + 1, P), dtype=torch.int32, device=DEV)
        stamp[table.long()] = (1000 + slot).to(torch.int32).view(1, -1, P).expand(B, -1, -1)
        s["stamp"] = stamp[:n_pages].contiguous()
        s["budget"] = torch.tensor([case["budget"]] * B, dtype=torch.int32, device=DEV)
        s["keep_from"] = s["len"] + (1000 - case["recent"]) if case["recent"] else None
        s["len_out"], s["src"] = torch.empty_like(s["len"]), torch.empty((B, table.shape[1] * P), dtype=torch.int32, device=DEV)
        s["longest"] = case["cached"]
    else:
        H, m = case["heads"], sum(chunk)
        if case["packed"]:
            rows = normal(m, (H + 2 * Hkv) * D)
            q, k, v = rows.split([H * D, Hkv * D, Hkv * D], dim=1)
            s["q"], s["k"], s["v"] = q.unflatten(1, (H, D)), k.unflatten(1, (Hkv, D)), v.unflatten(1, (Hkv, D))
        else:
            s["q"], s["k"], s["v"] = normal(m, H, D), normal(m, Hkv, D), normal(m, Hkv, D)
        s["off"] = torch.tensor([sum(chunk[:b]) for b in range(B + 1)], dtype=torch.int32, device=DEV)
        s["scen"], s["beh"] = ids(m, N_SCEN), ids(m, N_BEH)
        s["tau"] = torch.rand((N_SCEN, N_BEH), generator=g, device=DEV) * 1.5 + 0.5
        s["o"] = torch.empty((m, H * D), dtype=dt, device=DEV)
        s["m_total"], s["m_max"] = m, max(chunk)
        s["longest"] = max(c + (t if appends else 0) for c, t in zip(cached, chunk))
        if case["mass"]:
            s["mass"] = torch.rand((n_pages, P), generator=g, device=DEV)
    if own:
        import paper_2502_09888_amd as C
        H = case.get("heads", Hkv)
        s["cfg"] = C.Config(n_heads=H, d_head=D, n_scen=N_SCEN, n_beh=N_BEH, dtype=C.F32 if case["dtype"] == "f32" else C.BF16,
                            flags=C.HIST_CAUSAL if case.get("causal") else 0, qk_scale=D ** -0.5)
        s["kv"] = C.paged_kv(s["k_pages"], s["v_pages"], s["table"], s["len"], s["longest"], mass=s["mass"], stamp=s["stamp"])
        s["ws"] = torch.empty(C.climber_paged_workspace_bytes(s["cfg"], s["kv"], s.get("m_total", 0), s.get("m_max", 0)),
                              dtype=torch.uint8, device=DEV)
    return s


def run(s):
    case = s["case"]
    if own:
        import paper_2502_09888_amd as C
        if case["path"] == "evict":
            C.climber_paged_evict(s["cfg"], s["kv"], s["rank"], s["budget"], s["keep_from"], s["len_out"], s["src"], s["ws"])
            return {"len": s["len_out"], "src": s["src"], "k": s["k_pages"], "v": s["v_pages"], "mass": s["mass"], "stamp": s["stamp"]}
        if case["path"] == "history":
            C.climber_attn_history_paged(s["cfg"], s["tau"], s["kv"], s["q"], s["k"], s["v"], s["off"], s["m_total"], s["m_max"],
                                         s["scen"], s["beh"], None, s["o"], s["ws"])
            return {"o": s["o"], "k": s["k_pages"], "v": s["v_pages"], "mass": s["mass"]}
        C.climber_attn_sumi_paged(s["cfg"], s["tau"], s["kv"], s["q"], s["k"], s["v"], s["off"], s["m_total"], s["m_max"],
                                  s["scen"], s["beh"], s["o"], s["ws"])
        return {"o": s["o"], "mass": s["mass"]}
    return _plain_evict(s) if case["path"] == "evict" else _plain_attention(s)


def _plain_attention(s):
    """Attention over the gathered cache in 32 bits: users padded to the longest."""
    case, m = s["case"], s["m_total"]
    B, P, Hkv, D, H = case["users"], case["page"], case["kv_heads"], case["d_head"], case["heads"]
    G, T, L = H // Hkv, case["chunk"], case["cached"]
    n, off, table = s["len"].long(), s["off"].long(), s["table"].long().clamp(min=0)
    row = torch.arange(m, device=DEV)
    seq = torch.searchsorted(off, row, right=True) - 1
    t = row - off[seq]
    if case["path"] == "history":
        at = n[seq] + t
        page = table[seq, at // P]
        s["k_pages"][page, :, at % P] = s["k"]
        s["v_pages"][page, :, at % P] = s["v"]
    slot = torch.arange(L, device=DEV)
    page = table[:, slot // P]                                                     # [B, L]
    K = s["k_pages"][page, :, slot % P].float().permute(0, 2, 1, 3)                # [B, Hkv, L, D]
    V = s["v_pages"][page, :, slot % P].float().permute(0, 2, 1, 3)
    pick = (off[:-1, None] + torch.arange(T, device=DEV)).clamp(max=m - 1)         # [B, T]
    counts = off[1:] - off[:-1]
    q = s["q"][pick].float().view(B, T, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * T, D)
    kn, vn = s["k"][pick].float().permute(0, 2, 1, 3), s["v"][pick].float().permute(0, 2, 1, 3)   # [B, Hkv, T, D]
    scale = D ** -0.5 / s["tau"][s["scen"].long(), s["beh"].long()][pick]          # [B, T]
    scale = scale[:, None, None, :].expand(B, Hkv, G, T).reshape(B, Hkv, G * T, 1)
    R = torch.matmul(q, K.transpose(2, 3).contiguous())                            # [B, Hkv, G T, L]
    R = R.masked_fill((slot >= n[:, None])[:, None, None, :], -math.inf)
    col = torch.arange(T, device=DEV)
    if case["path"] == "history":
        N = torch.matmul(q, kn.transpose(2, 3).contiguous())                       # [B, Hkv, G T, T]
        hidden = (col >= counts[:, None])[:, None, None, :]
        if case["causal"]:
            hidden = hidden | (col[None, :] > col[:, None]).repeat(G, 1)
        N = N.masked_fill(hidden & (col != col.repeat(G)[:, None]), -math.inf)     # (a padding row sees itself)
    else:
        N = (q.view(B, Hkv, G, T, D) * kn[:, :, None]).sum(-1).view(B, Hkv, G * T, 1)
    A = torch.cat([R, N], dim=3) * scale
    del R, N
    A = torch.exp(A - A.amax(dim=3, keepdim=True))
    A = A / A.sum(dim=3, keepdim=True)
    new = A[..., L:]
    o = torch.matmul(A[..., :L], V)
    if case["path"] == "history":
        o = o + torch.matmul(new, vn)
    else:
        o = (o.view(B, Hkv, G, T, D) + new.view(B, Hkv, G, T, 1) * vn[:, :, None]).view(B, Hkv, G * T, D)
    o = o.view(B, Hkv, G, T, D).permute(0, 3, 1, 2, 4).reshape(B, T, H * D)
    out = {"o": o[seq, t].to(s["o"].dtype)}
    if case["path"] == "history":
        out["k"], out["v"] = s["k_pages"], s["v_pages"]
    out["mass"] = s["mass"]
    if case["mass"]:
        valid = (col < counts[:, None])[:, None, None, :].expand(B, Hkv, G, T).reshape(B, Hkv, G * T, 1)
        w = (A * valid).sum(dim=(1, 2))                                            # [B, L + T or 1]
        flat, none = s["mass"].view(-1), s["mass"].numel()
        add = torch.cat([flat, flat.new_zeros(1)])
        where = torch.where(slot < n[:, None], page * P + slot % P, none)
        add[where] = add[where] + w[:, :L]
        if case["path"] == "history":
            at = n[seq] + t
            add[table[seq, at // P] * P + at % P] = w[seq, L + t]
        flat.copy_(add[:-1])
    return out


def _plain_evict(s):
    """The kept tokens by three stable sorts; the kept tokens behind the cut go, in order, into the places before it that are free."""
    case = s["case"]
    B, P = case["users"], case["page"]
    n, table = s["len"].long(), s["table"].long().clamp(min=0)
    L = table.shape[1] * P
    slot = torch.arange(L, device=DEV)
    page, inside = table[:, slot // P], slot % P
    valid = slot < n[:, None]
    keep = torch.minimum(s["budget"].long().clamp(min=0), n)
    rank = s["rank"][page, inside]
    first = s["stamp"][page, inside] >= s["keep_from"][:, None] if s["keep_from"] is not None else torch.zeros_like(valid)
    order = torch.sort(rank, dim=1, descending=True, stable=True).indices
    order = order.gather(1, torch.sort(first.gather(1, order).int(), dim=1, descending=True, stable=True).indices)
    order = order.gather(1, torch.sort(valid.gather(1, order).int(), dim=1, descending=True, stable=True).indices)
    kept = torch.zeros_like(valid).scatter(1, order, slot < keep[:, None])
    front = slot < keep[:, None]
    hole, mover = torch.nonzero(front & ~kept, as_tuple=True), torch.nonzero(kept & ~front, as_tuple=True)
    src = torch.where(front, slot, -1)
    src[hole] = mover[1]
    to_page, to_in, from_page, from_in = page[hole], inside[hole[1]], page[mover], inside[mover[1]]
    for name in ("k_pages", "v_pages"):
        s[name][to_page, :, to_in] = s[name][from_page, :, from_in]
    for name in ("mass", "stamp"):
        s[name][to_page, to_in] = s[name][from_page, from_in]
    return {"len": keep.to(torch.int32), "src": src.to(torch.int32), "k": s["k_pages"], "v": s["v_pages"], "mass": s["mass"],
            "stamp": s["stamp"]}


def _pairs(case):
    """Pairs of a row and a key that it sees."""
    pairs = 0
    for n, t in zip(_lengths(case, "cached"), _lengths(case, "chunk")):
        pairs += t * (n + 1) if case["path"] == "score" else t * n + (t * (t + 1) // 2 if case["causal"] else t * t)
    return pairs


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    row = 2 * case["kv_heads"] * case["d_head"] * e            # a token's key and value
    cached = _lengths(case, "cached")
    if case["path"] == "evict":
        moved = 0.0
        for n in cached:
            keep = min(case["budget"], n)
            recent = min(case["recent"], keep)                 # kept whatever they weigh, at the end
            behind = n - keep
            moved += min(recent, behind) + (max(0, behind - recent) * (keep - recent) / (n - recent) if n > recent else 0)
        return {"bytes": sum(cached) * 8 + moved * (2 * row + 16) + 8 * sum(min(case["budget"], n) for n in cached), "flops": 2 * sum(cached)}
    m, wide = sum(_lengths(case, "chunk")), case["heads"] * case["d_head"]
    total = m * (2 * wide * e + row + 8) + sum(cached) * row
    if case["path"] == "history":
        total += m * row
    if case["mass"]:
        total += 8 * (sum(cached) + (m if case["path"] == "history" else 0))
    return {"bytes": total, "flops": 4 * wide * _pairs(case)}


def exact(case, seed):
    """From the definition, in 64 bits, one user and one head of the cache after the other."""
    if case["path"] == "evict":
        return None                                            # nothing is computed: what is kept and where it lies has to be equal
    s = prepare(case, seed)
    P, D, G = case["page"], case["d_head"], case["heads"] // case["kv_heads"]
    out = torch.zeros(s["o"].shape, dtype=torch.float64, device=DEV).view(-1, case["heads"], D)
    mass = s["mass"].double() if case["mass"] else None
    r0 = 0
    for b, (n, t) in enumerate(zip(_lengths(case, "cached"), _lengths(case, "chunk"))):
        rows = slice(r0, r0 + t)
        r0 += t
        pages = s["table"][b, :-(-n // P)].long()
        tau = s["tau"].double()[s["scen"][rows].long(), s["beh"][rows].long()]
        weight = torch.zeros(n + t, dtype=torch.float64, device=DEV)
        for h in range(case["kv_heads"]):
            own_k, own_v = s["k"][rows, h].double(), s["v"][rows, h].double()
            keys = torch.cat([s["k_pages"][pages, h].double().view(-1, D)[:n], own_k])
            values = torch.cat([s["v_pages"][pages, h].double().view(-1, D)[:n], own_v])
            sees = torch.ones(t, n + t, dtype=torch.bool, device=DEV)
            if case["path"] == "score":
                sees[:, n:] = torch.eye(t, dtype=torch.bool, device=DEV)
            elif case["causal"]:
                sees = sees.tril(diagonal=n)
            for j in range(G):
                logits = s["q"][rows, h * G + j].double() @ keys.t() / math.sqrt(D) / tau[:, None]
                p = torch.softmax(torch.where(sees, logits, -math.inf), dim=1)
                out[rows, h * G + j] = p @ values
                weight += p.sum(0)
        if mass is not None:
            slots = torch.arange(n + t if case["path"] == "history" else n, device=DEV)
            pages = s["table"][b].long()[slots // P]
            before = torch.where(slots < n, mass[pages, slots % P], 0)
            mass[pages, slots % P] = before + weight[:slots.numel()]
    answer = {"o": out.view(s["o"].shape), "mass": mass}
    return answer if case["path"] == "score" else answer | {"k": None, "v": None}
