"""Performance cases of what keeps many users' histories in pages in 8 bits: the attention over such a cache, the pages themselves, and
the positions that rows are given before they go into it.

A case is a dict of plain values.  `path` selects what a pass does:

  history  a chunk of new behaviours per user attends to the cached history (8 bits, a scale for 16 tokens and head) and to itself
           (`causal`: to itself up to each row), and is stored
  score    candidates attend to the cached history and to themselves
  branch   every user's history is forked into `branches` rows of the page table, which take `rows` new behaviours each: pages are
           shared, handed out, and the shared ones that would be written are copied
  compact  half of the users leave, the others' pages are moved to the front of the pool, and as many new users get pages
  rotary   q and k rows are turned by their positions

`users` sequences; `cached` / `chunk`: tokens in the cache and new rows of the longest user, *_min those of the shortest.  `heads`
query heads share `kv_heads` heads of the cache.  `packed`: the rows are columns of one q | k | v matrix, as a projection writes
them.  Lengths follow from `layout` and so belong to the case; contents and the order of the pages follow from the seed.
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
N_SCEN, N_BEH = 8, 4   # scenarios x behaviours of the temperature table
BLOCK, LEAST = 16, 10  # tokens of a scale; the least scale, as it is stored: 2^(10 - 127)


def _attention(name, path, users, cached, chunk, heads, kv_heads, d_head, page, *, cached_min=None, chunk_min=None, causal=False, packed=False,
               layout=0):
    return dict(name=name, path=path, users=users, cached=cached, cached_min=cached if cached_min is None else cached_min, chunk=chunk,
                chunk_min=chunk if chunk_min is None else chunk_min, heads=heads, kv_heads=kv_heads, d_head=d_head, page=page, causal=causal,
                packed=packed, layout=layout)


def _branch(name, users, cached, branches, rows, kv_heads, d_head, page, dtype, *, cached_min=None, layout=0):
    return dict(name=name, path="branch", users=users, cached=cached, cached_min=cached if cached_min is None else cached_min, branches=branches,
                rows=rows, kv_heads=kv_heads, d_head=d_head, page=page, dtype=dtype, layout=layout)


def _compact(name, users, cached, kv_heads, d_head, page, dtype, *, cached_min=None, layout=0):
    return dict(name=name, path="compact", users=users, cached=cached, cached_min=cached if cached_min is None else cached_min,
                kv_heads=kv_heads, d_head=d_head, page=page, dtype=dtype, layout=layout)


def _rotary(name, rows, heads, kv_heads, d_head, rot, dtype, *, interleaved=False, scaling="none", factor=1.0, inverse=False, packed=False,
            far=0):
    return dict(name=name, path="rotary", rows=rows, heads=heads, kv_heads=kv_heads, d_head=d_head, rot=rot, dtype=dtype, interleaved=interleaved,
                scaling=scaling, factor=factor, inverse=inverse, packed=packed, far=far)


def listed():
    return [
        # The smallest call: one user with a short history does one thing.
        _attention("one behaviour, 8 bits", "history", 1, 70, 1, 2, 2, 64, 16, causal=True),
        # 64 users do one thing each, histories of 500 to 4000: a decode step, bound by reading the cache once.
        _attention("one token of 64, 8 bits", "history", 64, 4000, 1, 32, 8, 128, 64, cached_min=500, causal=True, layout=1),
        # One lifelong history, one new token: its keys have to be shared out over the whole card.
        _attention("one token, long, 8 bits", "history", 1, 98765, 1, 32, 8, 128, 256, causal=True),
        # Sessions of 60 to 500 behaviours join histories of 1000 to 4000.
        _attention("sessions, 8 bits", "history", 8, 4000, 500, 32, 8, 128, 64, cached_min=1000, chunk_min=60, causal=True, packed=True, layout=2),
        # The benchmark's candidate pass (64 users, histories of 1024, 512 candidates each, 8 heads of 64) from pages in 8 bits.
        _attention("scoring, 8 bits", "score", 64, 1024, 512, 8, 8, 64, 128),
        # Heavy users with grouped heads and very different lengths.
        _attention("scoring, ragged, 8 bits", "score", 16, 4096, 1024, 8, 2, 128, 16, cached_min=512, chunk_min=256, layout=5),
        # One user tries one continuation: what the page calls cost by themselves.
        _branch("one branch", 1, 40, 1, 1, 2, 64, 16, "bf16"),
        # 32 users' histories, four continuations each of a session's length.
        _branch("four branches of 32", 32, 4000, 4, 100, 8, 128, 64, "e4m3", cached_min=500, layout=3),
        # Half of the users leave a pool of 256 users, and their places are filled.
        _compact("half of 256 leave", 256, 2000, 8, 128, 64, "e4m3", cached_min=100, layout=4),
        # The rows of a decode step of 64 users.
        _rotary("positions of 64 rows", 64, 32, 8, 128, 128, "bf16", packed=True, far=100000),
        # Whole histories, positions far beyond the lengths that the model was made for.
        _rotary("positions of 20000 rows", 20000, 32, 8, 128, 128, "bf16", scaling="parts", factor=16.0, far=500000),
        # The gradient, in the reference precision, of neighbours turned in a part of the head.
        _rotary("gradient, fp32, part", 5000, 8, 4, 64, 48, "f32", interleaved=True, scaling="linear", factor=4.0, inverse=True),
    ]


def _log(rng, lo, hi):
    """An integer whose logarithm is uniform over [lo, hi]."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        path, layout, ragged = rng.choice(["step", "history", "score", "branch", "compact", "rotary"]), rng.randrange(1 << 20), rng.random() < 0.6
        page, kv_heads, d_head, dtype = 16 << rng.randint(0, 4), rng.choice([1, 2, 4, 8]), rng.choice([64, 128]), rng.choice(["bf16", "f32", "e4m3"])
        heads = kv_heads * rng.choice([1, 2, 4, 5, 8])
        if path == "rotary":
            if dtype == "e4m3":
                dtype = "bf16"
            d_head = rng.choice([32, 64, 80, 128, 256])
            rot = d_head if rng.random() < 0.5 else 2 * rng.randint(1, d_head // 2)
            case = _rotary("", _log(rng, 1, 20000), heads, kv_heads, d_head, rot, dtype, interleaved=rng.random() < 0.5,
                           scaling=rng.choice(["none", "linear", "base", "parts"]) if rot > 2 else "none", factor=rng.choice([2.0, 4.0, 10.0, 32.0]),
                           inverse=rng.random() < 0.3, packed=rng.random() < 0.4, far=rng.choice([0, 5000, 1000000]))
        elif path == "branch":
            cached = _log(rng, 1, 16384)
            case = _branch("", _log(rng, 1, 64), cached, rng.randint(1, 5), _log(rng, 1, 300), kv_heads, d_head, page, dtype,
                           cached_min=max(1, cached // 4) if ragged else None, layout=layout)
        elif path == "compact":
            cached = _log(rng, 16, 16384)
            case = _compact("", 2 * _log(rng, 1, 128), cached, kv_heads, d_head, page, dtype, cached_min=max(1, cached // 4) if ragged else None,
                            layout=layout)
        else:
            cached = _log(rng, 1, 65536)
            chunk = rng.randint(1, 4) if path == "step" else _log(rng, 2, 2048)
            case = _attention("", "score" if path == "score" else "history", _log(rng, 1, 64), cached, chunk, heads, kv_heads, d_head, page,
                              cached_min=cached // 4 if ragged else None, chunk_min=max(1, chunk // 4) if ragged else None,
                              causal=rng.random() < 0.7, packed=rng.random() < 0.3, layout=layout)
        del case["name"]
        # no more than the largest listed cases: ragged scoring, the token of 64 users, the pool of 256
        w = work(case)
        if w["flops"] > 1e11 or w["bytes"] > 5.5e8:
            continue
        if path in ("branch", "compact"):
            # the pool in memory: every user's tokens and, for each branch, a session more
            tokens = case["users"] * (case["cached"] + page) + case["users"] * case.get("branches", 0) * (case.get("rows", 0) + 2 * page)
            if tokens * kv_heads * d_head * (4 if dtype == "f32" else 2 if dtype == "bf16" else 1) > 4e8:
                continue
        if path in ("step", "history", "score"):
            n = case["cached"] + case["chunk"]
            if case["users"] * n * kv_heads * d_head > 3e8 or case["users"] * heads * case["chunk"] * n > 1.5e9:
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


# ---- inputs --------------------------------------------------------------------------------------
def _pages(g, need, pages):
    """The table of users that have `need` pages each, in any order."""
    order = torch.randperm(pages, generator=g, device=DEV)
    width = max(1, max(need))
    start = torch.tensor([sum(need[:b]) for b in range(len(need))], device=DEV)
    col = torch.arange(width, device=DEV)
    has = col < torch.tensor(need, device=DEV)[:, None]
    return torch.where(has, order[(start[:, None] + col).clamp(max=pages - 1)], -1).to(torch.int32)


def _scale_of(amax):
    """The stored scale, 127 + s: the least s from -117 on with amax <= 448 2^s."""
    f, x = torch.frexp(amax)
    s = x - 9 + (f > 0.875).int()
    return torch.where(amax > 0, s + 127, LEAST).clamp(min=LEAST)


def _two_to(e):
    """2^e in 32 bits, for whole numbers e from -126 to 127."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _filled(g, n_pages, kv_heads, page, d):
    """Pages in 8 bits and their scales, from normal values with a factor of its own for every head."""
    codes = torch.empty((n_pages, kv_heads, page, d), dtype=torch.uint8, device=DEV)
    scale = torch.empty((n_pages, kv_heads, page // BLOCK), dtype=torch.uint8, device=DEV)
    factor = torch.exp(0.5 * torch.randn((kv_heads, 1, 1), generator=g, device=DEV))
    for at in range(0, n_pages, 1024):
        n = min(1024, n_pages - at)
        x = (torch.randn((n, kv_heads, page, d), generator=g, device=DEV) * factor).view(n, kv_heads, page // BLOCK, BLOCK * d)
        s = _scale_of(x.abs().amax(-1))
        codes[at:at + n] = (x * _two_to(127 - s)[..., None]).to(torch.float8_e4m3fn).view(torch.uint8).view(n, kv_heads, page, d)
        scale[at:at + n] = s.to(torch.uint8)
    return codes, scale


def _held(codes):
    return codes.view(torch.float8_e4m3fn)


def _pool(case, g, n_pages, s):
    Hkv, P, D = case["kv_heads"], case["page"], case["d_head"]
    if case.get("dtype", "e4m3") == "e4m3":
        s["k_pages"], s["k_scale"] = _filled(g, n_pages, Hkv, P, D)
        s["v_pages"], s["v_scale"] = _filled(g, n_pages, Hkv, P, D)
    else:
        dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
        s["k_pages"] = torch.randn((n_pages, Hkv, P, D), generator=g, device=DEV, dtype=dt)
        s["v_pages"] = torch.randn((n_pages, Hkv, P, D), generator=g, device=DEV, dtype=dt)


def _frequencies(case):
    """Radians per position of each pair, in 64 bits, and what the turned values are multiplied by."""
    rot, factor, base, made_for = case["rot"], case["factor"], 10000.0, 4096.0
    i = torch.arange(rot // 2, dtype=torch.float64, device=DEV)
    scale = 1.0
    if case["scaling"] == "base":      # a larger base: the slowest pair by the factor, the fastest not at all
        base *= factor ** (rot / (rot - 2))
    f = base ** (-2 * i / rot)
    if case["scaling"] == "linear":
        f = f / factor
    if case["scaling"] == "parts":     # pairs with few turns within the length by the factor, those with many not at all
        r = ((made_for * f / (2 * math.pi) - 1) / (32 - 1)).clamp(0, 1)
        f = f * r + f / factor * (1 - r)
        scale = 0.1 * math.log(factor) + 1
    return f, scale


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    s = {"case": case}
    if own:
        import paper_2502_09888_amd as C
    if case["path"] == "rotary":
        H, Hkv, D, m = case["heads"], case["kv_heads"], case["d_head"], case["rows"]
        dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
        if case["packed"]:
            s["rows"] = torch.randn((m, (H + 2 * Hkv) * D), generator=g, device=DEV, dtype=dt)
            q, k, _ = s["rows"].split([H * D, Hkv * D, Hkv * D], dim=1)
            s["q"], s["k"] = q.unflatten(1, (H, D)), k.unflatten(1, (Hkv, D))
        else:
            s["q"], s["k"] = (torch.randn((m, h, D), generator=g, device=DEV, dtype=dt) for h in (H, Hkv))
        s["pos"] = (torch.arange(m, device=DEV) % 4000 + torch.randint(0, case["far"] + 1, (m,), generator=g, device=DEV)).to(torch.int32)
        s["q_out"], s["k_out"] = torch.empty((m, H, D), dtype=dt, device=DEV), torch.empty((m, Hkv, D), dtype=dt, device=DEV)
        s["freq"], s["mul"] = _frequencies(case)
        if own:
            s["cfg"] = C.Config(n_heads=H, d_head=D, dtype=C.F32 if case["dtype"] == "f32" else C.BF16)
            kind = {"none": C.ROTARY_PLAIN, "linear": C.ROTARY_LINEAR, "base": C.ROTARY_BASE, "parts": C.ROTARY_PARTS}[case["scaling"]]
            freq, mul = C.climber_rotary_frequencies(case["rot"], 10000.0, kind, case["factor"], 4096.0, 32.0, 1.0)
            s["freq"] = torch.tensor(freq, dtype=torch.float64, device=DEV)
            s["rot"] = C.rotary(s["freq"], case["rot"], interleaved=case["interleaved"], scale=mul, inverse=case["inverse"])
        return s
    B, P, Hkv, D = case["users"], case["page"], case["kv_heads"], case["d_head"]
    cached = _lengths(case, "cached")
    if case["path"] in ("branch", "compact"):
        need = [-(-c // P) for c in cached]
        F, rows = case.get("branches", 0), case.get("rows", 0)
        more = sum(F * (-(-(c + rows) // P) - c // P) for c in cached)
        n_pages = sum(need) + more + sum(need) // 8 + 1
        n_seqs, width = B * (1 + F), max(-(-(c + rows) // P) for c in cached)
        table = torch.full((n_seqs, width), -1, dtype=torch.int32, device=DEV)
        table[:B, :max(need)] = _pages(g, need, n_pages)
        held = torch.tensor(need + [0] * (B * F), dtype=torch.int32, device=DEV)
        refs = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
        refs[table[table >= 0].long()] = 1
        s["table"], s["held"], s["refs"] = table, held, refs
        s["len"] = torch.tensor(cached + [0] * (B * F), dtype=torch.int32, device=DEV)
        _pool(case, g, n_pages, s)
        s["copies"] = torch.zeros((max(n_seqs, n_pages // 2), 3), dtype=torch.int32, device=DEV)
        s["counts"], s["status"] = torch.zeros(2, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
        row = torch.arange(n_seqs, dtype=torch.int32, device=DEV)
        if case["path"] == "branch":
            s["parent"] = torch.where(row < B, row, (row - B) % B).to(torch.int32)
            s["rows"] = torch.where(row < B, 0, rows).to(torch.int32)
            s["most"] = n_seqs
        else:
            # two halves that take turns: who leaves in this pass comes back, as a new user of the same length, at its end
            s["turn"] = 0
            s["leave"] = [torch.where(row % 2 == t, -1, row).to(torch.int32) for t in (0, 1)]
            s["come"] = [torch.where(row % 2 == t, s["len"], 0).to(torch.int32) for t in (0, 1)]
            s["most"] = n_pages // 2
            s["copies2"], s["counts2"] = torch.zeros_like(s["copies"]), torch.zeros_like(s["counts"])
        if own:
            s["cfg"] = C.Config(n_heads=Hkv, d_head=D, dtype=C.F32 if case["dtype"] == "f32" else C.BF16)
            s["pool"] = C.page_pool(refs, table, held, s["len"], P)
            s["ws"] = torch.empty(C.climber_pages_workspace_bytes(s["pool"]), dtype=torch.uint8, device=DEV)
            if case["dtype"] == "e4m3":
                s["kv"] = C.paged_kv8(s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"], table, s["len"], width * P)
            else:
                s["kv"] = C.paged_kv(s["k_pages"], s["v_pages"], table, s["len"], width * P)
        return s
    H, chunk = case["heads"], _lengths(case, "chunk")
    appends, m = case["path"] == "history", sum(chunk)
    need = [-(-(c + (t if appends else 0)) // P) for c, t in zip(cached, chunk)]
    n_pages = sum(need) + sum(need) // 8 + 1            # one page in eight is free
    s["table"], s["len"] = _pages(g, need, n_pages), torch.tensor(cached, dtype=torch.int32, device=DEV)
    _pool(case, g, n_pages, s)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16)

    if case["packed"]:
        q, k, v = normal(m, (H + 2 * Hkv) * D).split([H * D, Hkv * D, Hkv * D], dim=1)
        s["q"], s["k"], s["v"] = q.unflatten(1, (H, D)), k.unflatten(1, (Hkv, D)), v.unflatten(1, (Hkv, D))
    else:
        s["q"], s["k"], s["v"] = normal(m, H, D), normal(m, Hkv, D), normal(m, Hkv, D)
    s["off"] = torch.tensor([sum(chunk[:b]) for b in range(B + 1)], dtype=torch.int32, device=DEV)
    s["scen"], s["beh"] = (torch.randint(0, hi, (m,), generator=g, device=DEV, dtype=torch.int32) for hi in (N_SCEN, N_BEH))
    s["tau"] = torch.rand((N_SCEN, N_BEH), generator=g, device=DEV) * 1.5 + 0.5
    s["o"] = torch.empty((m, H * D), dtype=torch.bfloat16, device=DEV)
    s["m_total"], s["m_max"] = m, max(chunk)
    if own:
        longest = max(c + (t if appends else 0) for c, t in zip(cached, chunk))
        s["cfg"] = C.Config(n_heads=H, d_head=D, n_scen=N_SCEN, n_beh=N_BEH, dtype=C.BF16, flags=C.HIST_CAUSAL if case["causal"] else 0,
                            qk_scale=D ** -0.5)
        s["kv"] = C.paged_kv8(s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"], s["table"], s["len"], longest)
        s["ws"] = torch.empty(C.climber_paged8_workspace_bytes(s["cfg"], s["kv"], m, s["m_max"]), dtype=torch.uint8, device=DEV)
    return s


# ---- a pass --------------------------------------------------------------------------------------
def _pool_of(s):
    out = {"k": s["k_pages"], "v": s["v_pages"]}
    if "k_scale" in s:
        out = {"k": _held(s["k_pages"]), "v": _held(s["v_pages"]), "k_scale": s["k_scale"], "v_scale": s["v_scale"]}
    return out


def run(s):
    case = s["case"]
    if own:
        import paper_2502_09888_amd as C
        if case["path"] == "history":
            C.climber_attn_history_paged8(s["cfg"], s["tau"], s["kv"], s["q"], s["k"], s["v"], s["off"], s["m_total"], s["m_max"], s["scen"],
                                          s["beh"], None, s["o"], s["ws"])
            return {"o": s["o"]} | _pool_of(s)
        if case["path"] == "score":
            C.climber_attn_sumi_paged8(s["cfg"], s["tau"], s["kv"], s["q"], s["k"], s["v"], s["off"], s["m_total"], s["m_max"], s["scen"],
                                       s["beh"], s["o"], s["ws"])
            return {"o": s["o"]}
        if case["path"] == "rotary":
            C.climber_rotary(s["cfg"], s["rot"], s["pos"], case["kv_heads"], s["q"], s["k"], s["q_out"], s["k_out"])
            return {"q": s["q_out"], "k": s["k_out"]}
        copy = C.climber_paged8_copy if case["dtype"] == "e4m3" else C.climber_paged_copy
        if case["path"] == "branch":
            C.climber_pages_fork(s["pool"], s["parent"], None, s["status"], s["ws"])
            C.climber_pages_extend(s["pool"], s["rows"], s["copies"], s["counts"], s["status"], s["ws"])
            copy(s["cfg"], s["kv"], s["copies"], s["counts"], s["most"])
            return _state(s)
        t, s["turn"] = s["turn"], 1 - s["turn"]
        C.climber_pages_fork(s["pool"], s["leave"][t], None, s["status"], s["ws"])
        C.climber_pages_compact(s["pool"], s["copies"], s["counts"], s["status"], s["ws"])
        copy(s["cfg"], s["kv"], s["copies"], s["counts"], s["most"])
        C.climber_pages_extend(s["pool"], s["come"][t], s["copies2"], s["counts2"], s["status"], s["ws"])
        s["len"] += s["come"][t]
        return _state(s)
    if case["path"] == "rotary":
        return _plain_rotary(s)
    if case["path"] == "branch":
        _plain_fork(s, s["parent"])
        _plain_extend(s, s["rows"], s["copies"], s["counts"])
        _plain_copy(s)
        return _state(s)
    if case["path"] == "compact":
        t, s["turn"] = s["turn"], 1 - s["turn"]
        _plain_fork(s, s["leave"][t])
        _plain_compact(s)
        _plain_copy(s)
        _plain_extend(s, s["come"][t], s["copies2"], s["counts2"])
        s["len"] += s["come"][t]
        return _state(s)
    o = _plain_attention(s)
    if case["path"] == "score":
        return {"o": o}
    _plain_append(s)
    return {"o": o} | _pool_of(s)


def _state(s):
    keep = ("table", "held", "refs", "len", "copies", "counts", "status", "copies2", "counts2")
    return {k: s[k] for k in keep if k in s} | _pool_of(s)


def _plain_rotary(s):
    """Angles in 64 bits, products in 32."""
    case, out = s["case"], {}
    rot, half = case["rot"], case["rot"] // 2
    angle = s["pos"].double()[:, None] * s["freq"]
    if case["inverse"]:
        angle = -angle
    c, sn = (torch.cos(angle) * s["mul"]).float()[:, None], (torch.sin(angle) * s["mul"]).float()[:, None]
    for name in ("q", "k"):
        x = s[name].float()
        turned = x[..., :rot]
        a, b = (turned[..., 0::2], turned[..., 1::2]) if case["interleaved"] else (turned[..., :half], turned[..., half:])
        u, v = a * c - b * sn, a * sn + b * c
        turned = torch.stack([u, v], dim=-1).flatten(-2) if case["interleaved"] else torch.cat([u, v], dim=-1)
        out[name] = torch.cat([turned, x[..., rot:]], dim=-1).to(s[name].dtype)
    return out


def _plain_fork(s, parent):
    """Row b of the table becomes row parent[b], up to the page of its last token; -1: empty.  A row that is its own parent stays."""
    P = s["case"]["page"]
    table, held, n = s["table"].long(), s["held"].long(), s["len"].long()
    me = torch.arange(n.numel(), device=DEV)
    col = torch.arange(table.shape[1], device=DEV)
    par = parent.long().clamp(min=0)
    new_len = torch.where(parent >= 0, n[par], 0)
    new_held = torch.where(parent == me, held, torch.minimum((new_len + P - 1) // P, held[par]))
    new_table = torch.where(col < new_held[:, None], table[par], -1)
    none = s["refs"].numel()
    flat = torch.zeros(none + 1, dtype=torch.int32, device=DEV)
    one = torch.ones(table.numel(), dtype=torch.int32, device=DEV)
    flat.scatter_add_(0, torch.where(col < held[:, None], table, none).view(-1), -one)
    flat.scatter_add_(0, torch.where(new_table >= 0, new_table, none).view(-1), one)
    s["refs"] += flat[:-1]
    s["table"].copy_(torch.where(col < torch.maximum(held, new_held)[:, None], new_table, table))
    s["held"].copy_(new_held)
    s["len"].copy_(new_len)


def _plain_extend(s, rows, copies, counts):
    """Pages for rows[b] more tokens: the lowest free ones, by sequence and place.  A shared page that is written is copied, unless all that
    share it write it: then the last of them keeps it."""
    P = s["case"]["page"]
    table, held, n, refs = s["table"].long(), s["held"].long(), s["len"].long(), s["refs"]
    col, none = torch.arange(table.shape[1], device=DEV), refs.numel()
    me = torch.arange(n.numel(), device=DEV)
    need = torch.where(rows > 0, (n + rows + P - 1) // P, held)
    fresh = (col >= held[:, None]) & (col < need[:, None])
    written = (col >= (n // P)[:, None]) & (col < torch.minimum(held, need)[:, None]) & (rows > 0)[:, None]
    at = torch.where(written, table, none)
    writers = torch.zeros(none + 1, dtype=torch.int32, device=DEV).scatter_add_(0, at.view(-1), torch.ones_like(at, dtype=torch.int32).view(-1))
    last = torch.full((none + 1,), -1, device=DEV).scatter_reduce_(0, at.view(-1), me[:, None].expand_as(at).reshape(-1), "amax")
    r = torch.cat([refs, refs.new_zeros(1)])[at]
    moved = written & (r > 1) & ~((writers[at] == r) & (last[at] == me[:, None]))
    new = fresh | moved
    free = torch.nonzero(refs == 0).view(-1)
    order = torch.cumsum(new.view(-1).long(), 0).view_as(table) - 1
    fits = (order.view(-1)[-1] < free.numel()) & (need <= table.shape[1]).all()
    new, moved = new & fits, moved & fits
    page = free[order.clamp(0, max(0, free.numel() - 1))] if free.numel() else torch.zeros_like(order)
    s["status"] |= torch.where(fits, 0, 128).to(torch.int32)
    part = moved & (col == (n // P)[:, None]) & (n % P > 0)[:, None]
    b, i = torch.nonzero(part, as_tuple=True)
    copies[:b.numel()] = torch.stack([table[b, i], page[b, i], n[b] % P], dim=1).to(torch.int32)
    delta = torch.zeros(none + 1, dtype=torch.int32, device=DEV)
    one = torch.ones(table.numel(), dtype=torch.int32, device=DEV)
    delta.scatter_add_(0, torch.where(new, page, none).view(-1), one)
    delta.scatter_add_(0, torch.where(moved, table, none).view(-1), -one)
    refs += delta[:-1]
    s["table"].copy_(torch.where(new, page, table))
    s["held"].copy_(torch.where(fits, torch.maximum(held, need), held))
    counts[0] = b.numel()
    counts[1] = (refs > 0).sum()


def _plain_compact(s):
    """The pages in use behind the place where the pages in use would end go, in order, to the free ones before it."""
    refs, used = s["refs"], s["refs"] > 0
    n_used, page = used.sum(), torch.arange(s["refs"].numel(), device=DEV)
    mover, hole = torch.nonzero(used & (page >= n_used)).view(-1), torch.nonzero(~used & (page < n_used)).view(-1)
    to = page.clone()
    to[mover] = hole
    refs[hole] = refs[mover]
    refs[mover] = 0
    has = torch.arange(s["table"].shape[1], device=DEV) < s["held"][:, None]
    s["table"].copy_(torch.where(has, to[s["table"].long().clamp(min=0)], s["table"]))
    s["copies"][:mover.numel()] = torch.stack([mover, hole, torch.full_like(mover, s["case"]["page"])], dim=1).to(torch.int32)
    s["counts"][0] = mover.numel()
    s["counts"][1] = n_used


def _plain_copy(s):
    P = s["case"]["page"]
    c = s["copies"][: int(s["counts"][0])].long()
    i, slot = torch.nonzero(torch.arange(P, device=DEV) < c[:, 2:], as_tuple=True)
    whole = bool((c[:, 2] == P).all())
    for name in ("k_pages", "v_pages"):
        if whole:
            s[name][c[:, 1]] = s[name][c[:, 0]]
        else:
            s[name][c[i, 1], :, slot] = s[name][c[i, 0], :, slot]
    if "k_scale" in s:
        i, block = torch.nonzero(torch.arange(P // BLOCK, device=DEV) * BLOCK < c[:, 2:], as_tuple=True)
        for name in ("k_scale", "v_scale"):
            s[name][c[i, 1], :, block] = s[name][c[i, 0], :, block]


def _values(s, name, page, slot):
    """The values that 8-bit slots stand for, in 32 bits: [..., kv_heads, d]."""
    return _held(s[name + "_pages"][page, :, slot]).float() * _two_to(s[name + "_scale"][page, :, slot // BLOCK].int() - 127)[..., None]


def _plain_attention(s):
    """Attention over the gathered cache in 32 bits: users padded to the longest."""
    case, m = s["case"], s["m_total"]
    B, P, Hkv, D, H = case["users"], case["page"], case["kv_heads"], case["d_head"], case["heads"]
    G, T, L = H // Hkv, case["chunk"], case["cached"]
    n, off, table = s["len"].long(), s["off"].long(), s["table"].long().clamp(min=0)
    row = torch.arange(m, device=DEV)
    seq = torch.searchsorted(off, row, right=True) - 1
    t = row - off[seq]
    slot = torch.arange(L, device=DEV)
    page = table[:, slot // P]                                                     # [B, L]
    K = _values(s, "k", page, slot % P).permute(0, 2, 1, 3)                        # [B, Hkv, L, D]
    V = _values(s, "v", page, slot % P).permute(0, 2, 1, 3)
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
    return o.view(B, Hkv, G, T, D).permute(0, 3, 1, 2, 4).reshape(B, T, H * D)[seq, t].to(s["o"].dtype)


def _plain_append(s):
    """New tokens into their pages: a block's scale is the largest that one of its tokens needs, and tokens that it held before are
    rounded again where it grew."""
    case, m = s["case"], s["m_total"]
    P, Hkv = case["page"], case["kv_heads"]
    n, off, table = s["len"].long(), s["off"].long(), s["table"].long()
    row = torch.arange(m, device=DEV)
    seq = torch.searchsorted(off, row, right=True) - 1
    slot = n[seq] + row - off[seq]
    page, inside = table[seq, slot // P], slot % P
    per = P // BLOCK
    block = (page[:, None] * Hkv + torch.arange(Hkv, device=DEV)) * per + (inside // BLOCK)[:, None]      # [m, Hkv]
    begins = (slot // BLOCK * BLOCK >= n[seq])[:, None].expand_as(block)     # a block without older tokens
    # the older tokens of the block that a sequence's first new one goes into
    old_slot = (n // BLOCK * BLOCK)[:, None] + torch.arange(BLOCK, device=DEV)
    b, j = torch.nonzero((old_slot < n[:, None]) & (off[1:] > off[:-1])[:, None], as_tuple=True)
    old_slot = old_slot[b, j]
    old_page, old_inside = table[b, old_slot // P], old_slot % P
    old_block = (old_page[:, None] * Hkv + torch.arange(Hkv, device=DEV)) * per + (old_inside // BLOCK)[:, None]
    for name in ("k", "v"):
        x = s[name].float()
        mine = _scale_of(torch.where(x.isfinite(), x.abs(), 0).amax(-1))                                    # [m, Hkv]
        scale = s[name + "_scale"].view(-1).int()
        before = scale[old_block]
        scale[block[begins]] = LEAST
        scale.scatter_reduce_(0, block.view(-1), mine.int().view(-1), "amax")
        s[name + "_scale"].view(-1).copy_(scale)
        codes = s[name + "_pages"]
        again = _held(codes[old_page, :, old_inside]).float() * _two_to((before - scale[old_block]).clamp(min=-126))[..., None]
        codes[old_page, :, old_inside] = again.to(torch.float8_e4m3fn).view(torch.uint8)
        codes[page, :, inside] = (x * _two_to(127 - scale[block])[..., None]).to(torch.float8_e4m3fn).view(torch.uint8)


# ---- what a pass cannot do without ---------------------------------------------------------------
def work(case):
    if case["path"] == "rotary":
        e, heads = 4 if case["dtype"] == "f32" else 2, case["heads"] + case["kv_heads"]
        return {"bytes": case["rows"] * (2 * e * heads * case["d_head"] + 4) + 4 * case["rot"], "flops": case["rows"] * heads * case["rot"] * 3}
    P, Hkv, D = case["page"], case["kv_heads"], case["d_head"]
    cached = _lengths(case, "cached")
    e = {"f32": 4, "bf16": 2}.get(case.get("dtype"), 1)
    token = 2 * Hkv * (D * e + (1 / BLOCK if e == 1 else 0))       # a cached token's key and value
    need = [-(-c // P) for c in cached]
    if case["path"] == "branch":
        F, rows = case["branches"], case["rows"]
        copied = sum(F * (c % P) for c in cached)                  # (a history that ends inside its page: the branches do)
        after = sum(F * -(-(c + rows) // P) for c in cached)
        pages = sum(need) + sum(F * (-(-(c + rows) // P) - c // P) for c in cached) + sum(need) // 8 + 1
        return {"bytes": 2 * copied * token + 4 * (sum(need) + 2 * after + 2 * pages), "flops": pages}
    if case["path"] == "compact":
        # The pages of the last pass's new users lie behind those that leave now, and move to their places as far as these reach.  (On the
        # very first pass pages lie in any order: half as many.)
        moved = min(sum(need[0::2]), sum(need[1::2]))
        pages = sum(need) + sum(need) // 8 + 1
        return {"bytes": 2 * moved * P * token + 4 * (4 * sum(need) + 4 * pages), "flops": pages}
    m, wide, pairs = sum(_lengths(case, "chunk")), case["heads"] * D, 0
    for n, t in zip(cached, _lengths(case, "chunk")):
        pairs += t * (n + 1) if case["path"] == "score" else t * n + (t * (t + 1) // 2 if case["causal"] else t * t)
    total = m * (2 * wide * 2 + 2 * Hkv * D * 2 + 8) + sum(cached) * token
    if case["path"] == "history":
        total += m * token
    return {"bytes": total, "flops": 4 * wide * pairs}


# ---- from the definitions, in 64 bits ------------------------------------------------------------
def exact(case, seed):
    if case["path"] in ("branch", "compact"):
        return None                                            # nothing is computed: what lies where has to be equal
    s = prepare(case, seed)
    if case["path"] == "rotary":
        # pairs as complex numbers, turned by exp(i angle)
        rot, out = case["rot"], {}
        turn = torch.polar(torch.full_like(s["freq"], s["mul"])[None].expand(case["rows"], -1).contiguous(),
                           s["pos"].double()[:, None] * s["freq"] * (-1 if case["inverse"] else 1))[:, None]
        for name in ("q", "k"):
            y = s[name].double().clone()
            first = slice(0, rot, 2) if case["interleaved"] else slice(0, rot // 2)
            second = slice(1, rot, 2) if case["interleaved"] else slice(rot // 2, rot)
            z = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * turn
            y[..., first], y[..., second] = z.real, z.imag
            out[name] = y
        return out
    P, D, G = case["page"], case["d_head"], case["heads"] // case["kv_heads"]
    out = torch.zeros(s["o"].shape, dtype=torch.float64, device=DEV).view(-1, case["heads"], D)
    r0 = 0
    for b, (n, t) in enumerate(zip(_lengths(case, "cached"), _lengths(case, "chunk"))):
        rows = slice(r0, r0 + t)
        r0 += t
        pages = s["table"][b, :-(-n // P)].long()
        tau = s["tau"].double()[s["scen"][rows].long(), s["beh"][rows].long()]
        for h in range(case["kv_heads"]):
            keys, values = (torch.cat([(_held(s[x + "_pages"][pages, h]).double() * 2.0 ** (s[x + "_scale"][pages, h].double() - 127)
                                        .repeat_interleave(BLOCK, dim=1)[..., None]).view(-1, D)[:n], s[x][rows, h].double()]) for x in ("k", "v"))
            sees = torch.ones(t, n + t, dtype=torch.bool, device=DEV)
            if case["path"] == "score":
                sees[:, n:] = torch.eye(t, dtype=torch.bool, device=DEV)
            elif case["causal"]:
                sees = sees.tril(diagonal=n)
            for j in range(G):
                logits = s["q"][rows, h * G + j].double() @ keys.t() / math.sqrt(D) / tau[:, None]
                out[rows, h * G + j] = torch.softmax(torch.where(sees, logits, -math.inf), dim=1) @ values
    answer = {"o": out.view(s["o"].shape)}
    return answer if case["path"] == "score" else answer | {"k": None, "v": None, "k_scale": None, "v_scale": None}
