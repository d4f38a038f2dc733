"""The paged history cache on the GPU against its definitions in 64 bits (paged_ref.py)."""
import math

import pytest
import torch

from paged_ref import Case, Device, evict_ref

pytestmark = pytest.mark.gpu

# (cached, chunk) of the sequences: one token; chunks that begin and end inside pages and tiles; sequences without rows or without a
# cache; lengths around the tiles
LENS = {
    "one token": ([1], [1]),
    "first token": ([0], [1]),
    "decode": ([5, 0, 64, 200, 33], [1, 1, 1, 1, 1]),
    "chunks": ([17, 0, 100, 63, 0], [3, 70, 0, 65, 0]),
    "prompts": ([0, 0, 0], [130, 1, 67]),
    "long": ([300, 1000], [20, 150]),
}


def same_bits(a, b):
    return torch.equal(a.cpu().view(torch.uint8), b.cpu().view(torch.uint8))


def check(case, dev, calls=1):
    """o, stored rows, masses and stamps after `calls` calls."""
    o, tol, weight, wtol = case.expect()
    got = dev.out()
    rows = sum(case.chunk)
    assert torch.isfinite(got[:rows]).all()
    off = (got[:rows] - o[:rows]).abs() - tol[:rows]
    assert off.max() <= 0 if rows else True, f"max over the bound {off.max():.3e}, error {(got[:rows] - o[:rows]).abs().max():.3e}"
    assert (got[rows:] == 77.0).all()           # rows of no sequence
    k, v = case.k.clone(), case.v.clone()
    mass, stamp = case.mass.double().clone(), case.stamp.clone()
    bound = torch.zeros_like(mass)
    for b, (n, t) in enumerate(zip(case.cached, case.chunk)):
        for j in range(n if case.sumi else n + t):
            pg, s = case.at(b, j)
            if j >= n:
                r = int(case.off[b]) + j - n
                k[pg, :, s], v[pg, :, s], stamp[pg, s] = case.kn[r], case.vn[r], case.stamp_new[r]
            if t:
                before = mass[pg, s] if j < n else 0.0
                mass[pg, s] = before + weight[b][j] * (calls if j < n else 1)
                bound[pg, s] = calls * (wtol[b][j] + mass[pg, s] * 2.0 ** -23)
    assert same_bits(dev.k, k) and same_bits(dev.v, v)
    if dev.stamp is not None:
        assert torch.equal(dev.stamp.cpu(), case.stamp if case.sumi else stamp)
    if dev.mass is not None:
        got = dev.mass.double().cpu()
        assert torch.equal(torch.isnan(got), torch.isnan(mass))
        over = (got - mass).abs().nan_to_num() - bound
        assert over.max() <= 0, f"mass: {over.max():.3e} over its bound"


@pytest.mark.parametrize("sumi", [False, True], ids=["history", "sumi"])
@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 32), ("f32", 64), ("f32", 100), ("f32", 128), ("f32", 4)])
@pytest.mark.parametrize("lens", LENS)
def test_attention_and_weights(lens, dtype, d, sumi):
    case = Case(*LENS[lens], d=d, dtype=dtype, sumi=sumi, seed=len(lens) + d)
    dev = Device(case, mass=True, stamp=True)
    dev.attend()
    check(case, dev)


@pytest.mark.parametrize("sumi", [False, True], ids=["history", "sumi"])
@pytest.mark.parametrize("H,Hkv", [(1, 1), (3, 3), (5, 1), (8, 2), (12, 4), (40, 1), (64, 8)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_head_layouts(H, Hkv, dtype, sumi):
    case = Case([70, 9], [7, 33], H=H, Hkv=Hkv, dtype=dtype, sumi=sumi, seed=H)
    dev = Device(case, mass=True)
    dev.attend()
    check(case, dev)


@pytest.mark.parametrize("page", [16, 32, 128, 1024])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pages_strides_and_whole_chunks(page, dtype):
    # without the causal flag every new token sees the whole chunk; rows are columns of wider rows; three rows belong to nobody
    for causal in (False, True):
        case = Case([page - 1, 40, 2 * page + 5], [page + 3, 9, 70], page=page, dtype=dtype, causal=causal, tail=3, seed=page)
        dev = Device(case, mass=True, packed=True, pad_o=8)
        dev.attend()
        check(case, dev)


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 64)])
def test_long_cache_of_one_token(dtype, d):
    # the keys are shared out over workgroups and the parts joined
    case = Case([5003], [1], d=d, page=64, dtype=dtype, seed=3)
    dev = Device(case, mass=True)
    dev.attend()
    check(case, dev)
    # ... with a launch sized for far longer sequences, so that most parts are empty
    wide = Case([37, 1], [1, 2], d=d, page=64, dtype=dtype, seed=4)
    wide.table = torch.cat([wide.table, torch.full((2, 1000), -1, dtype=torch.int32)], dim=1)
    dev = Device(wide, mass=True, max_len=60000)
    dev.attend()
    check(wide, dev)


@pytest.mark.parametrize("sumi", [False, True], ids=["history", "sumi"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_logits(dtype, sumi):
    # one-hot rows, and logits far above and below those before them
    case = Case([150, 80], [40, 100], dtype=dtype, std=6.0, scale=1.0, sumi=sumi, seed=11)
    case.tau.fill_(0.5)
    dev = Device(case, mass=True)
    dev.attend()
    check(case, dev)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf, 3.0e38])
@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 64)])
def test_a_token_has_no_influence_on_rows_that_do_not_see_it(dtype, d, bad):
    at = 50                                               # of the chunk's 100 tokens
    clean, case = Case([20], [100], d=d, dtype=dtype, seed=5), Case([20], [100], d=d, dtype=dtype, seed=5)
    for name in ("kn", "vn"):
        getattr(case, name)[at:] = bad
    a, b = Device(clean, mass=True), Device(case, mass=True)
    a.attend(), b.attend()
    x, y = a.out(), b.out()
    assert torch.equal(x[:at], y[:at])
    # a token's infinite value reaches the rows that do see it
    only = Case([20], [100], d=d, dtype=dtype, seed=5)
    if math.isinf(bad) or math.isnan(bad):
        only.vn[at, 1, 7] = bad
        dev = Device(only)
        dev.attend()
        z = dev.out()
        assert torch.equal(z[:at], x[:at])
        odd = z[at:, 2:, 7]                               # (heads 2 and 3 read cache head 1)
        assert (torch.isnan(odd) if math.isnan(bad) else odd == bad).all()
        z[at:, 2:, 7] = x[at:, 2:, 7]
        assert torch.equal(z, x)


def test_candidates_do_not_see_each_other():
    for dtype in ("bf16", "f32"):
        clean, case = Case([70], [90], dtype=dtype, sumi=True, seed=6), Case([70], [90], dtype=dtype, sumi=True, seed=6)
        case.kn[30] = math.nan
        case.vn[31] = math.inf
        a, b = Device(clean), Device(case)
        a.attend(), b.attend()
        x, y = a.out(), b.out()
        keep = [i for i in range(90) if i not in (30, 31)]
        assert torch.equal(x[keep], y[keep])
        assert torch.isnan(y[30]).all() and (y[31] == math.inf).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_chunk_by_chunk_is_the_whole(dtype):
    # a history appended in portions of any size gives the rows that it gives at once
    whole = Case([0], [150], dtype=dtype, seed=8, page=32)
    o, tol, _, _ = whole.expect()
    dev = Device(whole, mass=True)
    at = 0
    for size in (1, 40, 1, 64, 3, 41):
        dev.off.copy_(torch.tensor([0, size]))
        dev.m_max = size
        q, kn, vn, scen, beh, out = (x[at:at + size] for x in (dev.q, dev.kn, dev.vn, dev.scen, dev.beh, dev.o))
        dev.P.climber_attn_history_paged(dev.cfg, dev.tau, dev.kv, q, kn, vn, dev.off, size, size, scen, beh, None, out, dev.ws)
        dev.len += size
        at += size
    assert at == 150
    got = dev.out()
    assert ((got - o).abs() <= tol).all()


def test_shared_pages():
    # two sequences with the same first pages: read by both, written by none
    case = Case([64, 70], [5, 6], page=16, seed=9)
    case.table[1, :4] = case.table[0, :4]
    case.cached[0] = 64
    for name in ("k", "v"):
        assert not torch.isnan(getattr(case, name)[case.table[0, :4].long()]).any()
    dev = Device(case)
    dev.attend()
    check(case, dev)


def test_lengths_and_page_numbers_that_break_the_contract_stay_in_bounds():
    case = Case([30, 40], [4, 4], seed=10)
    dev = Device(case, mass=True, stamp=True)
    before = dev.k.clone()
    status = torch.zeros(1, dtype=torch.int32, device="cuda:0")
    dev.P.climber_check_paged(dev.cfg, dev.kv, dev.off, case.m, dev.m_max, True, status)
    assert status.item() == 0
    dev.table[0, :] = 10 ** 6
    dev.table[1, :] = -5
    dev.len.copy_(torch.tensor([-3, 10 ** 9]))
    dev.P.climber_check_paged(dev.cfg, dev.kv, dev.off, case.m, dev.m_max, True, status)
    assert status.item() == dev.P.BAD_PAGE | dev.P.BAD_LEN
    dev.history()
    dev.sumi()
    torch.cuda.synchronize()
    assert same_bits(dev.k, before)                       # a token without a page is not stored
    status.zero_()
    dev.off.copy_(torch.tensor([3, 2, 10 ** 9]))
    dev.P.climber_check_paged(dev.cfg, dev.kv, dev.off, case.m, dev.m_max, False, status)
    assert status.item() & dev.P.BAD_OFFSETS and status.item() & dev.P.BAD_M_MAX
    dev.history()
    dev.sumi()
    torch.cuda.synchronize()


@pytest.mark.parametrize("sumi", [False, True], ids=["history", "sumi"])
@pytest.mark.parametrize("lens", ["decode", "chunks"])
def test_captured_calls_follow_lengths_and_rows(lens, sumi):
    cached, chunk = LENS[lens]
    case = Case(cached, chunk, sumi=sumi, seed=12)
    dev = Device(case, mass=True, max_len=max(1, case.table.shape[1] * case.page))
    dev.attend()
    dev.out()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        dev.attend(torch.cuda.current_stream())
    for seed in (13, 14, 15):
        new = Case([max(0, c - seed % 3) for c in cached], chunk, sumi=sumi, seed=seed)
        for name in ("k", "v", "table", "len", "mass", "q", "kn", "vn", "scen", "beh", "tau"):
            to, x = getattr(dev, name), getattr(new, name)
            if name in ("k", "v", "mass") and x.shape != to.shape:
                x = torch.cat([x, x.new_full((to.shape[0] - x.shape[0],) + x.shape[1:], math.nan)])
                setattr(new, name, x)
            if name == "table" and x.shape != to.shape:
                x = torch.cat([x, x.new_full((x.shape[0], to.shape[1] - x.shape[1]), -1)], dim=1)
            to.copy_(x)
        dev.o.fill_(5.0)
        graph.replay()
        dev.c = new
        check(new, dev)


def test_other_streams_and_two_calls_at_once():
    # two caches, two streams, a workspace each
    cases = [Case([700], [50], seed=s, page=64) for s in (20, 21)]
    devs = [Device(c, mass=True) for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in devs]
    for _ in range(3):
        for d, s in zip(devs, streams):
            d.history(s)
    torch.cuda.synchronize()
    for c, d in zip(cases, devs):
        check(c, d, calls=3)


def test_same_call_same_bits():
    case = Case([300, 800, 5], [100, 1, 40], H=8, seed=22)
    results = []
    for _ in range(2):
        dev = Device(case, mass=True)
        dev.attend()
        results.append((dev.out(), dev.mass.cpu()))
    assert torch.equal(results[0][0], results[1][0]) and same_bits(results[0][1], results[1][1])


# ---- eviction ------------------------------------------------------------------------------------

def evict(case, budget, rank=None, keep_from=None, mass=True, stamp=True, src=True, in_place=False, max_len=None):
    dev = Device(case, mass=mass, stamp=stamp, max_len=max_len)
    dev_rank = rank.to("cuda:0") if rank is not None else None
    len_out = dev.len if in_place else torch.full_like(dev.len, -9)
    B = len(case.cached)
    src_t = torch.full((B, case.table.shape[1] * case.page), -9, dtype=torch.int32, device="cuda:0") if src else None
    dev.P.climber_paged_evict(dev.cfg, dev.kv, dev_rank, torch.tensor(budget, dtype=torch.int32, device="cuda:0"),
                              torch.tensor(keep_from, dtype=torch.int32, device="cuda:0") if keep_from is not None else None, len_out, src_t, dev.ws)
    torch.cuda.synchronize()
    used = rank if rank is not None else case.mass
    want = evict_ref(case.table, case.page, case.cached, budget, used, case.stamp, keep_from)
    k, v, m, st = (getattr(case, x).clone() for x in ("k", "v", "mass", "stamp"))
    for b, (keep, moved) in enumerate(want):
        assert int(len_out[b]) == keep
        if src:
            assert src_t[b].tolist() == moved + [-1] * (src_t.shape[1] - keep)
        for j, i in enumerate(moved):
            if i != j:
                (tp, ts), (fp, fs) = case.at(b, j), case.at(b, i)
                k[tp, :, ts], v[tp, :, ts], m[tp, ts], st[tp, ts] = case.k[fp, :, fs], case.v[fp, :, fs], case.mass[fp, fs], case.stamp[fp, fs]
    assert same_bits(dev.k, k) and same_bits(dev.v, v)
    if mass:
        assert same_bits(dev.mass, m)
    if stamp:
        assert torch.equal(dev.stamp.cpu(), st)


CACHED = [0, 1, 5, 64, 65, 200, 777]


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 4), ("f32", 64)])
@pytest.mark.parametrize("in_place", [False, True])
def test_evict(dtype, d, in_place):
    evict(Case(CACHED, [1] * 7, dtype=dtype, d=d, sumi=True, seed=30), [3, 1, 2, 33, 64, 150, 300], in_place=in_place)


def test_evict_none_all_and_beyond():
    evict(Case(CACHED, [1] * 7, sumi=True, seed=31), [0, 0, -4, 1000, 0, 200, 2 ** 31 - 1])


@pytest.mark.parametrize("recent", [0, 1, 40, 150, 10 ** 6])
def test_evict_keeps_the_stamped_first(recent):
    # fewer of them than the budget, as many, and more
    evict(Case(CACHED, [1] * 7, sumi=True, seed=32), [1, 1, 3, 40, 40, 100, 151], keep_from=[c - recent for c in CACHED])


def test_evict_ties_and_odd_ranks():
    case = Case(CACHED, [1] * 7, sumi=True, seed=33)
    g = torch.Generator().manual_seed(1)
    odd = torch.tensor([0.0, -0.0, 1.0, 1.0, math.nan, math.inf, -math.inf, -2.5, 1e-40, 3e38])
    rank = odd[torch.randint(0, len(odd), case.mass.shape, generator=g)]
    for budget in ([1, 1, 2, 20, 31, 90, 400], [0, 0, 4, 63, 64, 199, 776]):
        evict(case, budget, rank=rank)
        evict(case, budget, rank=torch.ones_like(rank))
    evict(case, [0, 1, 1, 1, 1, 1, 1], rank=rank, mass=False, stamp=False, src=False)


@pytest.mark.parametrize("n,budget", [(1024, 512), (1025, 1024), (2047, 1000), (4096, 1), (5000, 4999), (16384, 8192),
                                      (16385, 16384), (20011, 7), (20011, 4096), (20011, 13000), (33000, 16000)])
def test_evict_long(n, budget):
    case = Case([n, 3], [1, 1], H=1, Hkv=1, d=4, dtype="f32", page=64, sumi=True, seed=34)
    evict(case, [budget, 1])
    case.mass = torch.where(case.mass < 0.5, case.mass, 0.75)      # a cut inside equals
    evict(case, [budget, 1], keep_from=[n - 5, 0])


def test_append_score_and_evict_together():
    """A cache in use: sessions join it, candidates are scored, it is cut by what they looked at, and all again, against the definitions."""
    d, page, B = 64, 16, 2
    state = Case([60, 25], [30, 7], page=page, seed=40)
    dev = Device(state, mass=True, stamp=True, max_len=96)
    for step in range(3):
        # append
        state.sumi = dev.c.sumi = False
        dev.attend()
        check(state, dev)
        for b in range(B):
            for i in range(state.chunk[b]):
                pg, s = state.at(b, state.cached[b] + i)
                r = int(state.off[b]) + i
                state.k[pg, :, s], state.v[pg, :, s], state.stamp[pg, s] = state.kn[r], state.vn[r], state.stamp_new[r]
            state.cached[b] += state.chunk[b]
        state.mass = dev.mass.cpu()
        state.len = torch.tensor(state.cached, dtype=torch.int32)
        dev.len.copy_(state.len)
        # score, with the same rows as candidates
        state.sumi = True
        dev.attend()
        check(state, dev)
        state.mass = dev.mass.cpu()
        # cut: the weights as the GPU has them
        budget, keep_from = [50, 20], [1000 + 10 * step, 1003]
        want = evict_ref(state.table, page, state.cached, budget, state.mass, state.stamp, keep_from)
        dev.P.climber_paged_evict(dev.cfg, dev.kv, None, torch.tensor(budget, dtype=torch.int32, device="cuda:0"),
                                  torch.tensor(keep_from, dtype=torch.int32, device="cuda:0"), dev.len, None, dev.ws)
        torch.cuda.synchronize()
        old = {x: getattr(state, x).clone() for x in ("k", "v", "mass", "stamp")}
        for b, (keep, moved) in enumerate(want):
            for j, i in enumerate(moved):
                (tp, ts), (fp, fs) = state.at(b, j), state.at(b, i)
                for x in ("k", "v"):
                    getattr(state, x)[tp, :, ts] = old[x][fp, :, fs]
                for x in ("mass", "stamp"):
                    getattr(state, x)[tp, ts] = old[x][fp, fs]
            state.cached[b] = keep
        state.len = torch.tensor(state.cached, dtype=torch.int32)
        assert torch.equal(dev.len.cpu(), state.len)
        for x in ("k", "v", "mass", "stamp"):
            assert same_bits(getattr(dev, x), getattr(state, x))
