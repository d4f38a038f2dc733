"""The paged history cache in 8 bits on the GPU against its definitions in 64 bits (paged8_ref.py)."""
import math

import numpy as np
import pytest
import torch

from paged8_ref import Case8, Device8, check8, check_cache, decode
from test_gpu_paged import LENS

pytestmark = pytest.mark.gpu


@pytest.fixture(params=[0, 1100], ids=["few", "many"])
def batch(request, monkeypatch):
    """The case alone, and with 1100 sequences that have nothing: more than a few rows are then done in tiles of 128 or 256, not of 32."""
    monkeypatch.setattr(Device8, "more", request.param)


@pytest.mark.parametrize("sumi", [False, True], ids=["history", "sumi"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens", LENS)
def test_attention_and_append(lens, d, sumi, batch):
    case = Case8(*LENS[lens], d=d, sumi=sumi, seed=len(lens) + d)
    dev = Device8(case, stamp=True)
    dev.attend()
    check8(case, dev)


@pytest.mark.parametrize("sumi", [False, True], ids=["history", "sumi"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,Hkv", [(1, 1), (3, 3), (5, 1), (8, 2), (40, 1), (64, 8)])
def test_head_layouts(H, Hkv, d, sumi, batch):
    case = Case8([70, 9], [7, 33], H=H, Hkv=Hkv, d=d, sumi=sumi, seed=H)
    dev = Device8(case)
    dev.attend()
    check8(case, dev)


@pytest.mark.parametrize("page", [16, 32, 128, 1024])
@pytest.mark.parametrize("d", [64, 128])
def test_pages_strides_and_whole_chunks(page, d, batch):
    # without the causal flag every new token sees the whole chunk; rows are columns of wider rows; three rows belong to nobody
    for causal in (False, True):
        case = Case8([page - 1, 40, 2 * page + 5], [page + 3, 9, 70], page=page, d=d, causal=causal, tail=3, seed=page)
        dev = Device8(case, packed=True, pad_o=8)
        dev.attend()
        check8(case, dev)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [2047, 5003, 9000])
def test_long_cache(d, n, batch):
    # keys shared out over workgroups whose parts are joined; more page numbers and scales than a wave holds at once
    for chunk in (1, 50):
        case = Case8([n], [chunk], d=d, page=64, H=8, seed=n)
        dev = Device8(case)
        dev.attend()
        check8(case, dev)
    case = Case8([n, 40], [70, 3], d=d, page=16, H=8, sumi=True, seed=n)
    dev = Device8(case)
    dev.attend()
    check8(case, dev)


@pytest.mark.parametrize("d", [64, 128])
def test_short_sequences_in_a_launch_for_long_ones(d, batch):
    wide = Case8([37, 1], [1, 2], d=d, page=64, seed=4)
    wide.table = torch.cat([wide.table, torch.full((2, 1000), -1, dtype=torch.int32)], dim=1)
    dev = Device8(wide, max_len=60000)
    dev.attend()
    check8(wide, dev)


@pytest.mark.parametrize("sumi", [False, True], ids=["history", "sumi"])
@pytest.mark.parametrize("d", [64, 128])
def test_many_rows_on_a_longer_cache(d, sumi, batch):
    # whole tiles of rows over many blocks of cached keys and of the call's own
    for causal in (True, False):
        case = Case8([700, 33, 0, 512], [300, 140, 257, 64], H=4, Hkv=1, d=d, page=32, sumi=sumi, causal=causal, seed=d)
        dev = Device8(case)
        dev.attend()
        check8(case, dev)


@pytest.mark.parametrize("kind", ["plain", "far", "odd"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("sumi", [False, True], ids=["history", "sumi"])
def test_the_largest_tiles(sumi, causal, kind):
    # enough rows of enough sequences for tiles of 256 rows at d_head 64
    g = torch.Generator().manual_seed(3)
    lens, rows = (torch.randint(0, hi, (40,), generator=g).tolist() for hi in (200, 150))
    lens[:3], rows[:3] = [199, 0, 64], [150, 150, 149]
    case = Case8(lens, rows, H=8, Hkv=4, d=64, page=32, sumi=sumi, causal=causal, seed=91, scale=1.0 if kind == "far" else None)
    if kind == "far":                                     # (as in test_weights_that_exceed_the_first_ones_by_far, in several rows)
        case.q.mul_(0.05), case.tau.fill_(1.0)
        case.q[20, 1, 0] = case.q[130, 5, 0] = case.q[160, 2, 0] = 24.0
        for hit in (40, 198):
            pg, s = case.at(0, hit)
            case.k[pg, :, s] = 0.0
            case.k[pg, :, s, 0] = 24.0
        case.quantise()
        case.kn[155] = 0.0
        case.kn[155, :, 0] = 24.0
    if kind == "odd":
        case.vn[100, 1, 7], case.vn[140, 2, 9] = math.inf, math.nan
    dev = Device8(case)
    dev.attend()
    if kind != "odd":
        check8(case, dev)
        return
    clean = Case8(lens, rows, H=8, Hkv=4, d=64, page=32, sumi=sumi, causal=causal, seed=91)
    other = Device8(clean)
    other.attend()
    x, y = dev.out(), other.out()
    # of the first sequence's 150 rows, those that see row 100, and row 140
    for at, heads, e, value in ((100, (2, 3), 7, math.inf), (140, (4, 5), 9, math.nan)):
        sees = [at] if sumi else list(range(at if causal else 0, 150))
        for h in heads:
            got = x[sees, h, e]
            assert (torch.isnan(got) if math.isnan(value) else got == value).all()
            x[sees, h, e] = y[sees, h, e]
    assert torch.equal(x, y)


@pytest.mark.parametrize("sumi", [False, True], ids=["history", "sumi"])
@pytest.mark.parametrize("d", [64, 128])
def test_large_logits(d, sumi, batch):
    # one-hot rows, and logits far above and below those before them
    case = Case8([150, 80], [40, 100], d=d, std=6.0, scale=1.0, sumi=sumi, seed=11)
    case.tau.fill_(0.5)
    dev = Device8(case)
    dev.attend()
    check8(case, dev)


@pytest.mark.parametrize("sumi", [False, True], ids=["history", "sumi"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("std,values", [(4.0, 1e30), (1.0, 1e32), (4.0, 1e-30)])
def test_large_and_small_values(d, std, values, sumi, batch):
    # weights of later keys that exceed those of the first by 2^30 and more, on values with which unscaled sums pass 2^128; 700 tokens
    # of at most 6e32 stay below 2^119
    case = Case8([500, 33], [190, 4], d=d, std=std, sumi=sumi, seed=53)
    case.v, case.vn = (case.v.float() * values).to(case.dt), (case.vn.float() * values).to(case.dt)
    case.quantise()
    dev = Device8(case)
    dev.attend()
    check8(case, dev)


@pytest.mark.parametrize("sumi", [False, True], ids=["history", "sumi"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("late", ["cached", "last cached", "own"])
def test_weights_that_exceed_the_first_ones_by_far(d, late, sumi, batch):
    # one row's logits rise by more than 2^100 in exp2 units behind the first blocks: the sums so far vanish against it, and its neighbours
    # keep theirs
    case = Case8([299, 0], [140, 130], H=4, Hkv=2, d=d, sumi=sumi, scale=1.0, seed=71)
    case.q.mul_(0.05), case.tau.fill_(1.0)
    hit = {"cached": 200, "last cached": 298}.get(late)
    big = torch.zeros(d)
    big[0] = 24.0
    case.q[20, 1, 0] = 24.0
    if hit is not None:
        pg, s = case.at(0, hit)
        case.k[pg, 0, s] = big.to(case.dt)
        case.quantise()
    else:
        case.kn[20 if sumi else 15, 0] = big.to(case.dt)
    dev = Device8(case)
    dev.attend()
    check8(case, dev)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf, 3.0e38])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cached,chunk,at", [(20, 100, 50), (4, 7, 3), (260, 150, 140)])
def test_a_token_has_no_influence_on_rows_that_do_not_see_it(d, bad, cached, chunk, at, batch):
    clean, case = (Case8([cached], [chunk], d=d, seed=5) for _ in range(2))
    for name in ("kn", "vn"):
        getattr(case, name)[at:] = bad
    a, b = Device8(clean), Device8(case)
    a.attend(), b.attend()
    x, y = a.out(), b.out()
    assert torch.equal(x[:at], y[:at])
    # a token's infinite value reaches the rows that do see it
    if not math.isfinite(bad):
        only = Case8([cached], [chunk], d=d, seed=5)
        only.vn[at, 1, 7] = bad
        dev = Device8(only)
        dev.attend()
        z = dev.out()
        assert torch.equal(z[:at], x[:at])
        odd = z[at:, 2:, 7]                               # (heads 2 and 3 read cache head 1)
        assert (torch.isnan(odd) if math.isnan(bad) else odd == bad).all()
        z[at:, 2:, 7] = x[at:, 2:, 7]
        assert torch.equal(z, x)
        only.append()
        check_cache(only, dev)                            # it is held as no number, and its neighbours as they are


def test_a_cached_token_that_is_no_number_reaches_every_row():
    case = Case8([40], [3], seed=6)
    pg, s = case.at(0, 17)
    case.codes["v"][pg, 1, s, 9] = 0xFF
    dev = Device8(case)
    dev.attend()
    got = dev.out()
    assert torch.isnan(got[:, 2:, 9]).all() and torch.isfinite(got[:, :2]).all()


def test_candidates_do_not_see_each_other(batch):
    clean, case = Case8([70], [90], sumi=True, seed=6), Case8([70], [90], sumi=True, seed=6)
    case.kn[30] = math.nan
    case.vn[31] = math.inf
    a, b = Device8(clean), Device8(case)
    a.attend(), b.attend()
    x, y = a.out(), b.out()
    keep = [i for i in range(90) if i not in (30, 31)]
    assert torch.equal(x[keep], y[keep])
    assert torch.isnan(y[30]).all() and (y[31] == math.inf).all()
    case.kn[:, :, 0] = -math.inf                          # an own logit of -inf: the row is the history's alone
    case.q[:, :, 0] = 1.0
    case.kn[:, :, 1:], case.vn[31] = 0.0, 0.0
    dev = Device8(case)
    dev.attend()
    assert torch.isfinite(dev.out()).all()


@pytest.mark.parametrize("d", [64, 128])
def test_a_block_that_grows_is_rounded_again(d):
    # token by token with magnitudes from 2^-133 to 2^126 in any order, some zero, and tokens too small for their block's scale
    case = Case8([0, 5], [1, 1], d=d, page=16, free=14, seed=7)
    case.table = torch.cat([case.table, torch.full((2, 6), -1, dtype=torch.int32)], dim=1)
    used = set(case.table[case.table >= 0].tolist())
    left = [p for p in range(case.n_pages) if p not in used]
    for b in range(2):
        for i in range(4):
            if case.table[b, i] < 0:
                case.table[b, i] = left.pop()
    dev = Device8(case, stamp=True, max_len=64)
    g = torch.Generator().manual_seed(8)
    size = [2.0 ** e for e in (0, -3, 4, -133, 9, -20, 126, 0, -9, -9, 100, 3, 0.2, 0.7, 1.3, 2.6, -60, -117, -110, -126)]
    for step in range(40):
        for x, to in ((case.kn, dev.kn), (case.vn, dev.vn)):
            x.copy_((torch.rand(x.shape, generator=g) * 2 - 1) * (size[step % len(size)] if step % 7 else 0.0))
            to.copy_(x)
        dev.history()
        case.append()
        check_cache(case, dev)
        dev.len += 1
        case.cached = [c + 1 for c in case.cached]


def test_chunks_that_end_anywhere_give_the_same_cache_as_their_parts():
    # (values of one magnitude: a block's scale may differ on the way, what is rounded again is exact here but for the smallest)
    case = Case8([0], [150], seed=8, page=32)
    dev = Device8(case)
    at, o = 0, case.expect()[0]
    for size in (1, 40, 1, 64, 3, 41):
        dev.off.copy_(torch.tensor([0, size]))
        dev.m_max = size
        q, kn, vn, scen, beh, out = (x[at:at + size] for x in (dev.q, dev.kn, dev.vn, dev.scen, dev.beh, dev.o))
        dev.P.climber_attn_history_paged8(dev.cfg, dev.tau, dev.kv, q, kn, vn, dev.off, size, size, scen, beh, None, out, dev.ws)
        dev.len += size
        at += size
    assert at == 150
    got = dev.out()
    # cached values are off by half a step of e4m3, 2^-4 of theirs at most, and logits by as much of sum |q||k| c
    assert (got - o).abs().max() < 0.35 and (got - o).square().mean().sqrt() < 0.03
    whole = Device8(case)
    whole.attend()
    torch.cuda.synchronize()
    for name in ("k", "v"):
        assert torch.equal(getattr(dev, name + "_scale")[case.table[0, :4].long()], getattr(whole, name + "_scale")[case.table[0, :4].long()])
        for b in range(150):
            pg, s = case.at(0, b)
            a, c = (decode(getattr(x, name)[pg, :, s].cpu().numpy()) for x in (dev, whole))
            assert np.all(np.abs(a - c) <= 2.0 ** -9)     # one step of the smallest codes


def test_slots_behind_max_len_are_not_stored(batch):
    case = Case8([60, 20], [30, 9], page=16, seed=9)
    dev = Device8(case, stamp=True, max_len=70)
    dev.attend()
    torch.cuda.synchronize()
    case.append(limit=70)
    check_cache(case, dev)


def test_lengths_and_page_numbers_that_break_the_contract_stay_in_bounds():
    case = Case8([30, 40], [4, 4], seed=10)
    dev = Device8(case, stamp=True)
    status = torch.zeros(1, dtype=torch.int32, device="cuda:0")
    dev.P.climber_check_paged(dev.cfg, dev.kv.kv, dev.off, case.m, dev.m_max, True, status)
    assert status.item() == 0
    dev.table[0, :] = 10 ** 6
    dev.table[1, :] = -5
    dev.len.copy_(torch.tensor([-3, 10 ** 9]))
    dev.P.climber_check_paged(dev.cfg, dev.kv.kv, dev.off, case.m, dev.m_max, True, status)
    assert status.item() == dev.P.BAD_PAGE | dev.P.BAD_LEN
    dev.history()
    dev.sumi()
    check_cache(case, dev)                                # a token without a page is not stored
    dev.off.copy_(torch.tensor([3, 2, 10 ** 9]))
    dev.history()
    dev.sumi()
    torch.cuda.synchronize()


@pytest.mark.parametrize("sumi", [False, True], ids=["history", "sumi"])
@pytest.mark.parametrize("n_seqs,cached,chunk,Hkv", [(70, 150, 36, 8), (300, 40, 1, 2), (16, 600, 70, 2), (70, 150, 100, 8), (20, 1500, 200, 1)])
def test_batches_of_very_different_lengths(n_seqs, cached, chunk, Hkv, sumi):
    g = torch.Generator().manual_seed(50)
    lens, rows = (torch.randint(lo, hi + 1, (n_seqs,), generator=g).tolist() for lo, hi in ((0, cached), (int(chunk == 1), chunk)))
    case = Case8(lens, rows, H=8, Hkv=Hkv, page=32, sumi=sumi, seed=52, tail=3)
    dev = Device8(case, max_len=2000, pad_o=64)
    wide = torch.full((n_seqs, 63), 10 ** 8, dtype=torch.int32, device="cuda:0")
    wide[:, :dev.table.shape[1]] = dev.table
    dev.table = wide
    dev.describe()
    dev.attend()
    check8(case, dev)


def test_pool_beyond_32_bits(batch):
    # the same calls with their pages behind 4 GiB of others
    case = Case8([130, 40, 0], [5, 40, 17], page=256, d=128, seed=54)
    small, big = Device8(case, stamp=True), Device8(case, stamp=True)
    shift = (1 << 32) // case.codes["k"][0].size + 7
    for name in ("k", "v", "k_scale", "v_scale", "stamp"):
        x = getattr(small, name)
        pool = torch.empty((shift + x.shape[0],) + x.shape[1:], dtype=x.dtype, device="cuda:0")
        pool[shift:] = x
        setattr(big, name, pool)
    big.table = torch.where(small.table >= 0, small.table + shift, small.table)
    big.describe()
    for dev in (small, big):
        dev.history()
        dev.len[:3] += torch.tensor(case.chunk, dtype=torch.int32, device="cuda:0")
    check8(case, small)
    for dev in (small, big):
        dev.sumi()
    torch.cuda.synchronize()
    assert torch.equal(small.o, big.o)
    for name in ("k", "v", "k_scale", "v_scale", "stamp"):
        assert torch.equal(getattr(small, name), getattr(big, name)[shift:])


@pytest.mark.parametrize("chunk", [[1, 1, 1], [40, 3, 0]], ids=["decode", "chunks"])
def test_captured_steps_of_two_caches(chunk, batch):
    # one graph per cache, with a workspace each: append, lengths, scores; replays alternate, with eager work between them
    def start(seed):
        case = Case8([60, 30, 200], chunk, H=8, seed=seed, free=8)
        table = torch.full((3, 30), -1, dtype=torch.int32)
        n, at = case.table.shape[1], case.n_pages
        table[:, :n] = case.table
        for b in range(3):
            for i in range(30):
                if table[b, i] < 0:
                    table[b, i], at = at, at + 1
        for name in ("k", "v"):
            case.codes[name] = np.concatenate([case.codes[name], np.full((at - case.n_pages,) + case.codes[name].shape[1:], 0x7F, np.uint8)])
            case.scales[name] = np.concatenate([case.scales[name], np.full((at - case.n_pages,) + case.scales[name].shape[1:], 255, np.uint8)])
        case.stamp = torch.full((at, case.page), -7, dtype=torch.int32)
        case.table, case.n_pages = table, at
        return Device8(case, stamp=True, max_len=480)

    def step(dev, stream=None):
        dev.history(stream)
        dev.len[:3] += more
        dev.sumi(stream)

    more = torch.tensor(chunk, dtype=torch.int32, device="cuda:0")
    plain, captured, graphs = [start(s) for s in (60, 61)], [start(s) for s in (60, 61)], []
    step(start(62))
    torch.cuda.synchronize()
    for dev in captured:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(dev)
        graphs.append(graph)
    for _ in range(5):
        for g in graphs:
            g.replay()
        for dev in plain:
            step(dev)
        torch.cuda.synchronize()
        for a, b in zip(plain, captured):
            for name in ("o", "k", "v", "k_scale", "v_scale", "stamp", "len"):
                assert torch.equal(getattr(a, name), getattr(b, name)), name


def test_other_streams_and_two_calls_at_once():
    cases = [Case8([700], [50], seed=s, page=64) for s in (20, 21)]
    devs = [Device8(c) for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in devs]
    for d, s in zip(devs, streams):
        d.history(s)
    torch.cuda.synchronize()
    for c, d in zip(cases, devs):
        check8(c, d)


def test_same_call_same_bits(batch):
    results = []
    for _ in range(2):
        dev = Device8(Case8([300, 800, 5], [100, 1, 40], H=8, seed=22))
        dev.attend()
        results.append((dev.out(), dev.k.cpu(), dev.v_scale.cpu()))
    assert all(torch.equal(a, b) for a, b in zip(*results))
