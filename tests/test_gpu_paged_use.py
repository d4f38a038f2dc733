"""Calls on the paged history cache as a program makes them: batches of very different lengths, large pools, captured steps, extreme values
(against paged_ref.py's definitions in 64 bits, or against the same call made plainly, bit by bit)."""
import math

import pytest
import torch

from paged_ref import Case, Device
from test_gpu_paged import check, evict, same_bits

pytestmark = pytest.mark.gpu


def ragged(n, most, seed, least=0):
    return torch.randint(least, most + 1, (n,), generator=torch.Generator().manual_seed(seed)).tolist()


@pytest.mark.parametrize("sumi", [False, True], ids=["history", "sumi"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_seqs,cached,chunk,Hkv", [(70, 150, 36, 8), (300, 40, 1, 2), (16, 600, 70, 2)])
def test_batches_of_very_different_lengths(n_seqs, cached, chunk, Hkv, dtype, sumi):
    # enough workgroups that sequences take turns by their work, over more than one set of 64 of them
    case = Case(ragged(n_seqs, cached, 50), [min(c, chunk) for c in ragged(n_seqs, chunk, 51, least=int(chunk == 1))], H=8, Hkv=Hkv, page=32,
                dtype=dtype, sumi=sumi, seed=52, tail=3)
    dev = Device(case, mass=True, max_len=2000, pad_o=64)
    # (a table of 2000 tokens)
    wide = torch.full((n_seqs, 63), 10 ** 8, dtype=torch.int32, device="cuda:0")
    wide[:, :dev.table.shape[1]] = dev.table
    dev.table = wide
    dev.describe()
    dev.attend()
    check(case, dev)


@pytest.mark.parametrize("sumi", [False, True], ids=["history", "sumi"])
@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("std,values", [(4.0, 1e30), (1.0, 1e32), (4.0, 1e-30)])
def test_large_and_small_values(dtype, d, std, values, sumi):
    # weights of later keys that exceed those of the first by 2^30 and more, on values with which unscaled sums pass 2^128; 700 tokens
    # of at most 6e32 stay below 2^119
    case = Case([500, 33], [90, 4], d=d, std=std, dtype=dtype, sumi=sumi, seed=53)
    case.v, case.vn = (case.v.float() * values).to(case.dt), (case.vn.float() * values).to(case.dt)
    dev = Device(case, mass=True)
    dev.attend()
    check(case, dev)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pool_beyond_32_bits(dtype):
    # the same call with its pages behind 4 GiB of others
    case = Case([130, 40, 0], [5, 40, 17], page=256, dtype=dtype, seed=54)
    small = Device(case, mass=True, stamp=True)
    big = Device(case, mass=True, stamp=True)
    page_bytes = case.k[0].numel() * case.k.element_size()
    shift = (1 << 32) // page_bytes + 7
    for name in ("k", "v", "mass", "stamp"):
        x = getattr(small, name)
        pool = torch.empty((shift + x.shape[0],) + x.shape[1:], dtype=x.dtype, device="cuda:0")
        pool[shift:] = x
        setattr(big, name, pool)
    big.table = torch.where(small.table >= 0, small.table + shift, small.table)
    big.describe()
    budget = torch.tensor([100, 50, 9], dtype=torch.int32, device="cuda:0")
    for dev in (small, big):
        dev.history()
        dev.len += torch.tensor(case.chunk, dtype=torch.int32, device="cuda:0")
    check(case, small)
    for step in range(2):
        assert same_bits(small.o, big.o)
        for name in ("k", "v", "mass", "stamp"):
            assert same_bits(getattr(small, name), getattr(big, name)[shift:])
        for dev in (small, big):
            if step == 0:
                dev.P.climber_paged_evict(dev.cfg, dev.kv, None, budget, None, dev.len, None, dev.ws)
                dev.sumi()
    assert torch.equal(small.len, big.len) and small.len.tolist() == [100, 50, 9]


@pytest.mark.parametrize("chunk", [[1, 1, 1], [40, 3, 0]], ids=["decode", "chunks"])
def test_captured_step_of_append_score_and_evict(chunk):
    # One graph per cache: append, lengths, scores, cut.  Two caches with a workspace each; replays alternate, with eager work between them.
    def start(seed):
        return Device(Case([60, 30, 200], chunk, H=8, seed=seed, free=8), mass=True, stamp=True, max_len=256)

    def wide(dev):
        table = torch.empty(3, 16, dtype=torch.int32, device="cuda:0")
        table[:] = torch.arange(48, device="cuda:0").view(3, 16)
        n = dev.table.shape[1]
        for name in ("k", "v", "mass", "stamp"):
            x = getattr(dev, name)
            pool = torch.full((48,) + x.shape[1:], math.nan if x.is_floating_point() else -7, dtype=x.dtype, device="cuda:0")
            for b in range(3):
                for j in range(n):
                    if dev.table[b, j] >= 0:
                        pool[b * 16 + j] = x[dev.table[b, j]]
            setattr(dev, name, pool)
        dev.table = table
        dev.describe()
        return dev

    def step(dev, budget, more, stream=None):
        dev.history(stream)
        dev.len += more
        dev.sumi(stream)
        dev.P.climber_paged_evict(dev.cfg, dev.kv, None, budget, None, dev.len, None, dev.ws, stream)

    more = torch.tensor(chunk, dtype=torch.int32, device="cuda:0")
    budget = torch.tensor([50, 31, 150], dtype=torch.int32, device="cuda:0")
    plain, captured = [wide(start(s)) for s in (60, 61)], [wide(start(s)) for s in (60, 61)]
    graphs = []
    step(wide(start(62)), budget, more)
    torch.cuda.synchronize()
    for dev in captured:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(dev, budget, more)
        graphs.append(graph)
    for _ in range(4):
        for g in graphs:
            g.replay()
        for dev in plain:
            step(dev, budget, more)
        torch.cuda.synchronize()
        for a, b in zip(plain, captured):
            for name in ("o", "k", "v", "mass", "stamp", "len"):
                assert same_bits(getattr(a, name).contiguous(), getattr(b, name).contiguous()), name
    assert plain[0].len.tolist() == [50, 31, 150]


@pytest.mark.parametrize("max_len", [1024, 5000, 16384, 16385, 60000])
def test_evict_of_short_sequences_in_large_tables(max_len):
    case = Case([0, 1, 5, 64, 65, 200, 777], [1] * 7, sumi=True, seed=55)
    table = torch.full((7, -(-max_len // 16)), -1, dtype=torch.int32)
    table[:, :case.table.shape[1]] = case.table
    case.table = table
    evict(case, [3, 1, 2, 33, 64, 150, 300], max_len=max_len)
    evict(case, [0, 0, 5, 1, 65, 199, 776], max_len=max_len, keep_from=[0, 9, 3, 40, 64, 100, 700], in_place=True)


@pytest.mark.parametrize("n", [300, 20000])
def test_new_lengths_in_place_of_the_budget(n):
    case = Case([n, 5], [1, 1], H=1, Hkv=1, d=4, dtype="f32", page=64, sumi=True, seed=56)
    dev, other = Device(case, mass=True), Device(case, mass=True)
    budget = torch.tensor([n // 3, 9], dtype=torch.int32, device="cuda:0")
    out = torch.zeros_like(budget)
    dev.P.climber_paged_evict(dev.cfg, dev.kv, None, budget, None, out, None, dev.ws)
    other.P.climber_paged_evict(other.cfg, other.kv, None, budget, None, budget, None, other.ws)
    torch.cuda.synchronize()
    assert out.tolist() == budget.tolist() == [n // 3, 5]
    assert same_bits(dev.k, other.k) and same_bits(dev.v, other.v) and same_bits(dev.mass, other.mass)


def test_check_allows_rows_of_no_sequence():
    case = Case([30, 0, 7], [4, 0, 2], seed=57, tail=5)
    dev = Device(case)
    status = torch.zeros(1, dtype=torch.int32, device="cuda:0")
    for appends in (True, False):
        dev.P.climber_check_paged(dev.cfg, dev.kv, dev.off, case.m, dev.m_max, appends, status)
    assert status.item() == 0
    dev.off[3] = case.m + 1
    dev.P.climber_check_paged(dev.cfg, dev.kv, dev.off, case.m, dev.m_max, False, status)
    assert status.item() == dev.P.BAD_OFFSETS | dev.P.BAD_M_MAX
