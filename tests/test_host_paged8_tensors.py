"""Tensors that the attention calls on a cache in 8 bits do not read as they are: refused before anything would be launched, so no GPU is needed."""
import pytest

import paper_2502_09888_amd as P

torch = pytest.importorskip("torch")


class On0:
    """A tensor as one on device 0 appears to the calls."""

    def __init__(self, t):
        self.t = t

    def __getattr__(self, name):
        return getattr(self.t, name)

    def get_device(self):
        return 0


def cache(max_len=64, n_seqs=3, **kw):
    pages = [torch.zeros(10, 2, 32, 64, dtype=torch.uint8) for _ in range(2)] + [torch.zeros(10, 2, 2, dtype=torch.uint8) for _ in range(2)]
    kv8 = P.paged_kv8(*pages, torch.zeros(n_seqs, 4, dtype=torch.int32), torch.zeros(n_seqs, dtype=torch.int32), max_len, **kw)
    kv8._device = 0
    return kv8


CFG = dict(n_heads=4, d_head=64, n_scen=2, n_beh=3, dtype=P.BF16)
M = 6


def arguments(sumi):
    t = dict(tau_layer=torch.ones(2, 3), q=torch.zeros(M, 4, 64).bfloat16(), k=torch.zeros(M, 128).bfloat16(), v=torch.zeros(M, 2, 64).bfloat16(),
             off=torch.zeros(4, dtype=torch.int32), scen=torch.zeros(M, dtype=torch.int32), beh=torch.zeros(M, dtype=torch.int32),
             stamp=torch.zeros(M, dtype=torch.int32), o=torch.zeros(M, 256).bfloat16())
    if sumi:
        del t["stamp"]
    return t


def attend(sumi, t, kv8, m_total=M, native=True):
    """Every argument in order: the entry point is reached, and refuses the workspace, which is not where it has to be."""
    from paper_2502_09888_amd import climber
    t = {n: On0(x) if isinstance(x, torch.Tensor) else x for n, x in t.items()}
    ws = torch.zeros(1024, dtype=torch.uint8)
    ws = On0(ws[(1 - ws.data_ptr()) % 256:])
    f = P.climber_attn_sumi_paged8 if sumi else P.climber_attn_history_paged8
    given = [t["tau_layer"], kv8, t["q"], t["k"], t["v"], t["off"], m_total, min(m_total, 4), t["scen"], t["beh"], *([] if sumi else [t["stamp"]]), t["o"], ws]
    if native:
        return f(P.Config(**CFG), *given, stream=0)
    was = climber._native

    class ByCtypes:
        attn_history_paged8 = attn_sumi_paged8 = staticmethod(lambda *a: None)
    climber._native = ByCtypes
    try:
        return f(P.Config(**CFG), *given, stream=0)
    finally:
        climber._native = was


@pytest.fixture(autouse=True)
def loaded():
    from paper_2502_09888_amd import climber
    climber._native or climber._load_native(P.load_library())


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("sumi", [False, True])
def test_tensors_of_other_types_or_sizes_are_refused(sumi, native):
    right = arguments(sumi)
    with pytest.raises(P.ClimberError) as e:
        attend(sumi, right, cache(), native=native)
    assert e.value.code == -3, e.value
    wrong = {"tau_layer": [torch.ones(2, 3).double(), torch.ones(2, 3).bfloat16(), torch.ones(5), torch.ones(3, 2).t()]}
    for name in ("off", "scen", "beh", "stamp"):
        n = 4 if name == "off" else M
        wrong[name] = [torch.zeros(n, dtype=torch.int64), torch.zeros(n), torch.zeros(4 * n, dtype=torch.uint8), torch.zeros(n - 1, dtype=torch.int32),
                       torch.zeros(n, 2, dtype=torch.int32)[:, 0]]
    for name, wide in (("q", 256), ("k", 128), ("v", 128), ("o", 256)):
        wrong[name] = [torch.zeros(M, wide), torch.zeros(M, wide).half(), torch.zeros(M, wide, dtype=torch.int16), torch.zeros(M - 1, wide).bfloat16(),
                       torch.zeros(M, 2 * wide).bfloat16()[:, ::2], torch.zeros(1, M * wide).bfloat16()]
        if name in "qo":
            wrong[name].append(torch.zeros(M, 256).bfloat16()[:, :248])
    for name, bad in wrong.items():
        if name not in right:
            continue
        for x in bad:
            with pytest.raises(ValueError):
                attend(sumi, {**right, name: x}, cache(), native=native)
    both = torch.zeros(M, 256).bfloat16()                 # (k and v of one pitch, narrower than a row)
    with pytest.raises(ValueError):
        attend(sumi, {**right, "k": both[:, :120], "v": both[:, 128:248]}, cache(), native=native)


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("sumi", [False, True])
def test_what_is_right_is_taken(sumi, native):
    right = arguments(sumi)
    packed = torch.zeros(M + 3, 512).bfloat16()
    longer = dict(tau_layer=torch.ones(40), q=packed[:, :256], k=packed[:, 256:384], v=packed[:, 384:].unflatten(1, (2, 64)), o=torch.zeros(M + 1, 4, 64).bfloat16(),
                  off=torch.zeros(9, dtype=torch.int32), scen=torch.zeros(M + 1, dtype=torch.int32), beh=torch.zeros(2, M, dtype=torch.int32))
    if not sumi:
        longer["stamp"] = torch.zeros(M + 2, dtype=torch.int32)
    with pytest.raises(P.ClimberError) as e:
        attend(sumi, longer, cache(), native=native)
    assert e.value.code == -3
    # pointers, and no stamps
    for name, x in right.items():
        with pytest.raises(P.ClimberError) as e:
            attend(sumi, {**right, name: None if name == "stamp" else 0x55AA0000}, cache(), native=native)
        assert e.value.code in (-3, -4)
    # no rows: nothing is read
    attend(sumi, {n: torch.zeros(0) if n not in ("off", "tau_layer") else x for n, x in right.items()} | {"q": None, "k": None, "v": None, "o": None},
           cache(), m_total=0, native=native)
