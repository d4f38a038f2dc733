"""What a description of a paged cache refuses by itself: calls that do not fit its tensors (no GPU needed)."""
import ctypes as C

import pytest

import paper_2502_09888_amd as P

FAKE = 0x7F0000000000   # 256-byte aligned, never dereferenced on the host
SHAPE = -2


def cfg(**kw):
    return P.Config(**{**dict(n_heads=4, d_head=64, n_scen=8, n_beh=4, dtype=P.BF16, qk_scale=0.125), **kw})


def every_call(c, kv):
    """Codes of the calls on a cache (1: a workspace of some size), none of which gets as far as a launch: workspaces are too small, a status is
    missing."""
    lib, at = P.load_library(), [C.byref(c), FAKE, C.byref(kv), FAKE, 512, FAKE + (1 << 30), FAKE + (2 << 30), 512, FAKE, 4, 4, FAKE, FAKE]
    rest = [FAKE + (3 << 30), 512, FAKE, 0, None]
    return [lib.climber_attn_history_paged(*at, FAKE, *rest), lib.climber_attn_sumi_paged(*at, *rest),
            lib.climber_paged_evict(C.byref(c), C.byref(kv), FAKE, FAKE, None, FAKE, None, FAKE, 0, None),
            lib.climber_check_paged(C.byref(c), C.byref(kv), FAKE, 4, 4, 1, None, None),
            int(lib.climber_paged_workspace_bytes(C.byref(c), C.byref(kv), 4, 4) > 0)]


@pytest.mark.parametrize("dtype,d", [("bfloat16", 64), ("bfloat16", 128), ("float32", 64), ("float32", 128), ("float32", 32)])
def test_a_cache_knows_its_head_width_and_its_type(dtype, d):
    torch = pytest.importorskip("torch")
    pages = torch.zeros(10, 2, 16, d, dtype=getattr(torch, dtype))
    kv = P.paged_kv(pages, pages.clone(), torch.zeros(3, 4, dtype=torch.int32), torch.zeros(3, dtype=torch.int32), 64, mass=torch.zeros(10, 16))
    right = P.F32 if dtype == "float32" else P.BF16
    assert (kv.d_head, kv.elem_bytes) == (d, pages.element_size())
    for t, width in ((P.F32, 32), (P.F32, 64), (P.F32, 128), (P.BF16, 64), (P.BF16, 128)):
        codes = every_call(cfg(d_head=width, dtype=t), kv)
        if (t, width) == (right, d):
            assert SHAPE not in codes and codes[-1] == 1
        else:
            assert codes == [SHAPE] * 4 + [0], (t, width)


def test_a_description_without_them_is_taken_as_it_is():
    kv = P.PagedKV(FAKE, FAKE, FAKE, None, FAKE, FAKE, 10, 16, 2, 3, 4, 64)
    for c in (cfg(), cfg(d_head=128), cfg(dtype=P.F32)):
        assert SHAPE not in every_call(c, kv)
    kv.elem_bytes = 2
    assert SHAPE not in every_call(cfg(), kv) and every_call(cfg(dtype=P.F32), kv) == [SHAPE] * 4 + [0]


def test_a_cache_in_host_memory_reaches_no_kernel(monkeypatch):
    torch = pytest.importorskip("torch")
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    pages = torch.zeros(10, 2, 16, 64, dtype=torch.bfloat16)
    kv = P.paged_kv(pages, pages.clone(), torch.zeros(3, 4, dtype=torch.int32), torch.zeros(3, dtype=torch.int32), 64, mass=torch.zeros(10, 16))
    c = cfg()
    assert P.climber_paged_workspace_bytes(c, kv, 4, 4) > 0       # (needs no device)
    for stream in (None, 0, 5):                                    # (no workspace, no status: nothing would be launched anyway)
        with pytest.raises(ValueError):
            P.climber_attn_history_paged(c, FAKE, kv, FAKE, FAKE, FAKE, FAKE, 4, 4, FAKE, FAKE, None, FAKE, None, stream)
        with pytest.raises(ValueError):
            P.climber_attn_sumi_paged(c, FAKE, kv, FAKE, FAKE, FAKE, FAKE, 4, 4, FAKE, FAKE, FAKE, None, stream)
        with pytest.raises(ValueError):
            P.climber_paged_evict(c, kv, None, FAKE, None, FAKE, None, None, stream)
        with pytest.raises(ValueError):
            P.climber_check_paged(c, kv, FAKE, 4, 4, True, None, stream)
