"""Tensors on the GPU that the attention calls on a cache in 8 bits do not read as they are: refused, and nothing is written."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("sumi", [False, True])
def test_other_types_and_sizes_are_refused_and_write_nothing(sumi):
    import paper_2502_09888_amd as P
    dev, m = "cuda:0", 5
    k = torch.zeros((4, 2, 16, 64), dtype=torch.uint8, device=dev)
    v, ks = k.clone(), torch.full((4, 2, 1), 127, dtype=torch.uint8, device=dev)
    vs = ks.clone()
    kv = P.paged_kv8(k, v, ks, vs, torch.tensor([[0, 1], [2, 3]], dtype=torch.int32, device=dev), torch.tensor([3, 4], dtype=torch.int32, device=dev), 32)
    cfg = P.Config(n_heads=4, d_head=64, n_scen=1, n_beh=1, dtype=P.BF16)
    ints = dict(dtype=torch.int32, device=dev)
    right = dict(tau=torch.ones((1, 1), device=dev), q=torch.ones((m, 4, 64), device=dev).bfloat16(), k=torch.ones((m, 128), device=dev).bfloat16(),
                 v=torch.ones((m, 2, 64), device=dev).bfloat16(), off=torch.tensor([0, 2, 5], **ints), scen=torch.zeros(m, **ints),
                 beh=torch.zeros(m, **ints), o=torch.full((m, 256), 7.0, device=dev).bfloat16())
    ws = torch.empty(P.climber_paged8_workspace_bytes(cfg, kv, m, 3), dtype=torch.uint8, device=dev)

    def attend(t):
        a = (cfg, t["tau"], kv, t["q"], t["k"], t["v"], t["off"], m, 3, t["scen"], t["beh"])
        P.climber_attn_sumi_paged8(*a, t["o"], ws) if sumi else P.climber_attn_history_paged8(*a, None, t["o"], ws)
    for name, x in right.items():
        for bad in ((x.long(), x.double(), x.reshape(-1)[:-1]) if name in ("off", "scen", "beh") else
                    (x.double(), x.half(), x[:-1])):
            with pytest.raises(ValueError):
                attend({**right, name: bad})
    torch.cuda.synchronize()
    assert bool((right["o"].float() == 7).all()) and not k.any() and not v.any()
    attend(right)
    torch.cuda.synchronize()
    assert bool((right["o"].float() <= 1.01).all())
