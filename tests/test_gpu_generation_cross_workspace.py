"""The workspace of a conditioned layer's cross attention, one for all steps."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,H,H_kv,states_len", [(3, 23, 1, 6000), (2, 32, 8, 4099), (2, 4, 4, 77)])
def test_one_workspace_serves_every_step(B, H, H_kv, states_len):
    import paper_2411_17178_amd as lv
    from paper_2411_17178_amd.generation import GenerationLayer
    gen = GenerationLayer((1, 2, 3, 4, 5, 6, 8, 10, 13, 16), 3)
    sizes = [lv.litevar_cross_attn_workspace_bytes(B, H, H_kv, s * s, states_len) for s in gen.scales]
    assert gen.cross_workspace_bytes(B, H, H_kv, states_len) == max(sizes)
    assert (states_len < 1000) or sizes[-1] < max(sizes)                     # (the last step's own would not do)
    work = torch.empty(max(sizes), dtype=torch.uint8, device="cuda")
    k, v = (torch.randn(B, H_kv, states_len, 64, device="cuda").to(torch.bfloat16) for _ in range(2))
    cache = lv.litevar_kv8_store(lv.litevar_kv8_cache([states_len], B, H_kv), k, v)
    for s in gen.scales:
        q = torch.randn(B, H, s * s, 64, device="cuda").to(torch.bfloat16)
        for states in ((k, v), cache):
            assert torch.equal(gen.cross(q, states, 0.125, workspace=work), gen.cross(q, states, 0.125))
