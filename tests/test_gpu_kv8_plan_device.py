"""A plan whose blob lies on another device than the operands is refused."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_a_plan_of_another_device_is_refused():
    import paper_2411_17178_amd as lv
    plan = lv.litevar_mask_build((1, 2, 4), 1)
    cache = lv.litevar_kv8_cache([1, 4, 16], 1, 2)
    q = torch.zeros(1, 2, 21, 64, dtype=torch.bfloat16, device="cuda")
    lv.litevar_windowed_attn_kv8_fwd(plan, q, cache, 0.125)
    with pytest.raises(AssertionError):
        lv.litevar_windowed_attn_kv8_fwd(lv.Plan(plan.handle, plan.blob.cpu()), q, cache, 0.125)
