"""Windowed attention on an 8-bit cache whose values lie at the ends of their type's range, on every route.  Tolerances
as in test_gpu_kv8_windowed."""
import pytest
import torch

import _kv8_plain as plain
from test_gpu_kv8_windowed import ROUTES, SM, VAR256, _reference, _tolerance

pytestmark = pytest.mark.gpu
# the routes there, and one wave per patch of many
ALL = [(r, 1, 2) for r in ROUTES] + [(((9, 10), 4), 8, 40), (((4, 5), 0), 4, 30)]


@pytest.fixture(scope="module")
def lv():
    import paper_2411_17178_amd as m
    m.load_library()
    return m


def _run(lv, route, k, v, q, sm=SM):
    q_scales, waves = route
    B, H = k.shape[:2]
    plan = lv.litevar_mask_build(VAR256, 3, None, 0, q_scales, waves_per_group=waves)
    cache = lv.litevar_kv8_store(lv.litevar_kv8_cache([s * s for s in VAR256], B, H), k, v)
    q = q[:, :, :plan.q_len].to(torch.bfloat16)
    out = lv.litevar_windowed_attn_kv8_fwd(plan, q, cache, sm)
    want, A, S, floor = _reference(cache, q, lv.litevar_mask_export_dense(plan)[0].bool(), sm)
    plain.assert_close(out, want, _tolerance(A, S, floor))


def _randn(shape, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda")


@pytest.mark.parametrize("route,B,H", ALL, ids=str)
@pytest.mark.parametrize("power,some", [(-105.5, 1.0), (-115.5, 1.0), (-115.5, 2.0 ** 50), (-120.5, 1.0), (-120.5, 2.0 ** 50), (120.0, 1.0),
                                        (120.0, 2.0 ** -50)])
def test_v_near_the_ends_of_its_range(lv, route, B, H, power, some):
    """All of V around 2^-120.5, which bf16 holds as normal numbers, with block scales below 2^-126, or near the largest;
    a third of the last scale's blocks at another size."""
    q, k, v = (_randn((B, H, 680, 64), i) for i in range(3))
    v = 1 + 0.2 * v
    v[:, :, 424 + 64:424 + 128] *= some
    v[:, :, 5:14] *= some
    _run(lv, route, k, v * 2.0 ** power, q)
