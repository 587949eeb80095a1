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


@pytest.mark.parametrize("side", [16, 32], ids=["in_the_kernel", "through_a_copy"])
def test_long_flat_tails_keep_their_weight(lv, side):
    """One key with nearly all the weight, 16 639 of 2^-21 of it each, in a row's first steps or in its last: the tail's sum
    is 0.7 %, and all of the result.  A weight is off by its f16's last bit, 2^-24, over a row's sum of at least 2, so that
    the result of n keys of |v| <= 1 is off by 2^-25 (n + n |out|) <= 2^-24 n besides the relative roundings."""
    scales = (128, side)
    n = 128 * 128 + side * side
    plan = lv.litevar_mask_build(scales, -1, None, 0, (1, 2), waves_per_group=16)
    assert (lv.litevar_windowed_attn_kv8_workspace_bytes(plan, 1, 1) > 0) == (side == 32)
    for sink in (0, 5000, n - 1):
        q, k, v = torch.zeros(1, 1, side * side, 64, device="cuda"), torch.zeros(1, 1, n, 64, device="cuda"), torch.ones(1, 1, n, 64, device="cuda")
        q[..., 0], k[..., 0] = 8.0, -16.67                                   # (scores: 2^-24.05, and 2^-2.8)
        k[:, :, sink, 0], v[:, :, sink] = -1.97, 0
        cache = lv.litevar_kv8_store(lv.litevar_kv8_cache([s * s for s in scales], 1, 1), k, v)
        q = q.to(torch.bfloat16)
        out = lv.litevar_windowed_attn_kv8_fwd(plan, q, cache, SM)
        want, A, S, _ = _reference(cache, q, torch.ones(side * side, n, dtype=torch.bool, device="cuda"))
        assert 0.005 < want.min().item() <= want.max().item() < 0.01
        plain.assert_close(out, want, (3.25 * plain.U + 2 * torch.expm1(2.0 ** -11 * S)) * A + 2.0 ** -24 * n)
