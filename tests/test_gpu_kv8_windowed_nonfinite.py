"""Windowed attention on an 8-bit cache with a block whose scale is not finite: it reaches the queries that keep one of
the block's tokens, all of their dimensions, and no others -- on every route.  Tolerances of the others as in
test_gpu_kv8_windowed."""
import pytest
import torch

import _kv8_plain as plain
from test_gpu_kv8_windowed import ROUTES, SM, VAR256, _cache, _reference, _tolerance

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lv():
    import paper_2411_17178_amd as m
    m.load_library()
    return m


# the routes there, and one wave per patch of many
ALL = [(r, 1, 2) for r in ROUTES] + [(((9, 10), 4), 8, 40), (((4, 5), 0), 4, 30)]


@pytest.mark.parametrize("route,B,H", ALL, ids=str)
@pytest.mark.parametrize("name", ["k", "v"])
@pytest.mark.parametrize("stored", [False, True])
@pytest.mark.parametrize("value", [NAN, INF])
def test_a_scale_that_is_not_finite_stays_in_its_rows(lv, route, B, H, name, stored, value):
    q_scales, waves = route
    print(f"  windowed kv8 {route} {B}x{H} {name} {value} stored={stored}", flush=True)
    plan = lv.litevar_mask_build(VAR256, 1, None, 0, q_scales, waves_per_group=waves)
    mask = lv.litevar_mask_export_dense(plan)[0].bool()
    g = torch.Generator(device="cuda").manual_seed(21)
    q = torch.randn(B, H, plan.q_len, 64, generator=g, device="cuda").to(torch.bfloat16)
    clean = _cache(lv, VAR256, B, H, 5)
    want, A, S, floor = _reference(clean, q, mask)
    tol = _tolerance(A, S, floor)
    last = 10 if q_scales is None else q_scales[1]
    for scale in (last - 1, 1):
        cache = _cache(lv, VAR256, B, H, 5)
        lo = cache.offsets[scale]
        n = min(64, cache.offsets[scale + 1] - lo)
        if stored:
            k, v = (t[:, :, lo:cache.offsets[scale + 1]].clone() for t in lv.litevar_kv8_load(cache))
            (k if name == "k" else v)[0, 1, n // 2, 9] = value
            others = [t.clone() for t in (cache.k8, cache.k_scale, cache.v8, cache.v_scale)]
            lv.litevar_kv8_store(cache, k, v, (scale, scale + 1))
            codes, scales = (cache.k8, cache.k_scale) if name == "k" else (cache.v8, cache.v_scale)
            bad_codes, bad_scale = codes[0, 1, lo:lo + n].clone(), scales[0, 1, cache.first_block[scale]].clone()
            for t, o in zip((cache.k8, cache.k_scale, cache.v8, cache.v_scale), others):
                t.copy_(o)
            codes[0, 1, lo:lo + n], scales[0, 1, cache.first_block[scale]] = bad_codes, bad_scale
        else:
            (cache.k_scale if name == "k" else cache.v_scale)[0, 1, cache.first_block[scale]] = value
        out = lv.litevar_windowed_attn_kv8_fwd(plan, q, cache, SM)
        hit = torch.zeros(B, H, plan.q_len, dtype=torch.bool, device="cuda")
        hit[0, 1] = mask[:, lo:lo + n].any(-1)
        assert bool(hit.any())
        plain.assert_close(out[~hit], want[~hit], tol[~hit])
        assert not bool(torch.isfinite(out[hit]).any())
        if value != value or stored:
            assert bool(torch.isnan(out[hit]).all())


@pytest.mark.parametrize("route,B,H", ALL, ids=str)
def test_an_infinite_k_scale_under_negative_products(lv, route, B, H):
    """Every score of the block is -inf: no weight, were the scale not taken for NaN."""
    q_scales, waves = route
    plan = lv.litevar_mask_build(VAR256, 1, None, 0, q_scales, waves_per_group=waves)
    mask = lv.litevar_mask_export_dense(plan)[0].bool()
    g = torch.Generator(device="cuda").manual_seed(22)
    q = -torch.randn(B, H, plan.q_len, 64, generator=g, device="cuda").abs().to(torch.bfloat16)
    k, v = (torch.randn(B, H, 680, 64, generator=g, device="cuda") for _ in range(2))
    cache = lv.litevar_kv8_store(lv.litevar_kv8_cache([s * s for s in VAR256], B, H), k.abs() + 0.5, v)
    want, A, S, floor = _reference(cache, q, mask)
    tol = _tolerance(A, S, floor)
    scale = (10 if q_scales is None else q_scales[1]) - 1
    lo = cache.offsets[scale]
    cache.k_scale[0, 1, cache.first_block[scale]] = INF
    out = lv.litevar_windowed_attn_kv8_fwd(plan, q, cache, SM)
    hit = torch.zeros(B, H, plan.q_len, dtype=torch.bool, device="cuda")
    hit[0, 1] = mask[:, lo:min(lo + 64, cache.offsets[scale + 1])].any(-1)
    plain.assert_close(out[~hit], want[~hit], tol[~hit])
    assert bool(torch.isnan(out[hit]).all())


@pytest.mark.parametrize("route,B,H", ALL, ids=str)
@pytest.mark.parametrize("whole", [False, True])
def test_a_query_of_nan_stays_in_its_row(lv, route, B, H, whole):
    q_scales, waves = route
    plan = lv.litevar_mask_build(VAR256, 2, None, 0, q_scales, waves_per_group=waves)
    cache = _cache(lv, VAR256, B, H, 5)
    g = torch.Generator(device="cuda").manual_seed(23)
    q = torch.randn(B, H, plan.q_len, 64, generator=g, device="cuda").to(torch.bfloat16)
    want, A, S, floor = _reference(cache, q, lv.litevar_mask_export_dense(plan)[0].bool())
    tol = _tolerance(A, S, floor)
    for i in (0, plan.q_len - 1):
        bad = q.clone()
        bad[0, 1, i, slice(None) if whole else 7] = NAN
        out = lv.litevar_windowed_attn_kv8_fwd(plan, bad, cache, SM)
        assert bool(torch.isnan(out[0, 1, i]).all())
        out[0, 1, i] = want[0, 1, i].to(torch.bfloat16)
        plain.assert_close(out, want, tol)
