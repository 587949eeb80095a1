"""Windowed attention on the 8-bit cache against the formula in 64 bits on the cache's own values.

Tolerance, element by element (A = sum of weights x |v|, S = the row's largest sum of |q_d k_d| x sm_scale, U = half a
step of bf16): probabilities rounded, or their products with the V scales, 2 U A; output rounded, U A; V rounded to f16,
2^-11 A = U A / 8; K rounded to f16, which moves a score by 2^-11 S at most and so a weight, the sum included, by the factor
exp(2^-10 S): (exp(2^-10 S) - 1) A, of which the tests allow 2 (exp(2^-11 S) - 1) A, which is less.  Sums in 32 bits: below U A / 8.
Probabilities in f16 have an absolute floor as well: their last bit is 2^-24 below 2^-14, and a row's sum is at least
2^-3 (it starts at a reference of 0, and a step that leaves the sum below 2^-3 is formed again under a reference that
makes its largest probability at least 2^-0.5), so a weight is off by 2^-21 at most; over n kept keys with |v| <= V the
result by 2^-21 (n V + n |out|) <= 2^-20 n V."""
import pytest
import torch

import _kv8_plain as plain
import workloads

pytestmark = pytest.mark.gpu
SM = 0.125
VAR256 = workloads.configs.VAR256


@pytest.fixture(scope="module")
def lv():
    import paper_2411_17178_amd as m
    m.load_library()
    return m


def _tolerance(A, S, floor):
    return (3.25 * plain.U + 2 * torch.expm1(2.0 ** -11 * S)) * A + 2.0 ** -20 * floor


def _cache(lv, scales, B, H, seed, seen=None):
    """A cache with the scales before `seen` stored (default: all), nothing usable behind them."""
    seg = [s * s for s in scales]
    seen = len(seg) if seen is None else seen
    cache = lv.litevar_kv8_cache(seg, B, H)
    for t in (cache.k_scale, cache.v_scale):
        t.fill_(float("nan"))
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = cache.offsets[seen]
    k, v = (torch.randn(B, H, n, 64, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    lv.litevar_kv8_store(cache, k, v, (0, seen))
    return cache


def _reference(cache, q, mask, sm=SM):
    kd, vd = (plain.dequantise(c, s, cache.segments) for c, s in ((cache.k8, cache.k_scale), (cache.v8, cache.v_scale)))
    used = mask.any(-2 if mask.dim() == 2 else 1)                            # tokens that some query keeps
    used = used.view(1, -1, mask.shape[-1], 1)
    zero = torch.zeros((), dtype=torch.float64, device="cuda")
    kd, vd = torch.where(used, kd, zero), torch.where(used, vd, zero)
    largest = torch.where(mask, vd.abs().amax(-1)[:, :, None], zero).amax(-1, keepdim=True)   # |v| of a row's kept keys
    return (*plain.attention(q, kd, vd, mask, sm), mask.sum(-1)[..., None] * largest)


CASES = [  # scales, query scales, radius, sink scales, mask mode, batch, heads, plan options
    ((1, 2, 3, 4), None, 1, 0, 0, 1, 1, 0), (VAR256, (0, 1), 3, 0, 0, 2, 3, 0), (VAR256, (3, 4), 2, 0, 0, 2, 16, 0),
    (VAR256, (6, 7), 3, 0, 0, 2, 5, 0), (VAR256, (7, 8), 3, 3, 0, 3, 5, 0), (VAR256, (9, 10), 3, 0, 0, 4, 30, 0),
    (VAR256, (9, 10), 3, 0, 0, 4, 30, 16), (VAR256, (9, 10), 3, 0, 0, 2, 3, (16, 0, 0, -1, 1)),
    (VAR256, None, 2, 0, 0, 2, 16, 0), (VAR256, None, 2, 0, 0, 2, 16, 16), (VAR256, None, -1, 0, 0, 2, 30, 0),
    (VAR256, (9, 10), -1, 0, 0, 2, 30, 0), (VAR256, None, 12, 0, 1, 2, 4, 0), (VAR256, (8, 9), 24, 0, 1, 2, 4, 16),
    ((5, 9, 7, 13), None, 2, 0, 0, 2, 3, 16), ((5, 9, 7, 13), (2, 3), 2, 1, 0, 2, 3, 8), ((1,) * 20 + (12,), (20, 21), 1, 0, 0, 1, 2, 16),
    (workloads.configs.VAR512, None, 4, 0, 0, 2, 6, 0), (workloads.configs.VAR512, (9, 10), 4, 0, 0, 2, 36, 0),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{len(c[0])}x{c[0][-1]}-{c[1]}-r{c[2]}-s{c[3]}-m{c[4]}-{c[5]}x{c[6]}-{c[7]}")
def test_windowed_attention_on_the_cache(lv, case):
    scales, q_scales, radius, sink, mode, B, H, waves = case
    print(f"  windowed kv8 {case}", flush=True)
    plan = lv.litevar_mask_build(scales, radius, None, sink, q_scales, waves_per_group=waves, mask_mode=mode)
    cache = _cache(lv, scales, B, H, 1, None if q_scales is None else q_scales[1])
    g = torch.Generator(device="cuda").manual_seed(2)
    q = torch.randn(B, H, plan.q_len, 64, generator=g, device="cuda").to(torch.bfloat16)
    out = lv.litevar_windowed_attn_kv8_fwd(plan, q, cache, SM)
    mask = lv.litevar_mask_export_dense(plan)[0].bool()
    want, A, S, floor = _reference(cache, q, mask)
    plain.assert_close(out, want, _tolerance(A, S, floor))
    lv.litevar_plan_check(plan)


def test_one_radius_table_per_head(lv):
    K, H, B = len(VAR256), 4, 2
    tables = [[[(h + j) % 4 for j in range(K)] for _ in range(K)] for h in range(H)]
    for waves, q_scales in ((0, (9, 10)), (16, None), (4, (5, 6))):
        plan = lv.litevar_mask_build(VAR256, 0, tables, 0, q_scales, waves_per_group=waves)
        cache = _cache(lv, VAR256, B, H, 3, None if q_scales is None else q_scales[1])
        q = torch.randn(B, H, plan.q_len, 64, device="cuda").to(torch.bfloat16)
        out = lv.litevar_windowed_attn_kv8_fwd(plan, q, cache, SM)
        mask = torch.stack([lv.litevar_mask_export_dense(plan, head=h)[0].bool() for h in range(H)])
        want, A, S, floor = _reference(cache, q, mask)
        plain.assert_close(out, want, _tolerance(A, S, floor))


@pytest.mark.parametrize("waves", [0, 16])
def test_output_sharing_and_strides(lv, waves):
    B, H = 4, 6
    plan = lv.litevar_mask_build(VAR256, 3, None, 0, (9, 10), waves_per_group=waves)
    cache = _cache(lv, VAR256, B, H, 4)
    share = (torch.arange(H)[:, None] % 2 == 0).expand(H, 10).contiguous().to(torch.uint8).cuda()
    q = torch.randn(B, 256, H, 64, device="cuda").to(torch.bfloat16).transpose(1, 2)
    big = torch.full((B, 258, H, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    out = big[:, 1:-1].transpose(1, 2)
    lv.litevar_windowed_attn_kv8_fwd(plan, q, cache, SM, out=out, cfg_share=share)
    alone = lv.litevar_windowed_attn_kv8_fwd(plan, q, cache, SM)
    shared = share[:, 9].bool()
    assert torch.equal(out[:2], alone[:2]) and torch.equal(out[2:, ~shared], alone[2:, ~shared])
    assert torch.equal(out[2:, shared], out[:2, shared])
    assert bool((big[:, 0] == 7).all()) and bool((big[:, -1] == 7).all())


def test_values_that_are_not_finite_stay_in_their_rows(lv):
    """A block whose scale is not finite reaches the queries that keep one of its tokens and no others."""
    B, H = 1, 2
    for waves in (16,):
        plan = lv.litevar_mask_build(VAR256, 1, None, 0, None, waves_per_group=waves)
        cache = _cache(lv, VAR256, B, H, 5)
        block = cache.first_block[9] + 1                                     # tokens 64 .. 127 of the last scale
        cache.v_scale[0, 1, block] = float("inf")
        q = torch.randn(B, H, plan.q_len, 64, device="cuda").to(torch.bfloat16)
        out = lv.litevar_windowed_attn_kv8_fwd(plan, q, cache, SM)
        mask = lv.litevar_mask_export_dense(plan)[0].bool()
        lo = cache.offsets[9] + 64
        hit = mask[:, lo:lo + 64].any(-1)
        clean = _cache(lv, VAR256, B, H, 5)
        want, A, S, floor = _reference(clean, q, mask)
        tol = _tolerance(A, S, floor)
        plain.assert_close(out[:, :1], want[:, :1], tol[:, :1])
        plain.assert_close(out[:, 1, ~hit], want[:, 1, ~hit], tol[:, 1, ~hit])
        assert not bool(torch.isfinite(out[:, 1, hit]).all(-1).any())


def test_whole_generation_with_graph(lv):
    """All steps of a layer, one captured graph each: the scale is stored, then attended to."""
    B, H = 2, 6
    seg = [s * s for s in VAR256]
    plans = [lv.litevar_mask_build(VAR256, 3, None, 0, (k, k + 1)) for k in range(10)]
    full = lv.litevar_mask_build(VAR256, 3)
    mask = lv.litevar_mask_export_dense(full)[0].bool()
    cache = lv.litevar_kv8_cache(seg, B, H)
    q, k, v = (torch.randn(B, H, 680, 64, device="cuda").to(torch.bfloat16) for _ in range(3))
    work = torch.empty(max(lv.litevar_windowed_attn_kv8_workspace_bytes(p, B, H) for p in plans), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)

    def steps():
        for i, p in enumerate(plans):
            lo, hi = cache.offsets[i], cache.offsets[i + 1]
            lv.litevar_kv8_store(cache, k[:, :, lo:hi], v[:, :, lo:hi], (i, i + 1))
            lv.litevar_windowed_attn_kv8_fwd(p, q[:, :, lo:hi], cache, SM, out=out[:, :, lo:hi], workspace=work)
    steps()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        steps()
    for i in range(3):
        q.copy_(torch.randn(q.shape, device="cuda"))
        k.copy_(torch.randn(q.shape, device="cuda"))
        cache.k8.zero_()
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        want, A, S, floor = _reference(cache, q, mask)
        plain.assert_close(out, want, _tolerance(A, S, floor))
        replayed = out.clone()
        steps()
        assert torch.equal(out, replayed)


ROUTES = [((9, 10), 0), (None, 16), (None, 4), ((9, 10), 8)]     # converted in the kernel, through a copy, gathered, gathered


@pytest.mark.parametrize("route", ROUTES, ids=str)
def test_block_scales_far_apart(lv, route):
    """K or V blocks 2^-30, 2^-70 and 2^60 times as large as the others, or of zeros: every value at its own size."""
    q_scales, waves = route
    B, H = 1, 6
    plan = lv.litevar_mask_build(VAR256, 2, None, 0, q_scales, waves_per_group=waves)
    seg = [s * s for s in VAR256]
    cache = lv.litevar_kv8_cache(seg, B, H)
    g = torch.Generator(device="cuda").manual_seed(6)
    k, v = (torch.randn(B, H, 680, 64, generator=g, device="cuda") for _ in range(2))
    lo = cache.offsets[9]
    v[:, 0, lo:lo + 64] *= 2.0 ** -30
    v[:, 1, :lo] *= 2.0 ** -70
    k[:, 2, lo + 64:lo + 128] *= 2.0 ** -30
    k[:, 3, lo:] = 0
    v[:, 4, lo + 64:] = 0
    v[:, 5, lo:lo + 64] *= 2.0 ** 60
    lv.litevar_kv8_store(cache, k, v)
    q = torch.randn(B, H, plan.q_len, 64, generator=g, device="cuda").to(torch.bfloat16)
    out = lv.litevar_windowed_attn_kv8_fwd(plan, q, cache, SM)
    want, A, S, floor = _reference(cache, q, lv.litevar_mask_export_dense(plan)[0].bool())
    plain.assert_close(out, want, _tolerance(A, S, floor))


@pytest.mark.parametrize("route", ROUTES, ids=str)
@pytest.mark.parametrize("shift,spread,size", [(0.0, 0.0, 1.0), (0.0, 6.0, 1.0), (-24.0, 6.0, 1.0), (40.0, 1.0, 1e4), (0.0, 30.0, 1e-4), (-300.0, 1.0, 1.0)])
def test_distributions_of_scores(lv, route, shift, spread, size):
    """Flat, peaked, low and high scores, V of many sizes: the weights keep their relative precision."""
    q_scales, waves = route
    B, H = 1, 3
    plan = lv.litevar_mask_build(VAR256, 3, None, 0, q_scales, waves_per_group=waves)
    cache = lv.litevar_kv8_cache([s * s for s in VAR256], B, H)
    g = torch.Generator(device="cuda").manual_seed(7)
    k, v = (torch.randn(B, H, 680, 64, generator=g, device="cuda") for _ in range(2))
    q = torch.randn(B, H, plan.q_len, 64, generator=g, device="cuda") * spread
    q[..., 0] = 1.0
    k[..., 0] = shift / SM                                # (a score's mean; the codes keep it to half a step)
    lv.litevar_kv8_store(cache, k, v * size)
    q = q.to(torch.bfloat16)
    out = lv.litevar_windowed_attn_kv8_fwd(plan, q, cache, SM)
    want, A, S, floor = _reference(cache, q, lv.litevar_mask_export_dense(plan)[0].bool())
    plain.assert_close(out, want, _tolerance(A, S, floor))


@pytest.mark.parametrize("route", ROUTES, ids=str)
@pytest.mark.parametrize("k_power,v_power", [(0, -100), (0, 110), (-110, 0), (60, -90), (-60, 89)])
def test_values_near_the_ends_of_their_type(lv, route, k_power, v_power):
    """All of K or V very small or very large, queries the other way round: powers of two do not change relative errors."""
    q_scales, waves = route
    B, H = 1, 2
    plan = lv.litevar_mask_build(VAR256, 3, None, 0, q_scales, waves_per_group=waves)
    cache = lv.litevar_kv8_cache([s * s for s in VAR256], B, H)
    g = torch.Generator(device="cuda").manual_seed(12)
    k, v = (torch.randn(B, H, 680, 64, generator=g, device="cuda") for _ in range(2))
    q = torch.randn(B, H, plan.q_len, 64, generator=g, device="cuda")
    lv.litevar_kv8_store(cache, k * 2.0 ** k_power, v * 2.0 ** v_power)
    q = (q * 2.0 ** -k_power).to(torch.bfloat16)
    out = lv.litevar_windowed_attn_kv8_fwd(plan, q, cache, SM)
    want, A, S, floor = _reference(cache, q, lv.litevar_mask_export_dense(plan)[0].bool())
    plain.assert_close(out, want, _tolerance(A, S, floor))


@pytest.mark.parametrize("sm", [1e-30, 1e-6, 1.0, 1e4])
def test_softmax_scales(lv, sm):
    B, H = 1, 2
    for q_scales, waves in ROUTES:
        plan = lv.litevar_mask_build(VAR256, 3, None, 0, q_scales, waves_per_group=waves)
        cache = _cache(lv, VAR256, B, H, 8)
        q = (torch.randn(B, H, plan.q_len, 64, device="cuda") * min(1.0, 1.0 / sm)).to(torch.bfloat16)
        out = lv.litevar_windowed_attn_kv8_fwd(plan, q, cache, sm)
        want, A, S, floor = _reference(cache, q, lv.litevar_mask_export_dense(plan)[0].bool(), sm)
        plain.assert_close(out, want, _tolerance(A, S, floor))


@pytest.mark.parametrize("route", ROUTES, ids=str)
def test_bounds_checking_build_finds_nothing(lv, route):
    from paper_2411_17178_amd import build as hip_build
    q_scales, waves = route
    B, H = 2, 3
    plan = lv.litevar_mask_build(VAR256, 3, None, 0, q_scales, waves_per_group=waves)
    cache = _cache(lv, VAR256, B, H, 9)
    q = torch.randn(B, H, plan.q_len, 64, device="cuda").to(torch.bfloat16)
    out = lv.litevar_windowed_attn_kv8_fwd(plan, q, cache, SM)
    with lv.use_library(hip_build.LIB_DEBUG_BOUNDS):
        checked = lv.litevar_windowed_attn_kv8_fwd(plan, q, cache, SM)
    lv.litevar_plan_check(plan)
    assert torch.equal(out, checked)


def test_calls_on_two_streams(lv):
    """Calls that run beside each other, each with what it allocates itself."""
    B, H = 4, 16
    plans = [lv.litevar_mask_build(VAR256, 3, None, 0, q_scales, waves_per_group=waves) for q_scales, waves in ROUTES]
    cache = _cache(lv, VAR256, B, H, 10)
    qs = [torch.randn(B, H, p.q_len, 64, device="cuda").to(torch.bfloat16) for p in plans]
    want = [lv.litevar_windowed_attn_kv8_fwd(p, q, cache, SM) for p, q in zip(plans, qs)]
    streams = [torch.cuda.Stream() for _ in plans]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [[lv.litevar_windowed_attn_kv8_fwd(p, q, cache, SM, stream=s) for p, q, s in zip(plans, qs, streams)] for _ in range(5)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for outs in got for a, b in zip(outs, want))


def test_the_binding_refuses_what_does_not_fit(lv):
    B, H = 2, 3
    plan = lv.litevar_mask_build(VAR256, 3, None, 0, (9, 10))
    cache = _cache(lv, VAR256, B, H, 11)
    q = torch.zeros(B, H, 256, 64, dtype=torch.bfloat16, device="cuda")
    other = lv.litevar_kv8_cache([s * s for s in (1, 2, 3, 4, 5, 6, 8, 10, 16, 13)], B, H)
    for bad in (other, lv.litevar_kv8_cache([680], B, H), lv.litevar_kv8_cache([s * s for s in VAR256], B, H + 1)):
        with pytest.raises(AssertionError):
            lv.litevar_windowed_attn_kv8_fwd(plan, q, bad, SM)
    with pytest.raises(TypeError):
        lv.litevar_windowed_attn_kv8_fwd(plan, q.float(), cache, SM)
    with pytest.raises(AssertionError):
        lv.litevar_cross_attn_kv8_fwd(q, cache, SM)
    full = lv.litevar_mask_build(VAR256, 2, waves_per_group=16)
    need = lv.litevar_windowed_attn_kv8_workspace_bytes(full, B, H)
    assert need == B * H * 680 * 256
    with pytest.raises(lv.LitevarError):
        lv.litevar_windowed_attn_kv8_fwd(full, torch.zeros(B, H, 680, 64, dtype=torch.bfloat16, device="cuda"), cache, SM,
                                         workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda"))
    with pytest.raises(lv.LitevarError):
        lv.litevar_windowed_attn_kv8_fwd(plan, q, cache, -1.0)
    k = torch.zeros(B, H, 4, 64, dtype=torch.bfloat16, device="cuda")
    for args, kw in (((cache, k, k, (2, 3)), {}), ((cache, k, k, (1, 2)), dict(lens=torch.zeros(B, dtype=torch.int64, device="cuda"))),
                     ((cache, k, k[:, :, :3], (1, 2)), {}), ((cache, k, k, (9, 11)), {})):
        with pytest.raises(AssertionError):
            lv.litevar_kv8_store(*args, **kw)
    with pytest.raises(TypeError):
        lv.litevar_kv8_store(cache, k.half(), k.half(), (1, 2))
