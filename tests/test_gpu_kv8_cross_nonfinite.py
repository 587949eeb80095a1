"""What is not a number stays visible: a NaN in Q, or in a row of K or V that counts, reaches what the formula makes of it
in every kernel that a call may take, and nothing else.  Tolerances of what it does not reach as in test_gpu_cross_attn."""
import pytest
import torch

import _kv8_plain as plain
from test_gpu_cross_attn import _randn, _tolerance

pytestmark = pytest.mark.gpu
SM = 0.125
NAN, INF = float("nan"), float("inf")

# batch, heads, kv heads, rows, keys: rows of their own, in parts of the axis, rows that share K and V in workgroups of four
# waves and of eight, shared in parts of a long axis
ROWS, ROW_PARTS, TILES, TILES8, TILE_PARTS = (2, 4, 2, 40, 150), (2, 4, 4, 3, 5000), (16, 32, 32, 130, 150), (16, 32, 32, 520, 150), (2, 30, 1, 120, 5200)
SHAPES = [ROWS, ROW_PARTS, TILES, TILES8, TILE_PARTS]


@pytest.fixture(scope="module")
def lv():
    import paper_2411_17178_amd as m
    m.load_library()
    return m


def _reference(kind, q, k, v):
    keep = torch.ones(1, 1, 1, k.shape[2], dtype=torch.bool, device="cuda")
    want, A, S = plain.attention(q, k, v, keep, SM)
    return want, _tolerance(kind, want, A, S, k.shape[2])


def _check(out, want, tol, hit):
    """hit (broadcast over [B, H, n, 64]): NaN there, right elsewhere."""
    hit = hit.expand(out.shape)
    assert bool(torch.isnan(out[hit]).all())
    plain.assert_close(out[~hit], want[~hit], tol[~hit])


def _hit(shape, **where):
    """Truth values [B, H, n, 64]: batch row 0, the heads of kv head 0, and the row or dimension that is given."""
    B, H, Hkv, n, L = shape
    hit = torch.zeros(B, H, n, 64, dtype=torch.bool, device="cuda")
    hit[0, :where.get("heads", H // Hkv), where.get("row", slice(None)), where.get("dim", slice(None))] = True
    return hit


def _operands(shape, kind):
    B, H, Hkv, n, L = shape
    dtype = torch.float32 if kind == "f32" else torch.bfloat16
    return tuple(_randn(s, i, dtype) for i, s in enumerate([(B, H, n, 64), (B, Hkv, L, 64), (B, Hkv, L, 64)]))


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_nan_in_an_operand(lv, shape, kind):
    B, H, Hkv, n, L = shape
    q, k, v = _operands(shape, kind)
    want, tol = _reference(kind, q, k, v)
    print(f"  nan {kind} {shape}", flush=True)

    def call(name, at):
        x = dict(q=q, k=k, v=v)
        x[name] = x[name].clone()
        x[name][at] = NAN
        return lv.litevar_cross_attn_fwd(x["q"], x["k"], x["v"], SM)
    everything, key = (0, 0), L - 70
    _check(call("k", everything), want, tol, _hit(shape))
    _check(call("k", (0, 0, key, 5)), want, tol, _hit(shape))
    _check(call("k", (0, 0, 0)), want, tol, _hit(shape))
    _check(call("k", (0, 0, slice(L - 50, L))), want, tol, _hit(shape))
    _check(call("v", (0, 0, key, 5)), want, tol, _hit(shape, dim=5))
    _check(call("q", (0, 0, n - 1, 5)), want, tol, _hit(shape, heads=1, row=n - 1))


@pytest.mark.parametrize("kind", ["bf16", "f32", "codes"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_scores_below_the_range_of_fp32(lv, shape, kind):
    """Keys whose scores are -inf in fp32 have no weight, in the first blocks of the axis or all over it."""
    B, H, Hkv, n, L = shape
    for at in (slice(0, 64), slice(64, 128), slice(0, L, 2)):
        q, k, v = (x.float() for x in _operands(shape, "bf16"))
        q[..., 0], k[..., 0] = 2.0 ** 66, 0
        k[:, :, at] = 0
        k[:, :, at, 0] = -2.0 ** 66
        keep = torch.ones(L, dtype=torch.bool, device="cuda")
        keep[at] = False
        if kind == "codes":
            if at.step:                                                      # (a block's keys share its scale)
                continue
            cache = lv.litevar_kv8_store(lv.litevar_kv8_cache([L], B, Hkv), k, v)
            q = q.to(torch.bfloat16)
            out = lv.litevar_cross_attn_kv8_fwd(q, cache, SM)
            k, v = (plain.dequantise(c, s, [L]) for c, s in ((cache.k8, cache.k_scale), (cache.v8, cache.v_scale)))
        else:
            dtype = torch.float32 if kind == "f32" else torch.bfloat16
            q, k, v = (x.to(dtype) for x in (q, k, v))
            out = lv.litevar_cross_attn_fwd(q, k, v, SM)
        q0 = q.double()
        q0[..., 0] = 0                                                       # (scores of the other keys: exactly these)
        want, A, S = plain.attention(q0, k, v, keep[None, None, None], SM)
        plain.assert_close(out, want, _tolerance(kind, want, A, S, L))


@pytest.mark.parametrize("block", [0, 1, -1])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_scales_that_are_not_finite(lv, shape, block):
    """A NaN scale, or an infinite one of K, makes NaN of the rows that read its block, an infinite one of V no number."""
    B, H, Hkv, n, L = shape
    q, k, v = _operands(shape, "codes")
    cache = lv.litevar_kv8_store(lv.litevar_kv8_cache([L], B, Hkv), k, v)
    k, v = (plain.dequantise(c, s, [L]) for c, s in ((cache.k8, cache.k_scale), (cache.v8, cache.v_scale)))
    want, tol = _reference("codes", q, k, v)
    hit = _hit(shape)
    for name, value in (("k", NAN), ("k", INF), ("v", NAN), ("v", INF)):
        scale = cache.k_scale if name == "k" else cache.v_scale
        good = scale[0, 0, block].clone()
        scale[0, 0, block] = value
        out = lv.litevar_cross_attn_kv8_fwd(q, cache, SM)
        scale[0, 0, block] = good
        if name == "v" and value == INF:
            assert not bool(torch.isfinite(out[hit]).any())
            out[hit] = NAN
        _check(out, want, tol, hit)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("value", [NAN, -NAN, INF, -INF])
def test_stored_values_that_are_not_finite_show_in_the_scale(lv, value, dtype):
    """Its block's scale is NaN, or infinite, with codes of zero, so that every value of the block is NaN; other blocks,
    and rows that do not count, are as without it."""
    seg, B, H = [5, 130, 64], 2, 3
    k, v = _randn((B, H, 199, 64), 1, dtype), _randn((B, H, 199, 64), 2, dtype)
    lens = torch.tensor([199, 100], dtype=torch.int32).cuda()
    empty = [torch.full((B, H, 199, 64), 55, dtype=torch.int8, device="cuda") for _ in range(2)]
    clean, cache = (lv.KV8Cache(seg, empty[0].clone(), torch.full((B, H, 5), -5.0, device="cuda"), empty[1].clone(),
                                torch.full((B, H, 5), -5.0, device="cuda")) for _ in range(2))
    lv.litevar_kv8_store(clean, k, v, lens=lens)
    k[0, 1, 5 + 64 + 3, 63] = value                                          # block 2 of batch row 0, head 1
    v[1, 2, 5 + 10, 0] = value                                               # block 1 of batch row 1, head 2
    v[1, 0, 150, 7] = value                                                  # behind the length
    lv.litevar_kv8_store(cache, k, v, lens=lens)
    for name, b, h, block, rows in (("k", 0, 1, 2, slice(69, 133)), ("v", 1, 2, 1, slice(5, 69))):
        codes, scale = getattr(cache, name + "8"), getattr(cache, name + "_scale")
        want_codes, want_scale = getattr(clean, name + "8").clone(), getattr(clean, name + "_scale").clone()
        assert bool(torch.isnan(scale[b, h, block]) if value != value else scale[b, h, block] == INF)
        want_codes[b, h, rows] = 0
        want_scale[b, h, block] = scale[b, h, block]
        assert torch.equal(codes, want_codes)
        assert torch.equal(scale.view(torch.int32), want_scale.view(torch.int32))
    for loaded, sound, (b, h, rows) in zip(lv.litevar_kv8_load(cache), lv.litevar_kv8_load(clean), ((0, 1, slice(69, 133)), (1, 2, slice(5, 69)))):
        assert bool(torch.isnan(loaded[b, h, rows]).all())
        loaded[b, h, rows] = sound[b, h, rows]
        assert torch.equal(loaded.view(torch.int16), sound.view(torch.int16))


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_stored_values_that_are_not_finite_reach_the_rows(lv, shape):
    B, H, Hkv, n, L = shape
    q, k, v = _operands(shape, "codes")
    cache = lv.litevar_kv8_store(lv.litevar_kv8_cache([L], B, Hkv), k, v)
    want, tol = _reference("codes", q, *(plain.dequantise(c, s, [L]) for c, s in ((cache.k8, cache.k_scale), (cache.v8, cache.v_scale))))
    for value in (NAN, INF):
        for name in "kv":
            x = dict(k=k.clone(), v=v.clone())
            x[name][0, 0, L - 70, 5] = value
            out = lv.litevar_cross_attn_kv8_fwd(q, lv.litevar_kv8_store(cache, x["k"], x["v"]), SM)
            _check(out, want, tol, _hit(shape))


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_an_infinite_k_scale_under_negative_products(lv, shape):
    """Every score of the block is -inf: no weight, were the scale not taken for NaN."""
    B, H, Hkv, n, L = shape
    q, k, v = _operands(shape, "codes")
    q, k = -q.abs(), k.abs()
    cache = lv.litevar_kv8_store(lv.litevar_kv8_cache([L], B, Hkv), k, v)
    k, v = (plain.dequantise(c, s, [L]) for c, s in ((cache.k8, cache.k_scale), (cache.v8, cache.v_scale)))
    want, tol = _reference("codes", q, k, v)
    cache.k_scale[0, 0, 1] = INF
    _check(lv.litevar_cross_attn_kv8_fwd(q, cache, SM), want, tol, _hit(shape))


@pytest.mark.parametrize("kind", ["bf16", "f32", "codes"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_rows_whose_scores_all_lie_below_the_range_are_nan(lv, shape, kind):
    """fp32 does not hold their weights: NaN in every kernel, not the zeros of a row without keys, which the last batch row has."""
    B, H, Hkv, n, L = shape
    q, k, v = (x.float() for x in _operands(shape, "bf16"))
    q[..., 0], k[..., 0] = 2.0 ** 70, -2.0 ** 70
    lens = torch.full((B,), L, dtype=torch.int32, device="cuda")
    lens[-1] = 0
    if kind == "codes":
        cache = lv.litevar_kv8_store(lv.litevar_kv8_cache([L], B, Hkv), k, v)
        out = lv.litevar_cross_attn_kv8_fwd(q.to(torch.bfloat16), cache, SM, lens=lens)
    else:
        dtype = torch.float32 if kind == "f32" else torch.bfloat16
        out = lv.litevar_cross_attn_fwd(*(x.to(dtype) for x in (q, k, v)), SM, lens=lens)
    assert bool(torch.isnan(out[:-1]).all()) and bool((out[-1] == 0).all())
