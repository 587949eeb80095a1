"""Cross attention with scores that fp32 does not hold, in every kernel that a call may take.  Tolerances as in
test_gpu_cross_attn."""
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


def _operands(shape, kind):
    B, H, Hkv, n, L = shape
    dtype = torch.float32 if kind == "f32" else torch.bfloat16
    return tuple(_randn(s, i, dtype) for i, s in enumerate([(B, H, n, 64), (B, Hkv, L, 64), (B, Hkv, L, 64)]))


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
