"""Cross attention at the ends of its operands' ranges, in every kernel that a call may take.

Tolerance as for the ordinary operands (A = sum of weights x |v|, U = half a step of bf16): probabilities rounded to
bf16 while the sum is of the rounded ones 2 U A, the output U A, sums in 32 bits below U A / 8."""
import pytest
import torch

import _kv8_plain as plain

pytestmark = pytest.mark.gpu
SM = 0.125


@pytest.fixture(scope="module")
def lv():
    import paper_2411_17178_amd as m
    m.load_library()
    return m


def _randn(shape, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda")


# batch, heads, kv heads, rows, keys: rows of their own; in parts of the axis; rows that share K and V through LDS in
# workgroups of four waves and of eight; shared in parts of a long axis, of eight and of four
SHAPES = [(1, 6, 6, 40, 320), (2, 4, 4, 3, 5000), (16, 32, 32, 130, 300), (16, 32, 32, 520, 200), (3, 23, 1, 308, 6000), (2, 30, 1, 120, 5200)]


def _cross(lv, kind, q, k, v, sm, lens=None):
    """(output, reference, tolerance); "codes": k and v are stored first."""
    B, L = q.shape[0], k.shape[2]
    if kind == "codes":
        cache = lv.litevar_kv8_store(lv.litevar_kv8_cache([L], B, k.shape[1]), k, v)
        q = q.to(torch.bfloat16)
        out = lv.litevar_cross_attn_kv8_fwd(q, cache, sm, lens=lens)
        k, v = (plain.dequantise(c, s, [L]) for c, s in ((cache.k8, cache.k_scale), (cache.v8, cache.v_scale)))
    else:
        q, k, v = (x.to(torch.bfloat16) for x in (q, k, v))
        out = lv.litevar_cross_attn_fwd(q, k, v, sm, lens=lens)
    keep = torch.ones(1, 1, 1, L, dtype=torch.bool, device="cuda")
    if lens is not None:
        keep = (torch.arange(L, device="cuda")[None] < lens[:, None])[:, None, None]
    want, A, _ = plain.attention(q, k, v, keep, sm)
    return out, want, 3.125 * plain.U * A


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("few", [False, True])
def test_v_scales_that_are_subnormal(lv, shape, few):
    """V around 2^-120.5, which bf16 holds as normal numbers, with block scales below 2^-126; all blocks, or all but one
    whose scale is the smallest that is normal."""
    B, H, Hkv, n, L = shape
    q, k = _randn((B, H, n, 64), 1), _randn((B, Hkv, L, 64), 2)
    v = (1 + 0.2 * _randn((B, Hkv, L, 64), 3)) * 2.0 ** -120.5
    if few:
        v[:, :, 64:128] *= 4
    out, want, tol = _cross(lv, "codes", q, k, v, SM)
    plain.assert_close(out, want, tol)


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_softmax_scale_times_block_scale_leaves_the_range(lv, shape):
    """The product of the two scales is zero or infinite in fp32 though every score is a number: the weights are equal
    where it is zero or the queries are, and the largest score takes all where it is infinite."""
    B, H, Hkv, n, L = shape
    L -= 7                                                                   # (the last block has keys that do not exist)
    q, k, v = _randn((B, H, n, 64), 4), _randn((B, Hkv, L, 64), 5), _randn((B, Hkv, L, 64), 6)
    out, want, tol = _cross(lv, "codes", q, k * 2.0 ** -60, v, 1e-30)
    plain.assert_close(out, want, tol)
    # scores of one product: 2^-80 x code x scale x 1e3, thousands apart; q of zero in every second row
    q = torch.zeros_like(q)
    q[:, :, 1::2, 3] = 2.0 ** -80
    k = k * 1e37
    k[:, :, 5, 3], k[:, :, 5, 0] = 6e37, 6e37                                # (the largest: alone in its row)
    out, want, tol = _cross(lv, "codes", q, k, v, 1e3)
    plain.assert_close(out, want, tol)


@pytest.mark.parametrize("kind", ["bf16", "codes"])
@pytest.mark.parametrize("power", [80, 88, 100])
@pytest.mark.parametrize("shape", SHAPES[4:], ids=str)
def test_parts_whose_sums_grow_are_joined_without_overflow(lv, shape, power, kind):
    """Parts of the axis whose first block scores 2^-29 of the rest: products of a part are finite up to V of 2^88, those
    of all parts together are not."""
    B, H, Hkv, n, L = shape
    tiles = B * Hkv * -(-(H // Hkv * n) // 32)
    parts, rest = divmod(lv.litevar_cross_attn_workspace_bytes(B, H, Hkv, n, L), tiles * 32 * (64 * 4 + 8))
    assert parts > 4 and rest == 0
    blocks = -(-L // 64)
    q, k = 0.1 * _randn((B, H, n, 64), 7), 0.1 * _randn((B, Hkv, L, 64), 8)
    v = (1 + 0.2 * _randn((B, Hkv, L, 64), 9)) * 2.0 ** power
    v[..., 1:] *= 2.0 ** -20                                                 # (one dimension ends alone near 2^128)
    q[..., 0], k[..., 0] = 8.0, 20.125                                       # (a score of 20.125 is 29 in base 2)
    for p in range(parts):
        first = 64 * (blocks * p // parts)
        k[:, :, first:first + 64, 0] = 0
    out, want, tol = _cross(lv, kind, q, k, v, SM)
    plain.assert_close(out, want, tol)


# 113 tiles of 32 rows in each of two pairs, 82 blocks: the shape that shares K and V in parts in 16 and 8 bits alike
PARTS = (2, 30, 1, 120, 5200)


def _takes_shared_parts(lv, shape):
    B, H, Hkv, n, L = shape
    tiles = B * Hkv * -(-(H // Hkv * n) // 32)
    assert tiles == 226 and lv.litevar_cross_attn_workspace_bytes(*shape) == tiles * 10 * 32 * (64 * 4 + 8)


@pytest.mark.parametrize("kind", ["bf16", "codes"])
@pytest.mark.parametrize("flip", [False, True])
def test_shared_parts_join_scores_of_all_sizes(lv, kind, flip):
    """Scores that rise or fall along the axis by more than a part's sums may grow; one batch row is short."""
    _takes_shared_parts(lv, PARTS)
    B, H, Hkv, n, L = PARTS
    q, k, v = 3 * _randn((B, H, n, 64), 10), 3 * _randn((B, Hkv, L, 64), 11), 3 * _randn((B, Hkv, L, 64), 12)
    k = k * torch.linspace(0.01, 2.0, L, device="cuda")[:, None]
    k = k.flip(2) if flip else k
    lens = torch.tensor([L, 1300], dtype=torch.int32).cuda()
    out, want, tol = _cross(lv, kind, q.to(torch.bfloat16), k, v, SM, lens)
    plain.assert_close(out, want, tol)


def test_shared_parts_on_codes_with_v_scales_far_apart(lv):
    """V blocks between 2^-90 and 2^60 of one another, from part to part and inside one, and of zeros; K blocks of zeros."""
    _takes_shared_parts(lv, PARTS)
    B, H, Hkv, n, L = PARTS
    q, k, v = _randn((B, H, n, 64), 13), _randn((B, Hkv, L, 64), 14), _randn((B, Hkv, L, 64), 15)
    for power in (0, 60):
        v[0, 0, 64 * 8:64 * 16] *= 2.0 ** -90                                # (a part and more)
        v[0, 0, 64 * 20:64 * 21] *= 2.0 ** power
        v[0, 0, 64 * 30:64 * 50] = 0
        v[1, 0, 64::128] *= 2.0 ** -40
        v[1, 0, 64 * 70:64 * 71] = 0
        k[1, 0, 64 * 40:64 * 60] = 0
        out, want, tol = _cross(lv, "codes", q, k, v, SM)
        plain.assert_close(out, want, tol)


@pytest.mark.parametrize("shape", [PARTS, (16, 32, 32, 130, 300), (1, 6, 6, 40, 320)], ids=str)
@pytest.mark.parametrize("high", [64.0, 2.0 ** 14])
def test_far_scores_on_codes(lv, shape, high):
    """References of 2^19 and 2^27 in base 2: the rows are formed again from exact differences.  Scores are whole
    multiples of 64 x 2^-6 and no sum on the way passes 24 bits, so that they are exact."""
    B, H, Hkv, n, L = shape
    if shape is PARTS:
        _takes_shared_parts(lv, PARTS)
    g = torch.Generator(device="cuda").manual_seed(16)
    q = torch.zeros(B, H, n, 64, device="cuda")
    k = torch.zeros(B, Hkv, L, 64, device="cuda")
    k[..., 0] = 127 * 64.0                                                   # (block scales of 64)
    if high == 64.0:
        q[..., 1:9] = torch.randint(-1, 2, (B, H, n, 8), generator=g, device="cuda") / 64.0
        k[..., 1:9] = 64.0 * torch.randint(-1, 2, (B, Hkv, L, 8), generator=g, device="cuda")
    else:
        k[:, :, ::3, 0] = 126 * 64.0
    q[..., 0] = high
    out, want, tol = _cross(lv, "codes", q, k, _randn((B, Hkv, L, 64), 17), 1.0)
    plain.assert_close(out, want, tol)
