"""Cross attention in bf16, fp32 and on an 8-bit cache against the formula in 64 bits.

Tolerances, element by element, from A = sum of weights x |v| and S = the row's largest sum of |q_d k_d| x sm_scale:
  bf16, codes  a probability is rounded to bf16 (relative U = 2^-8 at most) while the sum is of the rounded ones:
               2 U A; the output is rounded: U |out| <= U A; sums in 32 bits: far below U A / 8 here.  3.125 U A.
  fp32         scores carry 64 roundings of partial sums (64 x 2^-24 S, doubled for the reference's own), the
               exponential and its argument 2^-21, n terms of the sums 2^-24 each; weights and sum: twice.
"""
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


def _randn(shape, seed, dtype=torch.float32, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def _lens(B, kv_len, seed):
    g = torch.Generator().manual_seed(seed)
    lens = torch.randint(0, kv_len + 1, (B,), generator=g, dtype=torch.int32)
    lens[0] = kv_len
    if B > 1:
        lens[-1] = 0
    return lens.cuda()


def _keep(lens, B, kv_len):
    if lens is None:
        return torch.ones(1, 1, 1, max(kv_len, 1), dtype=torch.bool, device="cuda")[..., :kv_len]
    return (torch.arange(kv_len, device="cuda")[None] < lens[:, None])[:, None, None]


def _tolerance(kind, out, A, S, n):
    if kind == "f32":
        return 2 * A * (2.0 ** -24 * (2 * 64 * S + n) + 2.0 ** -21)
    return 3.125 * plain.U * A


def _run(lv, kind, q, k, v, lens, sm=SM, **kw):
    """(output, reference, tolerance) for operands q, k, v in 32 bits; "codes": k, v are stored first."""
    B, kv_len = q.shape[0], k.shape[2]
    if kind == "codes":
        cache = lv.litevar_kv8_cache([kv_len], B, k.shape[1])
        cache.k8.fill_(99)
        cache.v8.fill_(-99)
        for t in (cache.k_scale, cache.v_scale):
            t.fill_(float("nan"))
        lv.litevar_kv8_store(cache, k, v, lens=lens)
        q = q.to(torch.bfloat16)
        out = lv.litevar_cross_attn_kv8_fwd(q, cache, sm, lens=lens, **kw)
        k, v = (plain.dequantise(c, s, [kv_len]) for c, s in ((cache.k8, cache.k_scale), (cache.v8, cache.v_scale)))
    else:
        dtype = torch.float32 if kind == "f32" else torch.bfloat16
        q, k, v = q.to(dtype), k.to(dtype), v.to(dtype)
        out = lv.litevar_cross_attn_fwd(q, k, v, sm, lens=lens, **kw)
    keep = _keep(lens, B, kv_len)
    used = keep.transpose(-1, -2) if lens is not None else keep.new_ones(1, 1, kv_len, 1)
    zero = torch.zeros((), dtype=torch.float64, device="cuda")
    want, A, S = plain.attention(q, torch.where(used, k.double(), zero), torch.where(used, v.double(), zero), keep, sm)
    return out, want, _tolerance(kind, want, A, S, kv_len)


SHAPES = [  # B, H, H_kv, q_len, kv_len
    (1, 1, 1, 1, 1), (2, 3, 3, 1, 77), (3, 2, 2, 31, 31), (2, 2, 2, 32, 32), (3, 2, 1, 33, 33), (2, 4, 2, 17, 63),
    (2, 4, 4, 64, 64), (2, 2, 2, 65, 65), (4, 3, 3, 100, 129), (2, 30, 30, 169, 333), (3, 6, 3, 257, 200),
    (2, 8, 1, 1, 1000), (1, 2, 2, 5, 4099), (2, 8, 2, 3, 9001), (1, 1, 1, 2240, 512), (2, 5, 5, 300, 1),
    (2, 3, 3, 7, 0), (2, 3, 3, 0, 7),
    # rows that share K and V through LDS, in four and in eight waves; with shared heads
    (8, 32, 32, 257, 200), (16, 32, 32, 100, 77), (16, 32, 8, 140, 130), (8, 64, 64, 300, 33), (4, 64, 64, 1000, 1), (16, 32, 32, 130, 0),
    (8, 64, 64, 530, 130), (16, 32, 32, 700, 65), (31, 34, 17, 300, 97),
    # few pairs of many rows (codes: four waves), on more blocks than a wave holds scales of
    (2, 24, 24, 500, 330), (1, 24, 24, 1000, 4300), (2, 160, 160, 150, 4165),
    # more batch rows than a wave has lanes, and as many
    (70, 12, 12, 140, 97), (64, 12, 6, 140, 97), (65, 9, 9, 160, 70),
    # rows that share K and V, in parts of a long axis: in eight waves and in four, with parts that hold nothing
    (2, 32, 1, 100, 5200), (16, 16, 1, 32, 5130), (5, 40, 1, 33, 5121), (3, 23, 1, 308, 6000),
    # parts of a long axis, more workgroups than a round
    (1, 130, 130, 40, 5200), (3, 100, 50, 60, 5121),
]
# (rows of a call that share K and V through LDS, whatever the type: 2560 tiles)
MANY = (16, 32, 130)
# (and in workgroups of eight waves, more of them than the chip holds)
MORE = (16, 32, 520)


@pytest.mark.parametrize("kind", ["bf16", "f32", "codes"])
@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_cross_attention(lv, shape, ragged, kind):
    B, H, Hkv, n, L = shape
    print(f"  cross {kind} {shape} ragged={ragged}", flush=True)
    q, k, v = _randn((B, H, n, 64), 1), _randn((B, Hkv, L, 64), 2), _randn((B, Hkv, L, 64), 3)
    lens = _lens(B, L, 4) if ragged else None
    out, want, tol = _run(lv, kind, q, k, v, lens)
    plain.assert_close(out, want, tol)


@pytest.mark.parametrize("kind", ["bf16", "f32", "codes"])
@pytest.mark.parametrize("B,H,n", [(6, 3, 40), MANY, MORE], ids=str)
def test_rows_behind_the_length_are_not_read(lv, kind, B, H, n):
    L = 150
    lens = torch.tensor(([150, 1, 64, 65, 0, 97] + list(range(20, 40)))[:B], dtype=torch.int32).cuda()
    q, k, v = _randn((B, H, n, 64), 5), _randn((B, H, L, 64), 6), _randn((B, H, L, 64), 7)
    for b, m in enumerate(lens.tolist()):
        k[b, :, m:] = float("nan")
        v[b, :, m:] = float("inf")
    out, want, tol = _run(lv, kind, q, k, v, lens)
    plain.assert_close(out, want, tol)
    assert bool((out[4] == 0).all())


@pytest.mark.parametrize("n", [3, 20000])
def test_lengths_outside_the_axis_are_taken_as_its_ends(lv, n):
    q, k, v = _randn((3, 2, n, 64), 8), _randn((3, 2, 70, 64), 9), _randn((3, 2, 70, 64), 10)
    wild = torch.tensor([1000, -1, 70], dtype=torch.int32).cuda()
    tame = torch.tensor([70, 0, 70], dtype=torch.int32).cuda()
    for dtype in (torch.bfloat16, torch.float32):
        args = [t.to(dtype) for t in (q, k, v)]
        assert torch.equal(lv.litevar_cross_attn_fwd(*args, SM, lens=wild), lv.litevar_cross_attn_fwd(*args, SM, lens=tame))


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("H,n", [(4, 1), (4, 50), (4, 300), (150, 141), (160, 600)])
def test_strides(lv, kind, H, n):
    """Rows as a fused projection leaves them, K and V of one prompt shared by the batch, an output inside a larger one."""
    B, L = 3, 90
    dtype = torch.float32 if kind == "f32" else torch.bfloat16
    q = _randn((B, n, H, 64), 11, dtype).transpose(1, 2)
    kv = _randn((1, L, 2 * H, 64), 12, dtype)
    k, v = (t.transpose(1, 2).expand(B, H, L, 64) for t in (kv[:, :, :H], kv[:, :, H:]))
    big = torch.full((B, n + 2, H, 64), 7.0, dtype=dtype, device="cuda")
    out = big[:, 1:n + 1].transpose(1, 2)
    lv.litevar_cross_attn_fwd(q, k, v, SM, out=out)
    want, A, S = plain.attention(q, k, v, _keep(None, B, L), SM)
    plain.assert_close(out, want, _tolerance(kind, want, A, S, L))
    assert bool((big[:, 0] == 7).all()) and bool((big[:, -1] == 7).all())


@pytest.mark.parametrize("kind", ["bf16", "f32", "codes"])
@pytest.mark.parametrize("B,H,n", [(2, 2, 2), (2, 2, 130), MANY, MORE], ids=str)
def test_peaked_and_far_scores(lv, kind, B, H, n):
    """Scores of many sizes: one key takes nearly everything, scores fall and rise along the axis."""
    L = 300
    q, k, v = _randn((B, H, n, 64), 13, scale=3.0), _randn((B, H, L, 64), 14, scale=3.0), _randn((B, H, L, 64), 15)
    k = k * torch.linspace(0.01, 2.0, L, device="cuda")[:, None]
    for flip in (False, True):
        kk = k.flip(2) if flip else k
        q16, k16 = q.to(torch.bfloat16).float(), kk.to(torch.bfloat16).float()    # (the operands of all kinds)
        out, want, tol = _run(lv, kind, q16, k16, v.to(torch.bfloat16).float(), None)
        plain.assert_close(out, want, tol)


@pytest.mark.parametrize("kind", ["bf16", "codes"])
@pytest.mark.parametrize("flip", [False, True])
def test_parts_join_scores_of_all_sizes(lv, kind, flip):
    """Scores that rise along the axis, from part to part and inside one; the last heads' beyond 2^24, whose rows are formed again."""
    B, H, n, L = 2, 32, 100, 5200
    q, k, v = _randn((B, H, n, 64), 31, scale=3.0), _randn((B, 1, L, 64), 32, scale=3.0), _randn((B, 1, L, 64), 33)
    k = k * torch.linspace(0.01, 2.0, L, device="cuda")[:, None]
    if flip:
        k = k.flip(2)
    q[:, 30:] = 0
    q[:, 30:, :, 0] = 2.0 ** 24                                              # (a score is then one product)
    k[..., 0] = torch.linspace(1.0, 127.0, L, device="cuda").round() * 64
    q, k, v = (x.to(torch.bfloat16).float() for x in (q, k, v))
    lens = torch.tensor([L, 1300], dtype=torch.int32).cuda()
    out, want, tol = _run(lv, kind, q[:, :30], k, v, lens)
    plain.assert_close(out, want, tol)
    if kind == "bf16":                                                       # (codes of a block differ from these keys)
        out, want, tol = _run(lv, kind, q, k, v, lens)
        plain.assert_close(out, want, tol)


@pytest.mark.parametrize("kind", ["bf16", "f32", "codes"])
@pytest.mark.parametrize("B,H,n", [(1, 1, 1), (1, 1, 100), MANY, MORE], ids=str)
def test_scores_that_fp32_holds_keep_their_differences(lv, kind, B, H, n):
    """Scores around 2^27 whose differences are whole numbers of 2^20: the largest keys win, exactly."""
    L = 128
    q = torch.zeros(B, H, n, 64, device="cuda")
    q[..., 0] = 2.0 ** 14
    k = torch.zeros(B, H, L, 64, device="cuda")
    k[..., 0] = 127.0 * 64
    k[:, :, ::2, 0] = 126.0 * 64
    v = _randn((B, H, L, 64), 16)
    out, want, tol = _run(lv, kind, q, k, v, None, sm=1.0)
    if kind == "f32":                                                    # (the scores are exact here: no term of theirs)
        tol = 2.0 ** -20 * (tol * 0 + v.abs().amax())
    plain.assert_close(out, want, tol)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,n", [(1, 2, 40), MANY, MORE], ids=str)
def test_values_near_the_end_of_the_range(lv, kind, B, H, n):
    """Values of 2^120 and scores that rise along the axis: sums under a reference that moves do not overflow into the
    result."""
    L = 200
    q, k, v = _randn((B, H, n, 64), 30), _randn((B, H, L, 64), 31) * 0.1, _randn((B, H, L, 64), 32) * 2.0 ** 120
    k = k + q.mean(2, keepdim=True) * torch.linspace(0.0, 30.0, L, device="cuda")[:, None]
    out, want, tol = _run(lv, kind, q.to(torch.bfloat16).float(), k.to(torch.bfloat16).float(), v.to(torch.bfloat16).float(), None)
    plain.assert_close(out, want, tol)


def test_blocks_of_very_different_scales(lv):
    """Blocks of K and V between 2^-110 and 2^110 of one another, blocks of zeros: each counts at its own size."""
    L = 64 * 5
    for B, H, n in ((1, 6, 1), (1, 6, 40), (1, 6, 290), (50, 6, 90)):
        q = _randn((B, H, n, 64), 17)
        k, v = _randn((B, H, L, 64), 18), _randn((B, H, L, 64), 19)
        k[:, 0, 64:128] *= 2.0 ** -110
        k[:, 1, :64] = 0
        v[:, 2, 64:128] *= 2.0 ** -110
        v[:, 3, 128:192] = 0
        v[:, 4, 192:256] *= 2.0 ** 100
        v[:, 5] *= 2.0 ** -110
        out, want, tol = _run(lv, "codes", q, k, v, None)
        plain.assert_close(out, want, tol)


@pytest.mark.parametrize("kind", ["bf16", "f32", "codes"])
@pytest.mark.parametrize("shape", [(2, 4, 4, 3, 5000), (2, 4, 4, 200, 300), (16, 32, 32, 130, 70), (16, 32, 32, 520, 70)], ids=str)
def test_workspace_contents_do_not_matter_and_runs_repeat(lv, kind, shape):
    B, H, Hkv, n, L = shape
    need = lv.litevar_cross_attn_workspace_bytes(B, H, Hkv, n, L)
    q, k, v = _randn((B, H, n, 64), 20), _randn((B, Hkv, L, 64), 21), _randn((B, Hkv, L, 64), 22)
    lens = _lens(B, L, 23)
    outs = []
    for fill in (0, 255):
        w = torch.full((need,), fill, dtype=torch.uint8, device="cuda")
        out, want, tol = _run(lv, kind, q, k, v, lens, workspace=w)
        plain.assert_close(out, want, tol)
        outs.append(out)
    assert torch.equal(outs[0], outs[1])


def test_offsets_beyond_32_bits(lv):
    """A cache whose rows of one head lie more than 2^32 bytes apart."""
    L, heads = 140_000, 256
    base = torch.empty(L, heads, 64, dtype=torch.bfloat16, device="cuda")     # 4.6 GB
    base[:, -1] = _randn((L, 64), 24, torch.bfloat16)
    kv = base.view(1, L, heads, 64).transpose(1, 2)[:, -1:]
    for n in (2, 100, 16000):
        q = _randn((1, 1, n, 64), 25, torch.bfloat16)
        out = lv.litevar_cross_attn_fwd(q, kv, kv, SM)
        want, A, S = plain.attention(q, kv, kv, _keep(None, 1, L), SM)
        plain.assert_close(out, want, _tolerance("bf16", want, A, S, L))


@pytest.mark.parametrize("H,n,L", [(4, 2, 6000), (4, 150, 300), (300, 130, 100), (300, 520, 100)])
def test_streams_and_graphs(lv, H, n, L):
    B = 2
    side = torch.cuda.Stream()
    q, k, v = (_randn(s, i, torch.bfloat16) for i, s in enumerate([(B, H, n, 64), (B, H, L, 64), (B, H, L, 64)]))
    cache = lv.litevar_kv8_cache([L], B, H)
    lens = torch.tensor([L, L // 2], dtype=torch.int32).cuda()
    side.wait_stream(torch.cuda.current_stream())
    lv.litevar_kv8_store(cache, k, v, lens=lens, stream=side)
    on_side = [lv.litevar_cross_attn_fwd(q, k, v, SM, lens=lens, stream=side),
               lv.litevar_cross_attn_kv8_fwd(q, cache, SM, lens=lens, stream=side)]
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lv.litevar_kv8_store(cache, k, v, lens=lens)
        got = [lv.litevar_cross_attn_fwd(q, k, v, SM, lens=lens), lv.litevar_cross_attn_kv8_fwd(q, cache, SM, lens=lens)]
    for i in range(4):
        graph.replay()
        torch.cuda.synchronize()
        if i == 0:
            assert all(torch.equal(a, b) for a, b in zip(got, on_side))
        eager = lv.litevar_kv8_store(lv.litevar_kv8_cache([L], B, H), k, v, lens=lens)
        assert torch.equal(got[0], lv.litevar_cross_attn_fwd(q, k, v, SM, lens=lens))
        assert torch.equal(got[1], lv.litevar_cross_attn_kv8_fwd(q, eager, SM, lens=lens))
        q.copy_(_randn(q.shape, 40 + i, torch.bfloat16))
        k.copy_(_randn(k.shape, 50 + i, torch.bfloat16))
        lens.copy_(torch.tensor([L - 7 * i, 3 * i], dtype=torch.int32))
