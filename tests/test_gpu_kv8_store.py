"""The 8-bit cache with block scales: what is stored equals the plain statement bit for bit (codes are decided in
binary32 on both sides), rows that do not count and blocks of other segments stay as they were."""
import numpy as np
import pytest
import torch

import _kv8_plain as plain

pytestmark = pytest.mark.gpu
VAR256 = [s * s for s in (1, 2, 3, 4, 5, 6, 8, 10, 13, 16)]


@pytest.fixture(scope="module")
def lv():
    import paper_2411_17178_amd as m
    m.load_library()
    return m


def _rows(B, H, L, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(B, H, L, 64, generator=g)
    # magnitudes that differ from block to block, by far
    x *= torch.exp(torch.randn(B, H, L, 1, generator=g) * 2)
    return x.to(dtype)


def _poisoned(lv, segments, B, H):
    c = lv.litevar_kv8_cache(segments, B, H)
    for t in (c.k8, c.v8):
        t.fill_(77)
    for t in (c.k_scale, c.v_scale):
        t.fill_(-5.0)
    return c


def _check(cache, k, v, segments, lens=None):
    for x, codes, scale in ((k, cache.k8, cache.k_scale), (v, cache.v8, cache.v_scale)):
        want_c, want_s, counts = plain.quantise(x.float().cpu().numpy(), segments, lens)
        want_c = np.where(counts[:, None, :, None], want_c, 77)
        any_row = np.stack([counts[:, t:t + n].any(1) for t, n in plain.blocks(segments)], -1)
        want_s = np.where(any_row[:, None], want_s, np.float32(-5))
        assert np.array_equal(scale.cpu().numpy(), want_s)
        assert np.array_equal(codes.cpu().numpy(), want_c)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("segments", [[1], [63], [64], [65], [333], [5, 0, 64, 1, 0, 130], VAR256], ids=str)
def test_store_equals_the_plain_statement(lv, segments, dtype):
    B, H, L = 3, 5, sum(segments)
    print(f"  store {segments} {dtype}", flush=True)
    k, v = _rows(B, H, L, dtype, 1), _rows(B, H, L, dtype, 2)
    cache = _poisoned(lv, segments, B, H)
    lv.litevar_kv8_store(cache, k.cuda(), v.cuda())
    _check(cache, k, v, segments)


def test_segments_one_by_one_equal_all_at_once(lv):
    B, H, L = 2, 3, sum(VAR256)
    k, v = _rows(B, H, L, torch.bfloat16, 3).cuda(), _rows(B, H, L, torch.bfloat16, 4).cuda()
    cache = _poisoned(lv, VAR256, B, H)
    for i in range(len(VAR256)):
        lo, hi = cache.offsets[i], cache.offsets[i + 1]
        before = cache.k8[:, :, hi:].clone()
        lv.litevar_kv8_store(cache, k[:, :, lo:hi], v[:, :, lo:hi], (i, i + 1))
        assert torch.equal(cache.k8[:, :, hi:], before)
    _check(cache, k.cpu(), v.cpu(), VAR256)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_behind_the_length_are_not_read_and_not_written(lv, dtype):
    lens, L = [130, 0, 1, 64, 65, 129, 200, -3], 130
    B, H = len(lens), 3
    k, v = _rows(B, H, L, dtype, 5), _rows(B, H, L, dtype, 6)
    for b, n in enumerate(lens):
        k[b, :, max(n, 0):] = float("nan")
        v[b, :, max(n, 0):] = float("inf")
    cache = _poisoned(lv, [L], B, H)
    lv.litevar_kv8_store(cache, k.cuda(), v.cuda(), lens=torch.tensor(lens, dtype=torch.int32).cuda())
    _check(cache, k, v, [L], lens)


def test_lengths_count_from_the_first_token_of_the_cache(lv):
    seg, B, H = [4, 70, 9], 2, 2
    k, v = _rows(B, H, sum(seg), torch.bfloat16, 7), _rows(B, H, sum(seg), torch.bfloat16, 8)
    cache = _poisoned(lv, seg, B, H)
    lens = torch.tensor([80, 69], dtype=torch.int32).cuda()
    lv.litevar_kv8_store(cache, k[:, :, :4].cuda(), v[:, :, :4].cuda(), (0, 1), lens=lens)
    lv.litevar_kv8_store(cache, k[:, :, 4:].cuda(), v[:, :, 4:].cuda(), (1, 3), lens=lens)
    _check(cache, k, v, seg, [80, 69])


def test_strided_rows(lv):
    B, H, L = 2, 6, 100
    base = _rows(B, L, H, torch.bfloat16, 9).cuda()                       # [B, L, H, 64]
    both = torch.cat([base, -base], -1)                                   # K and V in one projection
    k, v = both[..., :64].transpose(1, 2), both[..., 64:].transpose(1, 2)
    cache = _poisoned(lv, [L], B, H)
    lv.litevar_kv8_store(cache, k, v)
    _check(cache, k.cpu(), v.cpu(), [L])


def test_values_at_the_ends_of_their_range(lv):
    """Zero blocks, ties, subnormal and very large magnitudes: every quotient is the correctly rounded one."""
    rows = np.zeros((1, 12, 64, 64), np.float32)
    g = np.random.default_rng(3)
    for h, top in enumerate([0.0, 1e-45, 3e-44, 1e-38, 2e-38, 1e-31, 1e-30, 127.0, 1e30, 2e32, 3.4e38, 254.0]):
        rows[0, h] = (g.uniform(-1, 1, (64, 64)) * top).astype(np.float32)
        if top:
            rows[0, h, 0, 0] = top
    rows[0, 7, 1] = np.arange(64) - 31.5                                  # ties at s = 1
    rows[0, 11, 1] = np.arange(64) * 2 - 63                               # ties at s = 2
    k = torch.from_numpy(rows)
    cache = _poisoned(lv, [64], 1, 12)
    lv.litevar_kv8_store(cache, k.cuda(), (-k).cuda())
    _check(cache, k, -k, [64])


def test_quotients_next_to_a_border(lv):
    """Many magnitudes and values whose quotient lies within a few 2^-24 of a tie."""
    g = np.random.default_rng(11)
    H = 256
    rows = np.zeros((1, H, 64, 64), np.float32)
    for h in range(H):
        top = np.float32(np.exp(g.uniform(-30, 30)))
        s = top / np.float32(127)
        t = (g.integers(-126, 126, 4096) + 0.5) * np.float64(s)
        t = np.nextafter(t.astype(np.float32), np.where(g.random(4096) < 0.5, -np.inf, np.inf).astype(np.float32)) \
            if h % 2 else t.astype(np.float32)
        rows[0, h] = t.reshape(64, 64)
        rows[0, h, 0, 0] = top
    k = torch.from_numpy(rows)
    cache = _poisoned(lv, [64], 1, H)
    lv.litevar_kv8_store(cache, k.cuda(), k.cuda())
    _check(cache, k, k, [64])


def test_load_gives_the_products_rounded_once(lv):
    seg, B, H = [1, 4, 70], 2, 3
    k, v = _rows(B, H, 75, torch.float32, 12), _rows(B, H, 75, torch.float32, 13)
    cache = _poisoned(lv, seg, B, H)
    lv.litevar_kv8_store(cache, k.cuda(), v.cuda())
    out = tuple(torch.full((B, H, 75, 64), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    lv.litevar_kv8_load(cache, (1, 3), out=out)
    for t, codes, scale in ((out[0], cache.k8, cache.k_scale), (out[1], cache.v8, cache.v_scale)):
        # (a product of 24 and 7 bits is rounded to 32 bits first; the second rounding is the kernel's too)
        want = plain.dequantise(codes, scale, seg).float().to(torch.bfloat16)
        assert torch.equal(t[:, :, 1:], want[:, :, 1:]) and bool((t[:, :, :1] == 9).all())
    kk, vv = lv.litevar_kv8_load(cache)
    assert torch.equal(kk[:, :, 1:], out[0][:, :, 1:]) and torch.equal(vv[:, :, 1:], out[1][:, :, 1:])


def test_store_on_another_stream_and_captured(lv):
    B, H, L = 2, 4, 77
    k, v = _rows(B, H, L, torch.bfloat16, 14).cuda(), _rows(B, H, L, torch.bfloat16, 15).cuda()
    cache = _poisoned(lv, [L], B, H)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    lv.litevar_kv8_store(cache, k, v, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    _check(cache, k.cpu(), v.cpu(), [L])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lv.litevar_kv8_store(cache, k, v)
    for i in range(3):
        k.copy_(_rows(B, H, L, torch.bfloat16, 20 + i))
        v.copy_(_rows(B, H, L, torch.bfloat16, 30 + i))
        cache.k8.fill_(77)
        graph.replay()
        torch.cuda.synchronize()
        _check(cache, k.cpu(), v.cpu(), [L])
