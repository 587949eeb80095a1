"""Lengths of the 8-bit cache's store at the ends of their type: those below zero count as zero, those behind the rows as
all of them."""
import numpy as np
import pytest
import torch

import _kv8_plain as plain

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("segments,first", [([130], 0), ([4, 200, 9], 1)], ids=str)
def test_lengths_at_the_ends_of_their_type(segments, first):
    import paper_2411_17178_amd as lv
    lens = [-2 ** 31, -2 ** 31 + 1, -2 ** 31 + 64, -1, 0, 70, 2 ** 31 - 1]
    B, H, L = len(lens), 2, sum(segments)
    lo = sum(segments[:first])
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randn(B, H, L, 64, generator=g) for _ in range(2))
    cache = lv.litevar_kv8_cache(segments, B, H)
    for t, x in ((cache.k8, 77), (cache.v8, 77), (cache.k_scale, -5.0), (cache.v_scale, -5.0)):
        t.fill_(x)
    lv.litevar_kv8_store(cache, k[:, :, lo:].cuda(), v[:, :, lo:].cuda(), (first, len(segments)),
                         lens=torch.tensor(lens, dtype=torch.int32).cuda())
    for x, codes, scale in ((k, cache.k8, cache.k_scale), (v, cache.v8, cache.v_scale)):
        want_c, want_s, counts = plain.quantise(x.numpy(), segments, lens)
        counts[:, :lo] = False                                               # (segments that this call does not store)
        any_row = np.stack([counts[:, t:t + n].any(1) for t, n in plain.blocks(segments)], -1)
        assert np.array_equal(scale.cpu().numpy(), np.where(any_row[:, None], want_s, np.float32(-5)))
        assert np.array_equal(codes.cpu().numpy(), np.where(counts[:, None, :, None], want_c, 77))
