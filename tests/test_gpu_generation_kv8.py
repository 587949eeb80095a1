"""A conditioned layer's generation steps together: the scale's rows are stored into the 8-bit cache, its queries attend
to the cache and to an encoder's states, eagerly, on another stream and as one captured graph.  Tolerances are those of
the single operators' tests."""
import json
import subprocess
import sys

import pytest
import torch

import _kv8_plain as plain
import workloads
from test_gpu_cross_attn import _keep, _tolerance as cross_tolerance
from test_gpu_kv8_windowed import _reference, _tolerance

pytestmark = pytest.mark.gpu
SM = 0.125
VAR256 = workloads.configs.VAR256


@pytest.fixture(scope="module")
def lv():
    import paper_2411_17178_amd as m
    m.load_library()
    return m


@pytest.mark.parametrize("share_all", [False, True])
@pytest.mark.parametrize("states8", [False, True])
@pytest.mark.parametrize("by_token", [False, True])
def test_conditioned_generation(lv, share_all, states8, by_token):
    from paper_2411_17178_amd.generation import GenerationLayer
    B, H, N = 4, 5, 90
    gen = GenerationLayer(VAR256, 3, batch_heads=B * H)
    full = lv.litevar_mask_build(VAR256, 3)
    mask = lv.litevar_mask_export_dense(full)[0].bool()
    L = gen.kv_len

    def rows(n):
        t = torch.randn((B, n, H, 64) if by_token else (B, H, n, 64), device="cuda").to(torch.bfloat16)
        return t.transpose(1, 2) if by_token else t

    q, k, v, sk, sv = rows(L), rows(L), rows(L), rows(N), rows(N)
    lens = torch.tensor([N, 1, 0, 64], dtype=torch.int32).cuda()
    cache, states = gen.kv8_cache(B, H), (sk, sv)
    if states8:
        states = lv.litevar_kv8_store(lv.litevar_kv8_cache([N], B, H), sk, sv, lens=lens)
    out, cross = torch.empty_like(q), torch.empty_like(q)
    work = torch.empty(max(1, gen.kv8_workspace_bytes(B, H)), dtype=torch.uint8, device="cuda")

    def layer(stream=None):
        for s in range(gen.n_steps):
            lo, hi = gen.rows(s)
            gen.step_kv8(s, q[:, :, lo:hi], k[:, :, lo:hi], v[:, :, lo:hi], cache, SM, out_k=out[:, :, lo:hi],
                         share_all=share_all, workspace=work, stream=stream)
            gen.cross(q[:, :, lo:hi], states, SM, lens=lens, out_k=cross[:, :, lo:hi], stream=stream)

    def check():
        want, A, S, floor = _reference(cache, q, mask)
        tol = _tolerance(A, S, floor)
        half = B // 2
        plain.assert_close(out[:half], want[:half], tol[:half])
        if share_all:
            assert torch.equal(out[half:], out[:half])
        else:
            plain.assert_close(out[half:], want[half:], tol[half:])
        keep = _keep(lens, B, N)
        if states8:
            kd, vd = (plain.dequantise(c, s, [N]) for c, s in ((states.k8, states.k_scale), (states.v8, states.v_scale)))
            kd, vd = (torch.where(keep.transpose(-1, -2), t, torch.zeros_like(t)) for t in (kd, vd))
        else:
            kd, vd = sk.double(), sv.double()
        want, A, S = plain.attention(q, kd, vd, keep, SM)
        plain.assert_close(cross, want, cross_tolerance("codes" if states8 else "bf16", want, A, S, N))

    layer()
    check()
    eager = out.clone(), cross.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out.fill_(7)
    cross.fill_(7)
    side.wait_stream(torch.cuda.current_stream())
    layer(side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, eager[0]) and torch.equal(cross, eager[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer()
    for i in range(3):
        q.copy_(rows(L))
        k.copy_(rows(L))
        v.copy_(rows(L))
        cache.k8.fill_(55)
        cache.v_scale.fill_(float("nan"))
        out.fill_(float("nan"))
        cross.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        check()
        replayed = out.clone(), cross.clone()
        layer()
        assert torch.equal(out, replayed[0]) and torch.equal(cross, replayed[1])


def test_windows_agree_with_the_bf16_path_on_the_cache_values(lv):
    """The cache's values through litevar_kv8_load and the bf16 kernels: the same attention to their rounding."""
    B, H = 2, 30
    plan = lv.litevar_mask_build(VAR256, 3, None, 0, (9, 10))
    cache = lv.litevar_kv8_cache([s * s for s in VAR256], B, H)
    k, v, q = (torch.randn(B, H, n, 64, device="cuda").to(torch.bfloat16) for n in (680, 680, 256))
    lv.litevar_kv8_store(cache, k, v)
    kb, vb = lv.litevar_kv8_load(cache)
    a = lv.litevar_windowed_attn_kv8_fwd(plan, q, cache, SM)
    b = lv.litevar_windowed_attn_fwd(plan, q, kb, vb, SM)
    assert float((a.float() - b.float()).abs().max()) <= 3e-2


def test_bench_command_runs_the_conditioned_steps(lv):
    for extra in (["--kv8", "--states", "77", "--graph"], ["--states", "40", "--asc"], ["--kv8"]):
        run = subprocess.run([sys.executable, "-m", "paper_2411_17178_amd.bench_generation", "--layers", "2", "--iters", "2", "--warmup", "1",
                              "--batch", "2"] + extra, capture_output=True, text=True, timeout=100)
        assert run.returncode == 0, run.stderr[-2000:]
        line = json.loads(run.stdout.strip().splitlines()[-1])
        assert line["us_per_layer"] > 0 and line["config"]["kv8_cache"] == ("--kv8" in extra)
