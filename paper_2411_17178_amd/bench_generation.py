"""Times all KV-cache generation steps of the attention layers of a VAR model (paper
Section 2: scale-by-scale generation) on one GPU: per layer, one library call per scale, the
queries being that scale's tokens and the keys the cache rows of the scales so far; with
--asc the unconditional half of the batch reuses the conditional half's attention output
everywhere (paper Section 3).  Run as

    python -m paper_2411_17178_amd.bench_generation [--workload var_d30_kvstep] [--asc] [--graph] [--kv8] [--states N]

--kv8 keeps K and V in an 8-bit cache with block scales: every step stores its scale's rows and attends to the cache.
--states N adds what a conditioned layer does behind each step, attention to N encoder states (ragged lengths; with --kv8
from an 8-bit cache of their own, filled once).

Prints one JSON line: microseconds per layer (all steps of one layer), per step, and the
effective TFLOP/s over the retained (query, key) pairs that were computed.  With --kv8 and --states the time
includes the stores and the attention to the states, which the TFLOP/s do not count; the metric's name says so.  Inputs are
seeded synthetic N(0,1) tensors resident in HBM, each layer with its own Q, K, V and O.
"""
import argparse
import json
import sys
import time


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--workload", default="var_d30_kvstep", help="gives scales, radius, batch, heads")
    ap.add_argument("--layers", type=int, default=30)
    ap.add_argument("--iters", type=int, default=20)
    ap.add_argument("--warmup", type=int, default=3)
    ap.add_argument("--asc", action="store_true", help="share the conditional output everywhere")
    ap.add_argument("--graph", action="store_true", help="replay each layer's steps as one HIP graph")
    ap.add_argument("--kv8", action="store_true", help="8-bit K/V cache with block scales")
    ap.add_argument("--states", type=int, default=0, help="encoder states that each step attends to as well")
    ap.add_argument("--batch", type=int, default=0, help="batch size (0 = the workload's)")
    ap.add_argument("--no-hint", action="store_true", help="do not tell the plans the batch size")
    args = ap.parse_args()

    import torch

    import paper_2411_17178_amd as lv
    import workloads
    from paper_2411_17178_amd.generation import GenerationLayer

    lv.load_library()
    if not torch.cuda.is_available():
        print("bench_generation: no GPU visible; the HIP path has no CPU fallback", file=sys.stderr)
        sys.exit(3)
    dev = torch.device("cuda:0")
    torch.cuda.set_device(0)
    w = workloads.get(args.workload)
    B, H = args.batch or w.batch, w.heads
    working = B * H // 2 if args.asc else B * H          # (batch, head) pairs that compute
    gen = GenerationLayer(w.scales, w.radius, n_sink_scales=w.n_sink, device=dev,
                          batch_heads=0 if args.no_hint else working)
    L = gen.kv_len
    g = torch.Generator(device=dev).manual_seed(w.seed + 999)

    def draw():
        return (torch.randn((B, H, L, 64), generator=g, device=dev) * w.input_scale).to(torch.bfloat16)

    calls = []
    keep = []
    for _ in range(args.layers):
        q, k, v = draw(), draw(), draw()
        o = torch.empty_like(q)
        rows = [gen.rows(s) for s in range(gen.n_steps)]
        q_steps = [q[:, :, lo:hi] for lo, hi in rows]
        o_steps = [o[:, :, lo:hi] for lo, hi in rows]
        keep.append((q, k, v, o))
        calls.append((q_steps, k, v, o_steps))

    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        if args.kv8:
            work = torch.empty(max(1, gen.kv8_workspace_bytes(B, H)), dtype=torch.uint8, device=dev)
            rows = [gen.rows(s) for s in range(gen.n_steps)]

            def kv8_steps(qs, k, v, os_):
                cache = gen.kv8_cache(B, H, dev)
                return [lambda s=s, lo=lo, hi=hi: gen.step_kv8(s, qs[s], k[:, :, lo:hi], v[:, :, lo:hi], cache, w.sm_scale,
                                                               out_k=os_[s], share_all=args.asc, workspace=work)
                        for s, (lo, hi) in enumerate(rows)]
            layer_calls = [kv8_steps(*c) for c in calls]
        else:
            layer_calls = [gen.prepare(qs, k, v, w.sm_scale, os_, share_all=args.asc, stream=stream)
                           for qs, k, v, os_ in calls]
        if args.states:
            lens = torch.randint(args.states // 4, args.states + 1, (B,), generator=g, device=dev, dtype=torch.int32)
            cross_work = torch.empty(max(1, gen.cross_workspace_bytes(B, H, H, args.states)), dtype=torch.uint8, device=dev)

            def with_states(steps, qs):
                k, v = (torch.randn((B, H, args.states, 64), generator=g, device=dev).to(torch.bfloat16) for _ in range(2))
                states = lv.litevar_kv8_store(lv.litevar_kv8_cache([args.states], B, H, dev), k, v, lens=lens) if args.kv8 else (k, v)
                outs = [torch.empty_like(x) for x in qs]
                return [f for step, x, o in zip(steps, qs, outs)
                        for f in (step, lambda x=x, o=o: gen.cross(x, states, w.sm_scale, lens=lens, out_k=o, workspace=cross_work))]
            layer_calls = [with_states(steps, c[0]) for steps, c in zip(layer_calls, calls)]
        if args.graph:
            graphs = []
            for lc in layer_calls:
                for c in lc:        # one eager pass first
                    c()
                gr = torch.cuda.CUDAGraph()
                with torch.cuda.graph(gr, stream=stream):
                    for c in lc:
                        c()
                graphs.append(gr)

            def run_all():
                for gr in graphs:
                    gr.replay()
        else:
            def run_all():
                for lc in layer_calls:
                    for c in lc:
                        c()

        for _ in range(args.warmup):
            run_all()
        stream.synchronize()
        t0 = time.perf_counter()
        for _ in range(args.iters):
            run_all()
        stream.synchronize()
        t1 = time.perf_counter()

    us_layer = (t1 - t0) / (args.iters * args.layers) * 1e6
    pairs = gen.retained_pairs() * H * (B // 2 if args.asc else B)
    also = [name for name, timed in (("8-bit cache stores", args.kv8),
                                     (f"attention to {args.states} encoder states", args.states)) if timed]
    print(json.dumps({
        "metric": "windowed-attn effective TFLOP/s (retained pairs), all generation steps of a layer"
                  + (", timed with its " + " and ".join(also) if also else ""),
        "value": round(256.0 * pairs / (us_layer * 1e-6) / 1e12, 3), "unit": "TFLOP/s",
        "us_per_layer": round(us_layer, 2), "us_per_step": round(us_layer / gen.n_steps, 2),
        "steps_per_layer": gen.n_steps, "layers": args.layers, "iters": args.iters,
        "dtype": "bf16", "data": "synthetic (seeded N(0,1), drawn on the device)",
        "config": {"workload": w.name + " (all steps)", "scales": list(w.scales), "batch": B,
                   "heads": H, "radius": w.radius, "asc_everywhere": bool(args.asc),
                   "patches_per_group": [int(p.waves_per_group) for p in gen.plans],
                   "hip_graph": bool(args.graph), "kv8_cache": bool(args.kv8), "encoder_states": args.states}}))


if __name__ == "__main__":
    main()
