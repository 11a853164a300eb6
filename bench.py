#!/usr/bin/env python3
"""Benchmark of the ZipVL prefill hot path on one MI355X.

A step is one pass of the whole per-layer path over one batch of synthetic
input that is already resident in HBM:
    zipvl_score -> zipvl_select -> zipvl_compact_kv -> zipvl_sparse_prefill
all stream-ordered through the C ABI.  The default workload is the long-video
GQA layer (28 query heads / 4 KV heads, d=128, 18 432 tokens, bf16).

Prints ONE JSON line.  `value` is the dense-equivalent attention throughput
2*B*Hq*d*n*(n+1) / t_layer; `ms_per_step` is the per-layer latency; tokens kept,
per-kernel times, the dense run of the same attention kernel, the roofline of
the dominant kernel and the CPU-oracle baseline ride along in the same object.
"""
import argparse
import json
import os
import sys
import time

ROOT = os.path.dirname(os.path.abspath(__file__))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

MFMA_BF16_PEAK_TFLOPS = 2500.0      # MI355X dense bf16 matrix peak
MFMA_FP32_PEAK_TFLOPS = 157.3
HBM_PEAK_GBS = 8000.0
PAGE = 64                # rows of a page of the paged caches (--paged)
PREFILL_KERNELS = ("score_rowstats", "score_colsum", "select", "compact_kv", "pack_kv", "flash_kept")


def read_traffic(kernel: str, workload: str):
    """HBM bytes per launch measured with rocprofv3 --pmc (FETCH_SIZE, WRITE_SIZE),
    kept as text under profiles/; None when no measurement is stored."""
    path = os.path.join(ROOT, "profiles", "hbm_traffic.txt")
    if not os.path.exists(path):
        return None
    for line in open(path):
        f = line.split()
        if len(f) >= 4 and not line.startswith("#") and f[0] == kernel and f[1] == workload:
            return float(f[2]) + float(f[3])
    return None


TRAFFIC_NOTE = ("stored measurement: rocprofv3 --pmc FETCH_SIZE + WRITE_SIZE of this command, scaled by the copy calibration "
                "(profiles/hbm_traffic.txt); not re-measured in this run")


def cpu_baseline_stack(samples, spec, tau, dense_flops, n_layers):
    """The CPU oracle on a bounded sample of the stack: for each sampled layer, batch element 0 and 4 of the
    32 heads - score, select, compaction, kept-token attention (prefill) and one decode step (append + Eq. (5))
    over the evicted cache of those heads; times scaled to all heads, batch elements and layers."""
    import numpy as np
    from oracle import zipvl_oracle as oz
    try:
        from threadpoolctl import threadpool_info
        threads = max([p.get("num_threads", 1) for p in threadpool_info()] or [1])
    except Exception:
        threads = os.cpu_count() or 1
    t_prefill = t_decode = 0.0
    r = np.random.Generator(np.random.PCG64(9))
    for (li, Q, K, V, probe, scale) in samples:
        hs = Q.shape[0]
        t0 = time.perf_counter()
        mass, rank = oz.token_scores(Q, K, probe, scale)
        sel = [oz.select(mass[g].astype(np.float32), rank[g].astype(np.float32), tau) for g in range(hs)]
        caches = [oz.compact_kv(K[g], V[g], sel[g][1]) for g in range(hs)]
        for g in range(hs):
            oz.kept_token_attention(Q[g], K[g], V[g], sel[g][1], scale)
        t_prefill += time.perf_counter() - t0
        q, kn, vn = (r.standard_normal((hs, spec.d)) for _ in range(3))
        t0 = time.perf_counter()
        for g in range(hs):
            oz.decode_step(q[g], kn[g], vn[g], caches[g][0], caches[g][1], caches[g][2], scale)
        t_decode += time.perf_counter() - t0
    heads_sampled = sum(s[1].shape[0] for s in samples)
    per_head_layer = t_prefill / heads_sampled
    t_layer = per_head_layer * spec.Hq * spec.B
    return {
        "value": dense_flops / t_layer / 1e12, "unit": "TFLOP/s (dense-equivalent)", "cores": int(threads), "kind": "oracle",
        "sample": f"layers {[s[0] for s in samples]}, batch element 0, heads 0..{samples[0][1].shape[0] - 1}: score + select + compaction + "
                  f"kept-token attention timed whole, scaled x{spec.Hq * spec.B / samples[0][1].shape[0]:.0f} to {spec.B} x {spec.Hq} heads per layer "
                  "(extrapolated); decode: one oracle step (append + attention) on the same heads' evicted caches, scaled to "
                  f"{spec.B * spec.Hq} units x {n_layers} layers",
        "ms_per_layer_extrapolated": 1e3 * t_layer,
        "decode_ms_per_step_extrapolated": 1e3 * t_decode / heads_sampled * spec.Hq * spec.B * n_layers,
        "parts_s": {"prefill_sample": t_prefill, "decode_sample": t_decode},
        "host_cpu_count": os.cpu_count(),
    }


def cpu_baseline(w, tau, dense_flops):
    """The CPU oracle as it stands, timed on a bounded sample of the same layer."""
    import numpy as np
    from oracle import zipvl_oracle as oz
    try:
        from threadpoolctl import threadpool_info
        threads = max([p.get("num_threads", 1) for p in threadpool_info()] or [1])
    except Exception:
        threads = os.cpu_count() or 1
    spec = w.spec
    G = spec.Hq // spec.Hkv
    t0 = time.perf_counter()
    mass, rank = oz.token_scores(w.Q[0], w.K[0], w.probe_pos, w.scale)
    t_score = time.perf_counter() - t0
    t0 = time.perf_counter()
    sel = [oz.select(mass[g].astype(np.float32), rank[g].astype(np.float32), tau) for g in range(spec.Hkv)]
    t_select = time.perf_counter() - t0
    t0 = time.perf_counter()
    for g in range(spec.Hkv):
        oz.compact_kv(w.K[0, g], w.V[0, g], sel[g][1])
    t_compact = time.perf_counter() - t0
    # attention: query heads in an order that visits every KV group in turn, until all are done or 20 s have passed;
    # the time is scaled to all heads when the budget cuts the sample short
    order = [g * G + j for j in range(G) for g in range(spec.Hkv)]
    done = 0
    t0 = time.perf_counter()
    for hq in order:
        g = hq // G
        oz.kept_token_attention(w.Q[0, hq], w.K[0, g], w.V[0, g], sel[g][1], w.scale)
        done += 1
        if time.perf_counter() - t0 > 20.0:
            break
    t_attn_sample = time.perf_counter() - t0
    t_attn = t_attn_sample * spec.Hq / done
    t_layer = (t_score + t_select + t_compact + t_attn) * spec.B
    return {
        "value": dense_flops / t_layer / 1e12, "unit": "TFLOP/s (dense-equivalent)", "cores": int(threads),
        "kind": "oracle",
        "sample": f"batch 0: score+select+compaction on all {spec.Hkv} units (timed whole); kept-token attention on "
                  f"{done} of {spec.Hq} query heads" + ("" if done == spec.Hq else f", time scaled x{spec.Hq / done:.2f}")
                  + (f", then x{spec.B} batches" if spec.B > 1 else ""),
        "ms_per_layer_extrapolated": 1e3 * t_layer,
        "parts_s": {"score": t_score, "select": t_select, "compact": t_compact, "attention_sample": t_attn_sample},
        "host_cpu_count": os.cpu_count(),
    }


def run_stack(args):
    """Shape 5: 32 layers x [B4, 32 heads, n 8192, d 128] bf16.  Full prefill (score, select, compaction,
    kept-token attention per layer) and then memory-bound decode steps (cache append + one-query
    attention over every layer) against the evicted caches and against the full caches."""
    import numpy as np
    import torch

    import paper_2410_08584_amd as z
    from workloads import CONFIGS, make_stack_layer_device

    z.load_library()
    dev = "cuda:0"
    spec = CONFIGS[5]
    B, H, n, d = spec.B, spec.Hq, spec.n, spec.d
    L = args.layers or spec.layers
    steps_dec = args.decode_steps
    units = B * H
    tau = spec.taus[0]
    e = 2
    mass = torch.empty((units, n), dtype=torch.float32, device=dev)
    rank = torch.empty_like(mass)
    idx = torch.empty((units, n), dtype=torch.int32, device=dev)
    k = torch.empty((units,), dtype=torch.int32, device=dev)
    O = torch.empty((B, H, n, d), dtype=torch.bfloat16, device=dev)
    Kt = torch.empty((units, n, d), dtype=torch.bfloat16, device=dev)
    Vt = torch.empty_like(Kt)
    lt = torch.empty((units,), dtype=torch.int32, device=dev)
    Kt4, Vt4 = Kt.view(B, H, n, d), Vt.view(B, H, n, d)
    ws_s = ws_p = None
    caches, fulls, quants, paged, kept, layer_ms, samples = [], [], [], [], [], [], []
    kern_us = {}
    sample_layers = {0, (L - 1) // 2, L - 1}
    ev0, ev1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for layer in range(L):
        li = layer * (spec.layers - 1) // max(1, L - 1) if L < spec.layers else layer   # spread over the ramp
        Q, K, V, probe, scale = make_stack_layer_device(li, dev)
        if ws_s is None:
            dm = z.dims_of(Q, K, V)
            ws_s = torch.empty(max(256, z.workspace_bytes(z.OP_SCORE, dm, len(probe))), dtype=torch.uint8, device=dev)
            ws_p = torch.empty(max(256, z.workspace_bytes(z.OP_SPARSE_PREFILL, dm)), dtype=torch.uint8, device=dev)

        def one_layer():
            z.zipvl_score(Q, K, probe, scale, mass=mass, rank=rank, ws=ws_s)
            z.zipvl_select(mass, rank, tau, idx=idx, k=k)
            z.zipvl_compact_kv(K, V, idx, k, n, Kc=Kt, Vc=Vt, length=lt)
            z.zipvl_sparse_prefill(Q, Kt4, Vt4, idx, k, scale, z.OUT_FULL | z.KV_ALREADY_COMPACT, O=O, ws=ws_p)
        for _ in range(max(1, args.warmup)):           # warm-up of this layer's shapes
            one_layer()
        torch.cuda.synchronize()
        if layer in sample_layers and not args.no_cpu_baseline:
            samples.append((li, Q[0, :4].float().cpu().numpy(), K[0, :4].float().cpu().numpy(), V[0, :4].float().cpu().numpy(), probe, scale))
        ev0.record()
        for _ in range(args.steps):
            one_layer()
        ev1.record()
        torch.cuda.synchronize()
        layer_ms.append(ev0.elapsed_time(ev1) / args.steps)
        z.zipvl_timing_enable(True)                    # per-kernel times of this layer (library events), outside the timed region
        one_layer(); one_layer()
        torch.cuda.synchronize()
        for name in PREFILL_KERNELS:
            ms, cnt = z.zipvl_timing_read(z.KERNELS.index(name))
            if cnt:
                kern_us[name] = kern_us.get(name, 0.0) + 1e3 * ms / cnt
        z.zipvl_timing_enable(False)
        k_h = k.cpu().numpy().astype(np.int64)
        kept.append(k_h / n)
        cap_c = int(k_h.max()) + steps_dec + 8
        Kc = Kt[:, :cap_c].contiguous(); Vc = Vt[:, :cap_c].contiguous()
        caches.append((Kc, Vc, lt.clone(), cap_c))
        cap_f = n + steps_dec + 8
        Kf = torch.empty((units, cap_f, d), dtype=torch.bfloat16, device=dev); Vf = torch.empty_like(Kf)
        Kf[:, :n] = K.reshape(units, n, d); Vf[:, :n] = V.reshape(units, n, d)
        fulls.append((Kf, Vf, torch.full((units,), n, dtype=torch.int32, device=dev), cap_f))
        if args.quantized:
            # every token stays: T at 4 bits, the others at 2 bits; rows appended while decoding go to a bf16 tail
            qc = z.zipvl_quantize_kv(K, V, idx, k, int(k_h.max()), n - int(k_h.min()))
            cap_t = steps_dec + 8
            quants.append((qc, torch.empty((units, cap_t, d), dtype=torch.bfloat16, device=dev),
                           torch.empty((units, cap_t, d), dtype=torch.bfloat16, device=dev),
                           torch.zeros((units,), dtype=torch.int32, device=dev)))
        if args.paged:
            # the same rows as a prefix in pages, and pages for what args.paged conversations about each prompt will say
            own_pages = units * args.paged * (-(-(steps_dec + 8) // PAGE))
            width = -(-int(k_h.max()) // PAGE)
            cache = z.PagedCache.empty(units * width + own_pages, PAGE, d, torch.bfloat16, dev)
            order = torch.randperm(cache.num_pages, device=dev, dtype=torch.int64).to(torch.int32)
            ptable, otable = order[:units * width].view(units, width), order[units * width:].view(units * args.paged, -1)
            plen, _ = z.zipvl_paged_append(K, V, cache, ptable, torch.zeros_like(k), idx=idx, k=k, length=torch.empty_like(k))
            paged.append((cache, ptable, plen, otable, torch.zeros((units * args.paged,), dtype=torch.int32, device=dev)))
        del Q, K, V
    kept = np.stack(kept)
    gen = torch.Generator(device=dev); gen.manual_seed(12345)
    q = torch.randn((units, d), generator=gen, device=dev).to(torch.bfloat16)
    kn = torch.randn((units, d), generator=gen, device=dev).to(torch.bfloat16)
    vn = torch.randn((units, d), generator=gen, device=dev).to(torch.bfloat16)
    o = torch.empty((units, d), dtype=torch.bfloat16, device=dev)
    dmf = z.dims_of(None, None, None, B=B, Hq=H, Hkv=H, n=fulls[0][3], d=d, dtype=1)
    ws_d = torch.empty(max(256, z.workspace_bytes(z.OP_DECODE, dmf)), dtype=torch.uint8, device=dev)

    def decode(stack, nsteps):
        for _ in range(nsteps):
            for (Kc, Vc, ln, cap) in stack:
                z.zipvl_kv_append(Kc, Vc, ln, kn, vn, B=B, Hkv=H)
                z.zipvl_decode_attn(q, Kc, Vc, ln, 1.0 / float(np.sqrt(d)), B=B, Hq=H, Hkv=H, o=o, ws=ws_d)

    def timed_decode(run_steps, lens):
        """Eager steps, then the same step replayed from a HIP graph (the lengths live on the device and
        the append advances them there, so one captured step serves every position).  The replay is used
        only if it reproduces the eager output from the same starting lengths."""
        snap = [l.clone() for l in lens]
        def reset():
            for l, s0 in zip(lens, snap):
                l.copy_(s0)
        run_steps(2)
        torch.cuda.synchronize()
        o_ref = o.clone()
        t0 = time.perf_counter()
        run_steps(steps_dec - 2)
        torch.cuda.synchronize()
        eager = (time.perf_counter() - t0) / (steps_dec - 2)
        graph = None
        if not args.no_graph:
            reset()
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                run_steps(1)
            torch.cuda.current_stream().wait_stream(side)
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                run_steps(1)
            reset()
            torch.cuda.synchronize()
            g.replay(); g.replay()
            torch.cuda.synchronize()
            if torch.equal(o, o_ref):
                t0 = time.perf_counter()
                for _ in range(steps_dec - 2):
                    g.replay()
                torch.cuda.synchronize()
                graph = (time.perf_counter() - t0) / (steps_dec - 2)
        return eager, graph

    def entry(bytes_step, eager, graph, **extra):
        use_graph = graph is not None and graph < eager     # queued eager launches already run back to back
        dt = graph if use_graph else eager
        return {"ms_per_step": 1e3 * dt, "GBps": bytes_step / dt / 1e9, "GB_read_per_step": bytes_step / 1e9,
                "launch": "hipgraph replay of one decode step (output verified against the eager steps)" if use_graph else "eager",
                "eager_ms_per_step": 1e3 * eager, "hipgraph_ms_per_step": None if graph is None else 1e3 * graph, **extra}

    def decode_fused(stack, wss, nsteps):
        for _ in range(nsteps):
            for (Kc, Vc, ln, cap), wsf in zip(stack, wss):
                z.zipvl_decode_step(q, Kc, Vc, ln, kn, vn, 1.0 / float(np.sqrt(d)), B=B, Hq=H, Hkv=H, ws=wsf, o=o)

    res = {}
    for name, stack in (("evicted", caches), ("full", fulls)):
        len0 = [int(s[2].sum().item()) for s in stack]
        lens = [s[2] for s in stack]
        snap = [l.clone() for l in lens]
        eager, graph = timed_decode(lambda ns, st=stack: decode(st, ns), lens)
        rows = sum(l0 + units * (2 + (steps_dec - 2 + 1) / 2.0) for l0 in len0)     # mean cached rows read per step
        two_call = entry(2.0 * rows * d * e, eager, graph)
        for l, s0 in zip(lens, snap):
            l.copy_(s0)
        wss = [z.decode_step_workspace(B, H, H, cap, d, Kc) for (Kc, _, _, cap) in stack]
        eager, graph = timed_decode(lambda ns, st=stack, w_=wss: decode_fused(st, w_, ns), lens)
        res[name] = entry(2.0 * rows * d * e, eager, graph, kernels="zipvl_decode_step (append, attention and merge in one launch per layer)",
                          two_call_ms_per_step=two_call["ms_per_step"])
    if args.quantized:
        ws_q = torch.empty(max(256, z.workspace_bytes(z.OP_DECODE_Q, dmf)), dtype=torch.uint8, device=dev)

        def decode_q(nsteps):
            for _ in range(nsteps):
                for (qc, Kt, Vt, lt_) in quants:
                    z.zipvl_kv_append(Kt, Vt, lt_, kn, vn, B=B, Hkv=H)
                    z.zipvl_decode_attn_q(q, qc, 1.0 / float(np.sqrt(d)), B=B, Hq=H, Hkv=H, K_tail=Kt, V_tail=Vt,
                                          len_tail=lt_, o=o, ws=ws_q)
        eager, graph = timed_decode(decode_q, [qq[3] for qq in quants])
        rows_hi = sum(int(qc.len_hi.sum().item()) for qc, _, _, _ in quants)
        rows_lo = sum(int(qc.len_lo.sum().item()) for qc, _, _, _ in quants)
        tail_rows = len(quants) * units * (2 + (steps_dec - 2 + 1) / 2.0)
        bytes_step = 2.0 * (rows_hi * (d // 2 + 4) + rows_lo * (d // 4 + 4) + tail_rows * d * e)
        res["quantised_4_2bit"] = entry(bytes_step, eager, graph,
                                        bits_per_element_incl_params=8.0 * (rows_hi * (d // 2 + 4) + rows_lo * (d // 4 + 4)) / ((rows_hi + rows_lo) * d),
                                        note="all prefill tokens stay in the cache (important ones 4 bit, the others 2 bit), appended rows bf16")
    if args.paged:
        # a decode step of B * args.paged conversations: query, key rotated, key and value into pages, attention over the prompt's prefix and their own
        Bp = B * args.paged
        rope = z.Rope.of_sections((d // 2 - 2 * (3 * d // 16), 3 * d // 16, 3 * d // 16))
        begin = torch.arange(0, Bp + 1, args.paged, dtype=torch.int32, device=dev)
        qp, kp, vp = (torch.randn((Bp, H, 1, d), generator=gen, device=dev).to(torch.bfloat16) for _ in range(3))
        pos = torch.full((3, Bp, 1), n, dtype=torch.int32, device=dev)
        qr = torch.empty_like(qp)
        op = torch.empty((Bp * H, d), dtype=torch.bfloat16, device=dev)
        o = op                                               # what the replay is compared by
        ws_g = z.decode_paged_workspace(paged[0][0], paged[0][3], paged[0][1], B=Bp, Hq=H, Hkv=H)

        def decode_paged(nsteps):
            for _ in range(nsteps):
                for (cache, ptable, plen, otable, olen) in paged:
                    z.zipvl_paged_append(kp, vp, cache, otable, olen, pos=pos, rope=rope, Q=qp, Qo=qr)
                    z.zipvl_decode_attn_paged(qr, cache, otable, olen, 1.0 / float(np.sqrt(d)), B=Bp, Hq=H, Hkv=H, prefix_table=ptable,
                                              prefix_len=plen, group_begin=begin, o=op, ws=ws_g)
                pos.add_(1)
        eager, graph = timed_decode(decode_paged, [pp[4] for pp in paged] + [pos])
        rows = sum(int(pp[2].sum().item()) for pp in paged) + L * H * Bp * (2 + (steps_dec - 2 + 1) / 2.0)
        res["paged_shared_prefix"] = entry(2.0 * rows * d * e, eager, graph, conversations=Bp, page=PAGE,
                                           note=f"{args.paged} conversations about each of the {B} prompts share its evicted cache, which is read once for all of them")
    ms_layer = float(np.mean(layer_ms))
    dense_flops = 2.0 * B * H * d * n * (n + 1)
    out = {
        "metric": "sparse-prefill dense-equivalent TFLOP/s (ms/layer in ms_per_step, tokens kept % in kept_pct)",
        "value": dense_flops / (ms_layer * 1e-3) / 1e12, "unit": "TFLOP/s (dense-equivalent)",
        "n_gpus": 1, "steps": args.steps, "warmup": max(1, args.warmup), "ms_per_step": ms_layer, "higher_is_better": True,
        "scaling": "weak", "vs_baseline": None, "dtype": "bf16", "data": "synthetic (seeded torch device generator)",
        "config": {"workload": spec.name, "layers": L, "B": B, "Hq": H, "Hkv": H, "n": n, "d": d, "tau": tau,
                   "decode_steps": steps_dec},
        "kept_pct": 100.0 * float(kept.mean()), "kept_pct_first_last_layer": [100.0 * float(kept[0].mean()), 100.0 * float(kept[-1].mean())],
        "layer_ms_first_last": [layer_ms[0], layer_ms[-1]],
        "prefill_kernels_avg_us": {name: v / L for name, v in kern_us.items()},
        "decode": res, "decode_speedup_evicted_vs_full": res["full"]["ms_per_step"] / res["evicted"]["ms_per_step"],
        "roofline": {"kernel": "decode_step_kernel (evicted caches)", "bound": "hbm", "achieved": res["evicted"]["GBps"],
                     "peak": HBM_PEAK_GBS, "unit": "GB/s", "frac": res["evicted"]["GBps"] / HBM_PEAK_GBS,
                     "traffic": read_traffic("decode_step_kernel", spec.name + "-evicted"), "traffic_source": TRAFFIC_NOTE,
                     "bytes_per_launch": res["evicted"]["GB_read_per_step"] * 1e9 / L,
                     "avg_launch_us": 1e3 * res["evicted"]["ms_per_step"] / L,
                     "note": "whole decode step (one fused launch per layer: append, split-KV attention, merge); achieved = algorithmic "
                             "bytes of a step (2 x cached rows x d x 2 B over all layers) / step time; per launch: both divided by the layer count"},
        "paper_context": "paper reports 2.8x decode throughput at 16K tokens on one A100 (larger batch fits after eviction)",
    }
    if not args.no_peaks:
        tf, gb = z.zipvl_probe_peaks(dev)
        out["measured_peaks"] = {"mfma_bf16_TFLOPs": tf, "read_GBps": gb,
                                 "note": "sustained by this GPU in the library's probe kernels (independent MFMA chains; one 4 GiB read)"}
        out["roofline"]["frac_of_measured_peak"] = res["evicted"]["GBps"] / gb
    if not args.no_cpu_baseline:
        out["cpu_baseline"] = cpu_baseline_stack(samples, spec, tau, dense_flops, L)
    if args.copy_calibration:
        src = torch.empty(256 << 20, dtype=torch.uint8, device=dev).fill_(1)
        dst = torch.empty_like(src)
        for _ in range(3):
            dst.copy_(src)
        torch.cuda.synchronize()
    print(json.dumps(out))


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--gpus", type=int, default=1)
    ap.add_argument("--steps", type=int, default=50)
    ap.add_argument("--warmup", type=int, default=10)
    ap.add_argument("--workload", type=int, default=4, help="benchmark shape 1..5 (default 4: long video, GQA, 18432 tokens; "
                    "5 = 32-layer stack with decode steps)")
    ap.add_argument("--layers", type=int, default=0, help="shape 5: number of layers (default all 32)")
    ap.add_argument("--decode-steps", type=int, default=256, help="shape 5: decode steps per cache kind")
    ap.add_argument("--gamma", type=float, default=None, help="query-mean strength of the generator (default 1.75)")
    ap.add_argument("--probes", choices=["recent", "hybrid"], default="recent",
                    help="probe rows: the last 64 positions (benchmark configs) or the paper's 64 recent + 64 random")
    ap.add_argument("--score", choices=["probes", "all-rows"], default="probes",
                    help="token scores from the probe rows (the method) or from every row of the attention matrix "
                         "(exact Eq. (6)/(8): the accuracy reference, two more passes over the causal half of Q K^T)")
    ap.add_argument("--select", choices=["per-head", "per-layer"], default="per-head",
                    help="one important set per (batch, KV head) (benchmark configs) or one per batch element, "
                         "selected from the head-averaged scores")
    ap.add_argument("--quantized", action="store_true",
                    help="shape 5: also decode against the mixed-precision cache (important tokens 4 bit, the others 2 bit)")
    ap.add_argument("--paged", type=int, default=0, metavar="CONVERSATIONS",
                    help="shape 5: also decode steps of that many conversations about each prompt, over paged caches that share the evicted prefix")
    ap.add_argument("--no-peaks", action="store_true", help="skip the two probe kernels (sustained bf16 MFMA rate, sustained read bandwidth)")
    ap.add_argument("--no-cpu-baseline", action="store_true")
    ap.add_argument("--no-dense", action="store_true")
    ap.add_argument("--no-graph", action="store_true", help="skip the HIP-graph replay of the step")
    ap.add_argument("--copy-calibration", action="store_true",
                    help="also run 3 plain device copies of 256 MiB (a kernel of known HBM traffic, for scaling "
                         "the FETCH_SIZE / WRITE_SIZE counters of a rocprofv3 --pmc run)")
    args = ap.parse_args()
    if args.gpus != 1:
        print("bench.py: this build runs on one GPU only (no sharding, no collectives); use --gpus 1", file=sys.stderr)
        sys.exit(2)

    if args.workload == 5:
        if args.steps == 50:
            args.steps = 3
        if args.warmup == 10:
            args.warmup = 2
        return run_stack(args)

    import numpy as np
    import torch

    import paper_2410_08584_amd as z
    from workloads import make_workload
    from workloads.generators import GAMMA_DEFAULT

    z.load_library()                                  # raises if the HIP library is not built
    assert torch.cuda.is_available(), "bench.py needs a GPU"
    dev = "cuda:0"
    gamma = GAMMA_DEFAULT if args.gamma is None else args.gamma
    w = make_workload(args.workload, gamma=gamma)
    if args.probes == "hybrid":
        from workloads import hybrid_probes
        w.probe_pos = hybrid_probes(w.spec.n, seed=w.seed)
    spec, tau = w.spec, w.tau
    B, Hq, Hkv, n, d = spec.B, spec.Hq, spec.Hkv, spec.n, spec.d
    tdt = torch.bfloat16 if spec.dtype == "bf16" else torch.float32
    Q, K, V = (torch.from_numpy(a).to(dev).to(tdt) for a in (w.Q, w.K, w.V))
    units = B * Hkv

    dm = z.dims_of(Q, K, V)
    mass = torch.empty((units, n), dtype=torch.float32, device=dev)
    rank = torch.empty_like(mass)
    idx = torch.empty((units, n), dtype=torch.int32, device=dev)
    k = torch.empty((units,), dtype=torch.int32, device=dev)
    Kc = torch.empty((units, n, d), dtype=tdt, device=dev)
    Vc = torch.empty_like(Kc)
    Kc4, Vc4 = Kc.view(B, Hkv, n, d), Vc.view(B, Hkv, n, d)     # the evicted cache, as the attention call takes it
    ln = torch.empty((units,), dtype=torch.int32, device=dev)
    O = torch.empty((B, Hq, n, d), dtype=tdt, device=dev)
    ws_s = torch.empty(max(256, z.workspace_bytes(z.OP_SCORE, dm, len(w.probe_pos))), dtype=torch.uint8, device=dev)
    ws_p = torch.empty(max(256, z.workspace_bytes(z.OP_SPARSE_PREFILL, dm)), dtype=torch.uint8, device=dev)

    shared = args.select == "per-layer"
    if shared:                                              # one T per batch element: scores averaged over the KV heads
        mass_b = torch.empty((B, n), dtype=torch.float32, device=dev)
        rank_b = torch.empty_like(mass_b)
        idx = torch.empty((B, n), dtype=torch.int32, device=dev)
        k = torch.empty((B,), dtype=torch.int32, device=dev)
    tflag = z.T_PER_BATCH if shared else 0

    exact = args.score == "all-rows"
    if exact:
        ws_s = torch.empty(max(256, z.workspace_bytes(z.OP_SCORE_ALL_ROWS, dm)), dtype=torch.uint8, device=dev)

    def step():
        if exact:
            z.zipvl_score_all_rows(Q, K, w.scale, mass=mass, rank=rank, ws=ws_s)
        else:
            z.zipvl_score(Q, K, w.probe_pos, w.scale, mass=mass, rank=rank, ws=ws_s)
        if shared:
            z.zipvl_share_scores(mass, rank, B, mass_b=mass_b, rank_b=rank_b)
            z.zipvl_select(mass_b, rank_b, tau, idx=idx, k=k)
        else:
            z.zipvl_select(mass, rank, tau, idx=idx, k=k)
        z.zipvl_compact_kv(K, V, idx, k, n, tflag, Kc=Kc, Vc=Vc, length=ln)
        z.zipvl_sparse_prefill(Q, Kc4, Vc4, idx, k, w.scale, z.OUT_FULL | z.KV_ALREADY_COMPACT | tflag, O=O, ws=ws_p)

    # What this GPU sustains (two probe kernels of the library), measured before the workload: part of the set-up,
    # like the allocations above, and it leaves the clocks where a busy GPU has them.
    peaks = None if args.no_peaks else z.zipvl_probe_peaks(dev)

    for _ in range(args.warmup):
        step()
    torch.cuda.synchronize()
    z.zipvl_timing_enable(True)
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    for _ in range(args.steps):
        step()
    torch.cuda.synchronize()
    t1 = time.perf_counter()
    kern = {}
    for kid, name in enumerate(z.KERNELS):
        ms, cnt = z.zipvl_timing_read(kid)
        if cnt:
            kern[name] = {"avg_us": 1e3 * ms / cnt, "launches": cnt}
    z.zipvl_timing_enable(False)
    ms_per_step = 1e3 * (t1 - t0) / args.steps

    # The same step replayed from a HIP graph (no host launch cost, shorter gaps between the dependent
    # kernels): reported beside the eager number; every checked replay must reproduce the eager output.
    graph_ms = None
    if not args.no_graph:
        O_ref, idx_ref, k_ref = O.clone(), idx.clone(), k.clone()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        ok = True
        for _ in range(3):
            O.fill_(1.0); k.zero_()
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            ok = ok and torch.equal(O, O_ref) and torch.equal(k, k_ref) and torch.equal(idx, idx_ref)
            step()                                           # eager work between the replays
            torch.cuda.synchronize()
        if ok:
            for _ in range(args.warmup):                     # the checks above left gaps: warm-up replays, then the timed ones
                g.replay()
            torch.cuda.synchronize()
            t0 = time.perf_counter()
            for _ in range(args.steps):
                g.replay()
            torch.cuda.synchronize()
            graph_ms = 1e3 * (time.perf_counter() - t0) / args.steps
        else:
            graph_ms = None
    eager_ms = ms_per_step
    launch_mode = "eager (one C-ABI call per stage, HIP events around every kernel)"
    if graph_ms is not None:
        ms_per_step = graph_ms                               # same kernels, same step, replayed from the graph
        launch_mode = "hipgraph replay of the four C-ABI calls (outputs verified against the eager step)"

    k_h = k.cpu().numpy().astype(np.int64)
    if shared:
        k_h = np.repeat(k_h, Hkv)                            # every KV head of a batch element keeps the same k
    G = Hq // Hkv
    dense_flops = 2.0 * B * Hq * d * n * (n + 1)
    kept_flops = float(sum(G * 2.0 * d * kk * (kk + 1) for kk in k_h))
    r = k_h / n

    dense_ms = None
    if not args.no_dense:
        for _ in range(2):
            z.zipvl_sparse_prefill(Q, K, V, None, None, w.scale, O=O, ws=ws_p)
        torch.cuda.synchronize()
        reps = 5
        t0 = time.perf_counter()
        for _ in range(reps):
            z.zipvl_sparse_prefill(Q, K, V, None, None, w.scale, O=O, ws=ws_p)
        torch.cuda.synchronize()
        dense_ms = 1e3 * (time.perf_counter() - t0) / reps

    if args.copy_calibration:
        src = torch.empty(256 << 20, dtype=torch.uint8, device=dev).fill_(1)
        dst = torch.empty_like(src)
        for _ in range(3):
            dst.copy_(src)
        torch.cuda.synchronize()

    flash_us = kern["flash_kept"]["avg_us"]
    peak = MFMA_BF16_PEAK_TFLOPS if spec.dtype == "bf16" else MFMA_FP32_PEAK_TFLOPS
    achieved = kept_flops / (flash_us * 1e-6) / 1e12
    roofline = {"kernel": "flash_kept_kernel", "bound": "mfma", "achieved": achieved, "peak": peak,
                "unit": "TFLOP/s", "frac": achieved / peak,
                "traffic": read_traffic("flash_kept_kernel", spec.name), "traffic_source": TRAFFIC_NOTE,
                "flops_per_launch": kept_flops, "avg_launch_us": flash_us}
    e = 2 if spec.dtype == "bf16" else 4
    hbm = {}
    sc_bytes = B * Hkv * n * d * e + B * Hq * len(w.probe_pos) * d * e + 2 * units * n * 4
    if "score_rowstats" in kern:
        hbm["score_rowstats"] = sc_bytes / (kern["score_rowstats"]["avg_us"] * 1e-6) / 1e9
        hbm["score_colsum"] = sc_bytes / (kern["score_colsum"]["avg_us"] * 1e-6) / 1e9
    hbm["select"] = float(units * (8 * n) + 4 * k_h.sum() + 4 * units) / (kern["select"]["avg_us"] * 1e-6) / 1e9
    kv_bytes = float(sum(2 * 2 * kk * d * e + 4 * kk for kk in k_h))
    hbm["compact_kv"] = kv_bytes / (kern["compact_kv"]["avg_us"] * 1e-6) / 1e9
    if "pack_kv" in kern:                                    # not launched when the evicted cache is read in place
        hbm["pack_kv"] = kv_bytes / (kern["pack_kv"]["avg_us"] * 1e-6) / 1e9

    out = {
        "metric": "sparse-prefill dense-equivalent TFLOP/s (ms/layer in ms_per_step, tokens kept % in kept_pct)",
        "value": dense_flops / (ms_per_step * 1e-3) / 1e12,
        "unit": "TFLOP/s (dense-equivalent)",
        "n_gpus": 1, "steps": args.steps, "warmup": args.warmup, "ms_per_step": ms_per_step,
        "higher_is_better": True, "scaling": "weak", "vs_baseline": None,
        "dtype": spec.dtype, "data": "synthetic",
        "config": {"workload": spec.name, "B": B, "Hq": Hq, "Hkv": Hkv, "n": n, "d": d, "tau": tau,
                   "probes": ("every row (exact scores)" if exact else f"last {len(w.probe_pos)}" if args.probes == "recent" else "64 recent + 64 random"), "gamma": gamma, "seed": w.seed,
                   "important_set": "per (batch, KV head)" if not shared else "per batch element (head-averaged scores)"},
        "kept_pct": 100.0 * float(r.mean()), "kept_sq_pct": 100.0 * float((r * r).mean()),
        "k_per_unit": [int(x) for x in k_h[:16]],
        "kernels": kern,
        "hbm_GBps_algorithmic": hbm,
        "launch": launch_mode, "eager_ms_per_step_with_kernel_events": eager_ms, "hipgraph_ms_per_step": graph_ms,
        "dense_same_kernel_ms": dense_ms,
        "sparse_speedup_vs_dense": (dense_ms / ms_per_step) if dense_ms else None,
        "roofline": roofline,
        "paper_context": "paper reports 2.3x prefill (128K tokens) and 2.8x decode throughput (16K) on one A100, LLaVA-Next-13B",
    }
    if peaks is not None:
        tf, gb = peaks
        out["measured_peaks"] = {"mfma_bf16_TFLOPs": tf, "read_GBps": gb,
                                 "note": "sustained by this GPU in the library's probe kernels (independent MFMA chains; one 4 GiB read)"}
        if spec.dtype == "bf16":
            out["roofline"]["frac_of_measured_peak"] = achieved / tf
    if not args.no_cpu_baseline:
        out["cpu_baseline"] = cpu_baseline(w, tau, dense_flops)
    print(json.dumps(out))


if __name__ == "__main__":
    main()
