#!/usr/bin/env python3
"""SpMM throughput of the hyb(c,k) path on one MI355X.

One "step" is one sptir_spmm call (Y = A X on the decomposed matrix, every
launch it enqueues) with A, X and Y resident in HBM.  The format conversion
(sptir_hyb_build) is pre-processing of a stationary matrix, as in the paper,
and is timed separately.  The workload is the largest graph of the benchmark
set (232,965 rows, ~114.6M non-zeros, hyb(16, 11)) at the metric's feature
size 128; the same graph at its as-written feature size 256 and the four
smaller configurations are reported in extra keys of the same JSON line.
"""
from __future__ import annotations

import argparse
import ctypes
import glob
import hashlib
import json
import os
import sys
import time

ROOT = os.path.dirname(os.path.abspath(__file__))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

HBM_PEAK_GBS = 8000.0          # MI355X HBM3E, published
GATHER_THEORY_GBS = 39300.0    # 256 CUs x 64 B/clk x 2.4 GHz: what the vector-memory return path could carry
FMA_PEAK_TFLOPS = 157.3        # fp32 vector, published (plain v_fma_f32 measures ~129 here: the packed forms are not needed)


def bytes_min(nnz, n_rows, n_cols, feat):
    """Minimal-traffic byte model: every true non-zero's column and value once, X once, Y once."""
    return 8.0 * nnz + 4.0 * n_cols * feat + 4.0 * n_rows * feat


def bytes_hyb(info, n_rows, n_cols, feat):
    """What the decomposition as stored has to move at the least: every ELL slot (pads included) and row id,
    every remainder non-zero and piece descriptor, X once, Y once."""
    return (8.0 * info["n_ell_slots"] + 4.0 * info["n_ell_rows"] + 8.0 * info["n_rem_nnz"] + 12.0 * info["n_rem_pieces"]
            + 4.0 * n_cols * feat + 4.0 * n_rows * feat)


def bytes_build(info, nnz, n_rows):
    """Algorithmic bytes of sptir_hyb_build: the CSR read twice (validation reads column ids and values; the scatter
    reads both again; the piece boundaries come from a few probes per row piece), the canonical slots and the SpMM
    stream written."""
    slots = info["n_ell_slots"] + info["n_rem_nnz"]
    return 4.0 * nnz + 4.0 * nnz + 8.0 * nnz + 8.0 * slots + 8.0 * nnz + 8.0 * n_rows


def source_fingerprint():
    """Hash of the HIP sources (without those of the mixture-of-experts operators, which nothing here calls): a profile summary
    taken on other sources says nothing about this build."""
    h = hashlib.sha1()
    for path in sorted(glob.glob(os.path.join(ROOT, "paper_2207_04606_amd", "csrc", "*"))):
        if path.endswith((".hip", ".h")) and not os.path.basename(path).startswith("moe"):
            h.update(open(path, "rb").read())
    return h.hexdigest()[:12]


def time_spmm(sptir, torch, hyb, X, Y, steps, warmup):
    for _ in range(warmup):
        sptir.sptir_spmm(hyb, X, Y)
    torch.cuda.synchronize()
    e0 = torch.cuda.Event(enable_timing=True)
    e1 = torch.cuda.Event(enable_timing=True)
    t0 = time.perf_counter()
    e0.record()
    for _ in range(steps):
        sptir.sptir_spmm(hyb, X, Y)
    e1.record()
    torch.cuda.synchronize()
    wall_ms = (time.perf_counter() - t0) * 1e3 / steps
    event_ms = e0.elapsed_time(e1) / steps
    return wall_ms, event_ms


def median_spmm_ms(sptir, torch, hyb, X, Y, steps):
    """Median over single steps, each bracketed by its own pair of events (no host synchronisation in between)."""
    events = [(torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)) for _ in range(steps)]
    for e0, e1 in events:
        e0.record()
        sptir.sptir_spmm(hyb, X, Y)
        e1.record()
    torch.cuda.synchronize()
    times = sorted(e0.elapsed_time(e1) for e0, e1 in events)
    return times[len(times) // 2]


def kernel_times(sptir, torch, hyb, X, Y, reps):
    """Mean time of each group of launches of sptir_spmm_timed (HIP events on the launch stream, recorded by the
    library between its launches) and the launch counts.  It launches chunk lists and heavy lists apart; in sptir_spmm, and so in the
    timed steps, heavy lists may share the last launch of the chunk lists."""
    acc = None
    for _ in range(reps):
        t = sptir.sptir_spmm_timed(hyb, X, Y)
        if acc is None:
            acc = dict(t)
        else:
            for k in ("ms_lists", "ms_heavy", "ms_reduce"):
                acc[k] += t[k]
    for k in ("ms_lists", "ms_heavy", "ms_reduce"):
        acc[k] /= reps
    return acc


def time_graph_replay(sptir, torch, hyb, X, Y, calls_per_graph, replays):
    """sptir_spmm only enqueues kernels, so a stream capture records it: per-call time of replaying a graph of
    `calls_per_graph` calls (what a launch-bound small graph costs without the per-launch host work)."""
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            for _ in range(calls_per_graph):
                sptir.sptir_spmm(hyb, X, Y, stream=side)
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    for _ in range(replays):
        graph.replay()
    torch.cuda.synchronize()
    return (time.perf_counter() - t0) * 1e3 / (replays * calls_per_graph)


def time_cold(sptir, torch, hyb, X, Y, reps, scratch):
    """Per-step time with the caches flushed before every step (outside the timed region)."""
    times = []
    for _ in range(reps):
        scratch.add_(1.0)            # 1 GiB read + write: evicts L2 and the 256 MB Infinity Cache
        e0 = torch.cuda.Event(enable_timing=True)
        e1 = torch.cuda.Event(enable_timing=True)
        e0.record()
        sptir.sptir_spmm(hyb, X, Y)
        e1.record()
        torch.cuda.synchronize()
        times.append(e0.elapsed_time(e1))
    times.sort()
    return times[len(times) // 2]


def upload(torch, w):
    dev = torch.device("cuda:0")
    return (torch.from_numpy(w.indptr).to(dev), torch.from_numpy(w.indices).to(dev),
            torch.from_numpy(w.values).to(dev))


def read_traffic(key, fingerprint):
    """Bytes that crossed the L2 boundary per launch of the dominant kernel, from the committed rocprofv3 counter
    summary.  Returns (bytes or None, note): the figure only counts if the summary was taken on these sources."""
    path = os.path.join(ROOT, "profiles", "hbm_traffic.txt")
    if not os.path.exists(path):
        return None, "no profiles/hbm_traffic.txt"
    stamp, value = None, None
    for line in open(path):
        parts = line.split()
        if len(parts) >= 2 and parts[0] == "sources":
            stamp = parts[1]
        if len(parts) >= 2 and parts[0] == key:
            value = float(parts[1])
    if value is None:
        return None, "profiles/hbm_traffic.txt has no line for " + key
    if stamp != fingerprint:
        return None, f"profiles/hbm_traffic.txt was taken on sources {stamp}, this build is {fingerprint}: stale"
    return value, f"profiles/hbm_traffic.txt, sources {stamp}"


def gather_roof(sptir, torch, dev, quick=True):
    """Measured rate of random 128-byte row gathers (the access every stored non-zero costs) for working sets that
    sit in L1, in one XCD's L2 (the case of the SpMM kernels: a partition's slice of one feature tile), in the
    memory-side cache and in HBM, and over wavefronts per SIMD; of random rows out of LDS; plus the float32 FMA rate."""
    rows_max = 1 << (18 if quick else 21)
    X = torch.zeros(rows_max, 128, device=dev)
    sink = torch.zeros(16, device=dev)
    out = {"working_set_sweep": [], "occupancy_sweep": []}

    def run(n_rows, tiles, wgs, iters):
        ms, nbytes = sptir.sptir_roof_gather(X, n_rows, tiles, wgs, iters, sink)
        return nbytes / ms / 1e6

    sets = [(64, "L1: 8 KB per XCD and tile"), (1024, "0.13 MB"), (14561, "1.86 MB: one partition of the largest graph"),
            (32768, "4.2 MB"), (1 << 18, "33.5 MB: memory-side cache")]
    if not quick:
        sets.append((1 << 21, "268 MB per tile: HBM"))
    for n_rows, what in sets:
        gbs = run(n_rows, 4, 4096, 128)
        out["working_set_sweep"].append({"rows": n_rows, "bytes_per_xcd": n_rows * 128, "what": what,
                                         "gbs": round(gbs, 1)})
    for wgs in (256, 512, 768, 1024, 2048, 4096):
        out["occupancy_sweep"].append({"workgroups": wgs, "wavefronts_per_simd": wgs * 4 / 1024.0,
                                       "gbs_at_1.86MB": round(run(14561, 4, wgs, 512), 1)})
    out["l2_resident_gbs"] = max(p["gbs_at_1.86MB"] for p in out["occupancy_sweep"])
    out["theory_gbs"] = GATHER_THEORY_GBS
    # rows out of LDS, the case of the column slices: 64-byte rows are what k_spmm_slices reads, 512-byte rows a stride of
    # 160 floats apart what k_sddmm_slices does at 128 features
    out["lds_sweep"] = []
    for row_floats, stride in ((16, 16), (128, 160)) if quick else ((4, 4), (8, 8), (16, 16), (16, 20), (32, 32), (128, 128), (128, 160)):
        ms, nbytes = sptir.sptir_roof_lds_gather(row_floats, stride, 256, 1024 if row_floats == 128 else 4096, sink)
        out["lds_sweep"].append({"row_bytes": 4 * row_floats, "stride_bytes": 4 * stride, "gbs": round(nbytes / ms / 1e6, 1)})
    out["lds_64_byte_rows_gbs"] = next(p["gbs"] for p in out["lds_sweep"] if (p["row_bytes"], p["stride_bytes"]) == (64, 64))
    ms, flops = sptir.sptir_roof_fma(8192, 4096, sink)
    out["fma_tflops"] = round(flops / ms / 1e9, 2)
    return out


def cpu_baseline(oracle, np, w, X_host, feat, budget_s=10.0):
    """The fp64 oracle, untuned, on a bounded sample of rows of the same workload: all host threads, then one."""
    rng = np.random.default_rng(1)
    rows = rng.permutation(w.n_rows).astype(np.int32)
    deg = np.diff(w.indptr)
    probe = rows[:2000]
    t0 = time.perf_counter()
    oracle.spmm_csr_rows(probe, w.indptr, w.indices, w.values, X_host)
    dt = max(time.perf_counter() - t0, 1e-4)
    rate = deg[probe].sum() / dt                       # non-zeros per second
    want_nnz = rate * budget_s
    csum = np.cumsum(deg[rows])
    n_sel = int(min(w.n_rows, max(2000, np.searchsorted(csum, want_nnz))))
    sel = rows[:n_sel]
    t0 = time.perf_counter()
    Yr, Sr = oracle.spmm_csr_rows(sel, w.indptr, w.indices, w.values, X_host)
    dt = time.perf_counter() - t0
    nnz_sel = int(deg[sel].sum())
    threads = oracle.num_threads()
    base = dict(value=2.0 * nnz_sel * feat / dt / 1e9, unit="GFLOP/s", cores=threads, kind="oracle",
                sample=f"{n_sel} random rows ({nnz_sel} non-zeros) of the same graph and X, feat={feat}, "
                       f"{dt:.1f} s, fp64, OpenMP over rows")
    # one thread, on a sample a thread's worth as large (the OpenMP runtime the oracle links is told so; the
    # oracle itself is untouched)
    try:
        gomp = ctypes.CDLL("libgomp.so.1")
        gomp.omp_set_num_threads(1)
        one = rows[:max(500, n_sel // max(threads, 1))]
        t0 = time.perf_counter()
        oracle.spmm_csr_rows(one, w.indptr, w.indices, w.values, X_host)
        dt1 = time.perf_counter() - t0
        gomp.omp_set_num_threads(threads)
        base["one_thread_gflops"] = round(2.0 * int(deg[one].sum()) * feat / dt1 / 1e9, 2)
        base["one_thread_sample"] = f"{one.size} of those rows, {dt1:.1f} s"
    except OSError:
        base["one_thread_gflops"] = None
    return base, sel, Yr, Sr


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--gpus", type=int, default=1)
    ap.add_argument("--steps", type=int, default=50)
    ap.add_argument("--warmup", type=int, default=10)
    ap.add_argument("--no-extras", action="store_true", help="only the headline workload (for profiling runs)")
    ap.add_argument("--no-cpu", action="store_true", help="skip the CPU oracle baseline")
    ap.add_argument("--copy-calibration", action="store_true",
                    help="also run one plain 1 GiB device copy (known HBM bytes) to scale profiler byte counters")
    ap.add_argument("--gather-roof", action="store_true",
                    help="only the gather / FMA roof microbenchmarks (full sweep), one JSON line")
    ap.add_argument("--workload", default="social", help="headline workload for profiling runs (default: social)")
    args = ap.parse_args()
    if args.gpus != 1:
        print("bench.py: this build measures one GPU only (every box has one); run with --gpus 1", file=sys.stderr)
        sys.exit(2)

    import numpy as np
    import torch

    import paper_2207_04606_amd as sptir
    import workloads

    if not torch.cuda.is_available():
        print("bench.py: no GPU visible", file=sys.stderr)
        sys.exit(1)
    sptir.load_library()   # no fallback: raises if the HIP library is not built
    dev = torch.device("cuda:0")

    if args.gather_roof:
        print(json.dumps({"gather_roof": gather_roof(sptir, torch, dev, quick=False)}))
        return

    if args.copy_calibration:
        src = torch.ones(256 * 1024 * 1024, device=dev)   # 1 GiB written by the fill kernel
        dst = torch.empty_like(src)
        torch.add(src, 1.0, out=dst)                      # 1 GiB read + 1 GiB written by one elementwise kernel
        torch.cuda.synchronize()
        del src, dst

    # ---------------------------------------------------------------- headline
    w = workloads.make_config(args.workload)
    indptr, indices, values = upload(torch, w)
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    hyb = sptir.sptir_hyb_build(w.n_rows, w.n_cols, indptr, indices, values, w.n_col_parts, w.max_bucket_log2)
    torch.cuda.synchronize()
    build_first_ms = (time.perf_counter() - t0) * 1e3
    build_times = []
    for _ in range(3):
        t0 = time.perf_counter()
        hyb2 = sptir.sptir_hyb_build(w.n_rows, w.n_cols, indptr, indices, values, w.n_col_parts, w.max_bucket_log2)
        torch.cuda.synchronize()
        build_times.append((time.perf_counter() - t0) * 1e3)
        hyb2.destroy()
    build_ms = sorted(build_times)[1]
    # the same with the library's device memory coming from torch's caching allocator (sptir_set_allocator); the default
    # allocator keeps the blocks of released handles and temporaries itself, none larger than 1 GB
    sptir.sptir_set_allocator(True)
    try:
        cached_times = []
        for _ in range(4):
            t0 = time.perf_counter()
            hyb2 = sptir.sptir_hyb_build(w.n_rows, w.n_cols, indptr, indices, values, w.n_col_parts, w.max_bucket_log2)
            torch.cuda.synchronize()
            cached_times.append((time.perf_counter() - t0) * 1e3)
            hyb2.destroy()
    finally:
        sptir.sptir_set_allocator(False)
    build_cached_ms = sorted(cached_times[1:])[1]
    info = sptir.sptir_hyb_info(hyb)
    n_long = int(sptir.sptir_hyb_array(hyb, "plan_long_rows").size)   # rows summed from column slices in LDS

    results = {}
    X_host_128 = None
    for feat in (128, 256):
        if feat == 256 and (args.no_extras or args.workload != "social"):
            continue
        if feat == w.feat:
            Xh = w.X
        else:
            Xh = np.random.Generator(np.random.PCG64(7)).standard_normal((w.n_cols, feat), dtype=np.float32)
        if feat == 128:
            X_host_128 = Xh
        X = torch.from_numpy(Xh).to(dev)
        Y = torch.empty(w.n_rows, feat, device=dev)
        wall_ms, event_ms = time_spmm(sptir, torch, hyb, X, Y, args.steps, args.warmup)
        flops = 2.0 * w.nnz * feat
        bmin = bytes_min(w.nnz, w.n_rows, w.n_cols, feat)
        results[feat] = dict(wall_ms=wall_ms, event_ms=event_ms, gflops=flops / wall_ms / 1e6,
                             median_ms=median_spmm_ms(sptir, torch, hyb, X, Y, args.steps),
                             bmin_gbs=bmin / event_ms / 1e6, bmin=bmin,
                             # one row of X (feat * 4 bytes) is gathered per non-zero; bucket pads are not walked
                             gather_gbs=w.nnz * feat * 4.0 / event_ms / 1e6,
                             kernels=kernel_times(sptir, torch, hyb, X, Y, 5) if feat == 128 else None,
                             Y=Y if feat == 128 else None)
        if feat == 256:
            del X, Y
    head = results[128]

    out = {
        "metric": "SpMM GFLOP/s and achieved HBM GB/s (% of peak) at feat=128, 1 MI355X",
        "value": round(head["gflops"], 1), "unit": "GFLOP/s", "n_gpus": 1, "steps": args.steps, "warmup": args.warmup,
        "ms_per_step": round(head["wall_ms"], 4), "median_ms_per_step": round(head["median_ms"], 4),
        "higher_is_better": True, "scaling": "weak", "vs_baseline": None,
        "dtype": "f32", "data": "synthetic",
        "config": {"workload": "largest graph of the set (social-like: 232,965 rows, %d non-zeros, power-law "
                               "degrees, values 1/deg) decomposed as hyb(c=16, k=11), X 232,965 x 128 fp32 N(0,1); "
                               "Y = A X per step" % w.nnz if args.workload == "social" else args.workload,
                   "n_rows": w.n_rows, "nnz": w.nnz, "feat": 128, "n_col_parts": w.n_col_parts,
                   "max_bucket_log2": w.max_bucket_log2, "stored_slots": info["n_ell_slots"] + info["n_rem_nnz"],
                   "pad_slots": info["n_pad_slots"],
                   "walked_slots": (info["n_work_items"] + info["n_heavy_items"]) * info["item_slots"],
                   "rounds": info["rounds"], "row_block": info["row_block"], "heavy_len": info["heavy_len"],
                   "heavy_pieces": info["n_heavy_pieces"], "heavy_nnz": info["n_heavy_nnz"],
                   "values_per_row": info["values_per_row"]},
        "hbm_gbs_min_model": round(head["bmin_gbs"], 1),
        "hbm_gbs_hyb_model": round(bytes_hyb(info, w.n_rows, w.n_cols, 128) / head["event_ms"] / 1e6, 1),
        "hbm_pct_of_peak": round(100.0 * head["bmin_gbs"] / HBM_PEAK_GBS, 2),
        "target_note": "the 60 %-of-HBM target under the minimal byte model is missed: the path is a cache-served "
                       "gather (one 128-byte row of X per non-zero and feature tile through the vector-memory path), "
                       "see roofline.binding_roof",
        "hyb_build_ms": round(build_ms, 3), "hyb_build_first_call_ms": round(build_first_ms, 3),
        "hyb_build_caching_allocator_ms": round(build_cached_ms, 3),
        "hyb_build": {"ms": round(build_ms, 3), "ms_caching_allocator": round(build_cached_ms, 3),
                      "host_synchronisations": 4 if n_long else 3, "algorithmic_bytes": bytes_build(info, w.nnz, w.n_rows),
                      "gbs": round(bytes_build(info, w.nnz, w.n_rows) / build_ms / 1e6, 1),
                      "frac_of_hbm_peak": round(bytes_build(info, w.nnz, w.n_rows) / build_ms / 1e6 / HBM_PEAK_GBS, 4),
                      "device_bytes": info["device_bytes"]},
    }

    # ------------------------------------------------------------- roofline
    # The dominant kernel is whichever group of launches takes longer inside a timed call (see kernel_times); its launches are
    # timed live by HIP events the library records on the launch stream between its launches.
    kt = head["kernels"]
    fingerprint = source_fingerprint()
    feat = 128
    from_lds = n_long > 0 and kt["ms_heavy"] >= kt["ms_lists"]
    if kt["ms_heavy"] >= kt["ms_lists"]:
        # (rows in column slices: k_spmm_slices, and k_spmm_heavy for the few pieces left)
        kernel = "k_spmm_heavy<4, 8, true, false, %s>" % ("true" if info["values_per_row"] else "false")
        if n_long:
            kernel = "k_spmm_slices<%s> + %s" % ("true" if info["values_per_row"] else "false", kernel)
        n_launch, ms = kt["n_heavy_launches"], kt["ms_heavy"]
        # its share of the minimal byte model: the heavy pieces' entries once, X once, its partial sums written
        alg_bytes = (8.0 * info["n_heavy_nnz"] + 4.0 * w.n_cols * feat +
                     4.0 * feat * (info["n_heavy_pieces"] + info["n_heavy_lists"]))
        gathered = info["n_heavy_nnz"] * feat * 4.0
        key = args.workload + ("_feat128_k_spmm_slices_and_heavy" if n_long else "_feat128_k_spmm_heavy")
    else:
        kernel, n_launch, ms = "k_spmm_hyb<4, 8, true, false, %s>" % ("true" if info["values_per_row"] else "false"), \
            kt["n_list_launches"], kt["ms_lists"]
        light_nnz = w.nnz - info["n_heavy_nnz"]
        x_reads = kt["n_list_launches"] if info["rounds"] else 1     # every round sweeps all of X
        alg_bytes = 8.0 * light_nnz + 4.0 * w.n_cols * feat * x_reads + 4.0 * w.n_rows * feat
        gathered = light_nnz * feat * 4.0
        key = args.workload + "_feat128_k_spmm_hyb"
    per_launch_ms = ms / max(n_launch, 1)
    traffic, traffic_note = read_traffic(key, fingerprint)
    out["roofline"] = {
        "bound": "hbm", "achieved": round(alg_bytes / ms / 1e6, 1), "peak": HBM_PEAK_GBS,
        "unit": "GB/s", "frac": round(alg_bytes / ms / 1e6 / HBM_PEAK_GBS, 4),
        "traffic": traffic, "traffic_source": traffic_note,
        "kernel": kernel, "launches_per_timed_call": n_launch,
        "avg_launch_ms": round(per_launch_ms, 4), "algorithmic_bytes_per_launch": alg_bytes / max(n_launch, 1),
        "kernel_ms_per_timed_call": {"k_spmm_hyb": round(kt["ms_lists"], 4), "k_spmm_heavy": round(kt["ms_heavy"], 4),
                                     "k_heavy_reduce": round(kt["ms_reduce"], 4), "rows_in_column_slices": n_long,
                                     "launches": [kt["n_list_launches"], kt["n_heavy_launches"], kt["n_reduce_launches"]],
                                     "note": "chunk lists and heavy lists launched apart; in a step they may share a launch"},
        "whole_call": {"achieved": round(head["bmin_gbs"], 1), "frac": round(head["bmin_gbs"] / HBM_PEAK_GBS, 4),
                       "algorithmic_bytes": head["bmin"]},
        "sources": fingerprint,
    }
    # the path is a cache-served gather, not an HBM stream: each non-zero pulls feat*4 bytes of X through the
    # vector-memory return path or out of LDS.  Both roofs are measured here, on this GPU, by the library's microbenchmarks.
    roof = gather_roof(sptir, torch, dev, quick=True)
    binding_gbs = roof["lds_64_byte_rows_gbs"] if from_lds else roof["l2_resident_gbs"]
    out["roofline"]["binding_roof"] = {
        "name": "gather of 64-byte rows of X out of a CU's LDS" if from_lds else
                "vector-memory gather of 128-byte rows of X out of an XCD's L2",
        "roof_gbs": binding_gbs,
        "kernel_gathered_gbs": round(gathered / ms / 1e6, 1),
        "measured_l2_resident_gbs": roof["l2_resident_gbs"], "theory_gbs": GATHER_THEORY_GBS,
        "frac_of_measured": round(gathered / ms / 1e6 / binding_gbs, 4),
        "frac_of_theory": round(gathered / ms / 1e6 / GATHER_THEORY_GBS, 4),
        "whole_call_gathered_gbs": round(head["gather_gbs"], 1),
        "whole_call_frac_of_measured": round(head["gather_gbs"] / roof["l2_resident_gbs"], 4),
        "fma_tflops_measured": roof["fma_tflops"], "fma_tflops_peak": FMA_PEAK_TFLOPS,
        "fma_frac": round(2.0 * w.nnz * feat / head["event_ms"] / 1e9 / FMA_PEAK_TFLOPS, 4),
    }
    out["gather_roof"] = roof
    if traffic:
        # bytes that crossed the L2 boundary per second during the dominant kernel
        out["hbm_gbs_measured"] = round(traffic / per_launch_ms / 1e6, 1)
    else:
        out["hbm_gbs_measured"] = None

    # ------------------------------------------------- CPU oracle beside it
    if not args.no_cpu:
        import oracle
        base, sel, Yr, Sr = cpu_baseline(oracle, np, w, X_host_128, 128)
        out["cpu_baseline"] = base
        Yg = head["Y"][torch.from_numpy(sel.astype(np.int64)).to(dev)].cpu().numpy().astype(np.float64)
        nz = Sr > 0
        out["max_normalised_error_vs_oracle"] = float((np.abs(Yg - Yr)[nz] / Sr[nz]).max())
    head["Y"] = None

    if not args.no_extras and args.workload == "social":
        r256 = results[256]
        out["as_written_feat256"] = {"gflops": round(r256["gflops"], 1), "ms_per_step": round(r256["wall_ms"], 4),
                                     "median_ms_per_step": round(r256["median_ms"], 4),
                                     "hbm_gbs_min_model": round(r256["bmin_gbs"], 1),
                                     "gather_gbs": round(r256["gather_gbs"], 1)}
        scratch = torch.zeros(256 * 1024 * 1024, device=dev)
        X = torch.from_numpy(X_host_128).to(dev)
        Y = torch.empty(w.n_rows, 128, device=dev)
        out["cold_ms_per_step"] = round(time_cold(sptir, torch, hyb, X, Y, 10, scratch), 4)
        # the same matrix with a value stored per entry, and with a launch per partition instead of rounds
        for name, opts in (("values_kept", {"keep_values": 1}), ("launch_per_partition", {"rounds": 2})):
            hv = sptir.sptir_hyb_build_ex(w.n_rows, w.n_cols, indptr, indices, values, w.n_col_parts,
                                          w.max_bucket_log2, opts)
            vw, _ = time_spmm(sptir, torch, hv, X, Y, 20, 3)
            out[name] = {"ms_per_step": round(vw, 4), "gflops": round(2.0 * w.nnz * 128 / vw / 1e6, 1)}
            hv.destroy()
        # the single-pass CSR kernel ("no-hyb") on the same graph and X, for the comparison section 4.2.1 makes
        for _ in range(3):
            sptir.sptir_spmm_csr(w.n_rows, w.n_cols, indptr, indices, values, X, Y)
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        for _ in range(10):
            sptir.sptir_spmm_csr(w.n_rows, w.n_cols, indptr, indices, values, X, Y)
        torch.cuda.synchronize()
        csr_ms = (time.perf_counter() - t0) * 1e3 / 10
        out["no_hyb_csr"] = {"ms_per_step": round(csr_ms, 4), "gflops": round(2.0 * w.nnz * 128 / csr_ms / 1e6, 1),
                             "hyb_speedup": round(csr_ms / head["wall_ms"], 3)}
        # the format search of section 4.2.1 (build every candidate c, time it, keep the fastest) over a few
        # partition counts around the configured one; the headline above stays at the configured c
        cands = [8, 12, 16, 24]
        t0 = time.perf_counter()
        best, best_c, cand_ms = sptir.sptir_hyb_search(w.n_rows, w.n_cols, indptr, indices, values, 128, cands,
                                                       w.max_bucket_log2, reps=5)
        torch.cuda.synchronize()
        search_ms = (time.perf_counter() - t0) * 1e3
        best_wall_ms, _ = time_spmm(sptir, torch, best, X, Y, 20, 3)
        best.destroy()
        out["format_search"] = {"candidates": cands, "ms_per_candidate": [round(m, 4) for m in cand_ms],
                                "best_c": best_c, "best_ms_per_step": round(best_wall_ms, 4),
                                "best_gflops": round(2.0 * w.nnz * 128 / best_wall_ms / 1e6, 1),
                                "search_ms": round(search_ms, 1)}
        # SDDMM on the same graph (B_ij = A_ij <X_i, Yt_j>), entries in CSR order and in column-partition order
        Xl = torch.randn(w.n_rows, 128, device=dev, generator=torch.Generator(device=dev).manual_seed(3))
        Bv = torch.empty(w.nnz, device=dev)

        def timed(fn, reps=10):
            for _ in range(3):
                fn()
            torch.cuda.synchronize()
            t0 = time.perf_counter()
            for _ in range(reps):
                fn()
            torch.cuda.synchronize()
            return (time.perf_counter() - t0) * 1e3 / reps

        sddmm_csr_ms = timed(lambda: sptir.sptir_sddmm_csr(w.n_rows, w.n_cols, indptr, indices, values, Xl, X, Bv))
        t0 = time.perf_counter()
        plan = sptir.sptir_sddmm_plan_build(w.n_rows, w.n_cols, indptr, indices, 0, 128)
        torch.cuda.synchronize()
        plan_ms = (time.perf_counter() - t0) * 1e3
        sddmm_ms = timed(lambda: sptir.sptir_sddmm(plan, values, Xl, X, Bv))
        pinfo = sptir.sptir_sddmm_plan_info(plan)
        plan.destroy()
        out["sddmm_feat128"] = {"ms_per_step": round(sddmm_ms, 4), "gflops": round(2.0 * w.nnz * 128 / sddmm_ms / 1e6, 1),
                                "n_col_parts": pinfo["n_col_parts"], "plan_build_ms": round(plan_ms, 3),
                                "gather_gbs": round(w.nnz * 512.0 / sddmm_ms / 1e6, 1),
                                "csr_order_ms_per_step": round(sddmm_csr_ms, 4)}
        del Xl, Bv
        # relational gather-matmul-scatter on two synthetic heterogeneous graphs (feature size 32)
        out["rgms_feat32"] = []
        for hname in ("hetero_d", "hetero_e"):
            hw = workloads.make_hetero(hname)
            hip_, hix, hva = (torch.from_numpy(a).to(dev) for a in (hw.indptr, hw.indices, hw.values))
            t0 = time.perf_counter()
            rg = sptir.sptir_rgms_build(hw.n_rel, hw.n, hw.n, hip_, hix, hva)
            torch.cuda.synchronize()
            rg_build_ms = (time.perf_counter() - t0) * 1e3
            rinfo = sptir.sptir_rgms_info(rg)
            hX, hW = torch.from_numpy(hw.X).to(dev), torch.from_numpy(hw.W).to(dev)
            hY = torch.empty(hw.n, 32, device=dev)
            rg_ms = timed(lambda: sptir.sptir_rgms(rg, hX, hW, hY), reps=20)
            pairs = rinfo["n_stacked_rows_stored"]
            # algorithmic bytes: a 128-byte row of X in and 8 bytes of column and value per non-zero, Y and W once
            rg_bytes = 136.0 * hw.nnz + 128.0 * hw.n + 4.0 * hw.W.size
            out["rgms_feat32"].append({
                "workload": "%s: %d nodes, %d relations, %d non-zeros, d_in = d_out = 32" % (hname, hw.n, hw.n_rel, hw.nnz),
                "ms_per_step": round(rg_ms, 4), "build_ms": round(rg_build_ms, 3),
                "gflops": round((2.0 * hw.nnz * 32 + 2.0 * pairs * 32 * 32) / rg_ms / 1e6, 1),
                "gather_gbs": round(hw.nnz * 128.0 / rg_ms / 1e6, 1), "tiles": rinfo["n_tiles"],
                "entries_per_tile": round(hw.nnz / max(rinfo["n_tiles"], 1), 2),
                "roofline": {"bound": "hbm", "achieved": round(rg_bytes / rg_ms / 1e6, 1), "peak": HBM_PEAK_GBS,
                             "unit": "GB/s", "frac": round(rg_bytes / rg_ms / 1e6 / HBM_PEAK_GBS, 4),
                             "algorithmic_bytes": rg_bytes}})
            rg.destroy()
            del hX, hW, hY, hip_, hix, hva
        del X, Y
        hyb.destroy()
        del indptr, indices, values
        others = []
        for name in ("tiny", "small", "medium", "protein"):
            wc = workloads.make_config(name)
            ip, ix, va = upload(torch, wc)
            sptir.sptir_hyb_build(wc.n_rows, wc.n_cols, ip, ix, va, wc.n_col_parts, wc.max_bucket_log2).destroy()
            torch.cuda.synchronize()
            t0 = time.perf_counter()
            hc = sptir.sptir_hyb_build(wc.n_rows, wc.n_cols, ip, ix, va, wc.n_col_parts, wc.max_bucket_log2)
            torch.cuda.synchronize()
            b_ms = (time.perf_counter() - t0) * 1e3
            ci = sptir.sptir_hyb_info(hc)
            X = torch.from_numpy(wc.X).to(dev)
            Y = torch.empty(wc.n_rows, wc.feat, device=dev)
            wall_ms, event_ms = time_spmm(sptir, torch, hc, X, Y, 100, 10)
            cold = time_cold(sptir, torch, hc, X, Y, 10, scratch)
            bm = bytes_min(wc.nnz, wc.n_rows, wc.n_cols, wc.feat)
            others.append({"config": name, "nnz": wc.nnz, "feat": wc.feat,
                           "gflops": round(2.0 * wc.nnz * wc.feat / wall_ms / 1e6, 1),
                           "ms_per_step": round(wall_ms, 4),
                           "median_ms_per_step": round(median_spmm_ms(sptir, torch, hc, X, Y, 50), 4),
                           "graph_replay_ms_per_step": round(time_graph_replay(sptir, torch, hc, X, Y, 10, 20), 4),
                           "cold_ms_per_step": round(cold, 4),
                           "hbm_gbs_min_model_cold": round(bm / cold / 1e6, 1),
                           "hbm_frac_cold": round(bm / cold / 1e6 / HBM_PEAK_GBS, 4),
                           "rounds": ci["rounds"], "launches": ci["n_phases"], "heavy_pieces": ci["n_heavy_pieces"],
                           "hyb_build_ms": round(b_ms, 3)})
            hc.destroy()
        out["other_configs"] = others
    print(json.dumps(out))


if __name__ == "__main__":
    main()
