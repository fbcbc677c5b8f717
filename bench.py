#!/usr/bin/env python3
"""Benchmark of the LoSA hot path on one MI355X.

One step = one layer's whole LoSA cycle on the Wan2.1-1.3B-shaped workload
(B=1, H=12, d=128, N=32,760 padded to 32,768, block 128, tau=0.99, bf16):
  losa_construct (the dense construction step: its attention output and the
     exact block masses)
  -> losa_select_blocks (shortest prefix reaching tau, CSR)
  -> 49 x losa_sparse_attn_fwd over the frozen support, each on that reuse
     step's drifted Q/K/V.
After the timed steps (untimed for the step clock): standalone calibration
and dense-attention times for comparison, and the recall of the frozen
support at later steps (Eq. (2)) next to the fixed-ratio top-k rule at the
same coverage.
All inputs (the calibration step and every drifted reuse step) are generated
on the device before the timed region.  HIP events on the stream the library
launches on time each call; the wall clock brackets the K timed steps.

The reported value is the metric's ms per layer of the block-sparse attention
forward (mean over every timed reuse call).  Printed as one JSON line.

    python bench.py [--gpus 1] [--steps K] [--warmup W] [--workload wan]
"""
from __future__ import annotations

import argparse
import hashlib
import json
import math
import os
import sys
import time

ROOT = os.path.dirname(os.path.abspath(__file__))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

MFMA_BF16_PEAK_TFLOPS = 2500.0      # MI355X dense bf16 matrix-core peak
# fp32 inputs run on the vector ALUs (fp32 fma per thread, no matrix cores):
# 256 CUs x 2.4 GHz x 256 FLOP/clk (128 fp32 lanes per CU, fma = 2 FLOP,
# counting the packed two-wide fma; plain fma issue reaches half of it)
FP32_VECTOR_PEAK_TFLOPS = 157.3
HBM_PEAK_GBS = 8000.0
TRAFFIC_FILE = os.path.join(ROOT, "profiles", "sparse_fwd_traffic.json")
CSRC = os.path.join(ROOT, "paper_2608_12032_amd", "csrc")


def parse():
    ap = argparse.ArgumentParser()
    ap.add_argument("--gpus", type=int, default=1)
    ap.add_argument("--steps", type=int, default=3)
    ap.add_argument("--warmup", type=int, default=1)
    ap.add_argument("--workload", default="wan", choices=["wan", "cog", "hunyuan", "tiny"])
    ap.add_argument("--reuse", type=int, default=None, help="override the reuse-step count")
    ap.add_argument("--tau", type=float, default=None)
    ap.add_argument("--block-k", type=int, default=0,
                    help="key block size when it differs from the query block (32: the "
                         "paper's rectangular 128 x 32 setting)")
    ap.add_argument("--cpu-seconds", type=float, default=12.0,
                    help="budget of the CPU-oracle baseline sample")
    ap.add_argument("--no-cpu-baseline", action="store_true")
    ap.add_argument("--sweep", action="store_true",
                    help="time the density sweep (Wan shape, tau x locality weight) instead of "
                         "the default step; prints one JSON line with every point")
    ap.add_argument("--no-cold", action="store_true",
                    help="skip the cold-cache forward timings (512 MiB write before each call)")
    ap.add_argument("--no-clock-context", action="store_true",
                    help="skip the shader-clock samples and the bf16 GEMM reference")
    ap.add_argument("--no-dense-compare", action="store_true",
                    help="skip the untimed dense-attention comparison, which runs the sparse "
                         "kernel over a full support (for profiles of the sparse launches alone)")
    ap.add_argument("--copy-reference-mib", type=int, default=0,
                    help="first run one plain device-to-device copy of this many MiB, a "
                         "reference of known size for hardware byte counters")
    ap.add_argument("--record-traffic", nargs=2, metavar=("FETCH_CSV", "WRITE_CSV"),
                    help="(no GPU) read the counter_collection.csv files of a rocprofv3 "
                         "--pmc FETCH_SIZE run and a --pmc WRITE_SIZE run of this script "
                         "(with --copy-reference-mib) and record HBM bytes per launch in "
                         + os.path.relpath(TRAFFIC_FILE, ROOT))
    return ap.parse_args()


def _code_only(text: str) -> str:
    """C/C++ source with comments removed and whitespace collapsed, so that a
    comment edit does not count as a kernel change."""
    import re
    out, i, n = [], 0, len(text)
    while i < n:
        c = text[i]
        if c in "\"'":  # string or character literal, copied whole
            j = i + 1
            while j < n and text[j] != c:
                j += 2 if text[j] == "\\" else 1
            out.append(text[i:j + 1])
            i = j + 1
        elif text.startswith("//", i):
            i = text.find("\n", i)
            i = n if i < 0 else i
        elif text.startswith("/*", i):
            i = text.find("*/", i + 2)
            i = n if i < 0 else i + 2
        else:
            out.append(c)
            i += 1
    return re.sub(r"\s+", " ", "".join(out)).strip()


# the sources of the bf16 kernels that the traffic record covers, their shared
# headers and the C ABI that launches them (the fp32 path and the recall
# kernels are not in the record)
TRAFFIC_SOURCES = ("abi.cpp", "attn_bf16.hpp", "calib.hip", "common.hpp", "launch.hpp",
                   "select.hip", "sparse_fwd.hip")


def source_hash() -> str:
    """Hash of the code (comments and whitespace aside) of the sources behind
    the kernels whose traffic is recorded."""
    h = hashlib.sha256()
    for name in TRAFFIC_SOURCES:
        with open(os.path.join(CSRC, name), encoding="utf-8") as f:
            h.update(name.encode() + b"\0" + _code_only(f.read()).encode())
    return h.hexdigest()[:16]


def measured_traffic(workload: str):
    """Per-kernel HBM bytes per launch from the rocprofv3 counter runs recorded
    under profiles/, if they were taken on the current kernel sources."""
    try:
        rec = json.load(open(TRAFFIC_FILE))
    except (OSError, ValueError):
        return None
    if rec.get("workload") != workload or rec.get("source_sha256_16") != source_hash():
        return None
    return rec


# kernel-name substrings that identify each launch in a counter file.  The
# forward kernel's name comes mangled (its last template flag: Lb0E sparse,
# Lb1E dense); the calibration kernel's demangled (false: two sweeps, true:
# one sweep with block statistics).
KERNELS = {"sparse_fwd": ("sparse_fwd_bf16_kernel", "Lb0E"),
           "dense_fwd": ("sparse_fwd_bf16_kernel", "Lb1E"),
           "calibrate": ("calib_bf16_kernel", "true>"),
           "stat_mass": ("stat_mass_kernel",),
           "calibrate_two_sweep": ("calib_bf16_kernel", "false>"),
           "select_rows": ("select_rows_kernel",), "compact_rows": ("compact_rows_kernel",)}
COPY_KERNEL = "__amd_rocclr_copyBuffer"


def _counter_per_dispatch(path: str, counter: str):
    """{dispatch id: (kernel name, value in KiB)} of one rocprofv3 counter CSV."""
    import csv
    out = {}
    with open(path) as f:
        for r in csv.DictReader(f):
            if r["Counter_Name"] != counter:
                continue
            d = int(r["Dispatch_Id"])
            name, val = out.get(d, (r["Kernel_Name"], 0.0))
            out[d] = (name, val + float(r["Counter_Value"]))
    return out


def record_traffic(fetch_csv: str, write_csv: str, copy_mib: int, workload: str):
    """HBM bytes per launch from FETCH_SIZE / WRITE_SIZE, each scaled by what the
    same counter reads for the reference copy of copy_mib MiB (read and written
    once).  Written to TRAFFIC_FILE with the hash of the kernel source."""
    if copy_mib <= 0:
        sys.exit("--record-traffic needs the --copy-reference-mib the counter runs used")
    res = {"workload": workload, "source_sha256_16": source_hash(),
           "copy_reference_mib": copy_mib, "kernels": {}}
    for counter, path in (("FETCH_SIZE", fetch_csv), ("WRITE_SIZE", write_csv)):
        per = _counter_per_dispatch(path, counter)
        copies = [v for n, v in per.values() if n == COPY_KERNEL]
        if not copies:
            sys.exit(f"{path}: no {COPY_KERNEL} dispatch (run with --copy-reference-mib)")
        scale = copy_mib * 1024.0 / max(copies)   # known KiB / counted KiB
        res[counter.lower() + "_scale"] = round(scale, 4)
        for key, pats in KERNELS.items():
            vals = [v for n, v in per.values() if all(p in n for p in pats)]
            if vals:
                k = res["kernels"].setdefault(key, {"launches": len(vals)})
                k[counter.lower().replace("_size", "_bytes")] = int(sum(vals) / len(vals) * scale * 1024)
    fwd = res["kernels"].get("sparse_fwd", {})
    if "fetch_bytes" not in fwd or "write_bytes" not in fwd:
        sys.exit("no sparse forward dispatch in the counter files")
    res["bytes_per_launch"] = fwd["fetch_bytes"] + fwd["write_bytes"]
    os.makedirs(os.path.dirname(TRAFFIC_FILE), exist_ok=True)
    with open(TRAFFIC_FILE, "w") as f:
        json.dump(res, f, indent=1)
        f.write("\n")
    print(json.dumps(res))


def _host_info():
    model = None
    try:
        with open("/proc/cpuinfo") as f:
            for line in f:
                if line.startswith("model name"):
                    model = line.split(":", 1)[1].strip()
                    break
    except OSError:
        pass
    try:
        from threadpoolctl import threadpool_info
        threads = max([p.get("num_threads", 1) for p in threadpool_info()] or [1])
    except Exception:  # noqa: BLE001 - threadpoolctl missing: report the cpu count
        threads = os.cpu_count() or 1
    return {"nproc": os.cpu_count(), "cpu_model": model, "blas_threads": int(threads)}


def cpu_baseline(w, q, k, v, mass, rp, ci, budget_s: float):
    """Time the fp64 oracle on the host cores, per layer, for its three phases:
    calibration (Eq. (1)) and the sparse forward (Eq. (4)) on samples of query
    blocks / CSR rows scaled by the row count, selection (Eq. (3)) on every row.
    `value` is the sparse forward, the counterpart of the metric."""
    import numpy as np

    from oracle import losa_oracle as O
    host = _host_info()
    f64 = lambda x: x.float().cpu().numpy().astype(np.float64)  # noqa: E731
    qh, kh, vh = f64(q), f64(k), f64(v)
    rp_h = rp.cpu().numpy().astype(np.int64)
    ci_h = ci[:rp_h[-1]].cpu().numpy().astype(np.int64)
    rows = rp_h.size - 1
    order = np.random.default_rng(0).permutation(rows)

    def sampled(fn, budget):
        # rows in chunks, in a fixed random order, until the time budget is spent
        n, dt, chunk = 0, 0.0, 4
        while n < rows and dt < budget:
            part = order[n:n + chunk]
            t0 = time.perf_counter()
            fn(part)
            dt += time.perf_counter() - t0
            n += part.size
            chunk = min(2 * chunk, 64)
        return dt / n * rows * 1e3, n, dt

    fwd_ms, n_f, dt_f = sampled(lambda part: O.sparse_attention(
        qh, kh, vh, w.N, w.block, w.bk, w.scale, rp_h, ci_h, rows_subset=part), budget_s * 2 / 3)
    cal_ms, n_c, dt_c = sampled(lambda part: O.block_masses(
        qh, kh, w.N, w.block, w.bk, w.scale, rows_subset=part), budget_s / 3)
    mh = f64(mass)
    t0 = time.perf_counter()
    O.select_blocks(mh, w.N, w.block, w.bk, w.tau)
    sel_ms = (time.perf_counter() - t0) * 1e3
    return {"value": round(fwd_ms, 1), "unit": "ms/layer", "cores": host["blas_threads"],
            "kind": "oracle",
            "sample": f"fp64 oracle Eq.(4) on {n_f} of {rows} CSR rows (random, seed 0) of one "
                      f"reuse step, {dt_f:.1f} s, scaled by rows",
            "phases_ms_per_layer": {
                "calibrate": round(cal_ms, 1), "select": round(sel_ms, 1),
                "sparse_fwd": round(fwd_ms, 1)},
            "phase_samples": {"calibrate": f"Eq.(1) on {n_c} of {rows} query blocks, "
                                           f"{dt_c:.1f} s, scaled by rows",
                              "select": f"Eq.(3) on all {rows} rows"},
            "host": host}


def tiny_single_thread():
    """The oracle's three phases on the Tiny configuration (B=1, H=2, d=64, fp32,
    N=1,024, block 64, tau=0.99), whole, on one host thread: a second CPU figure
    that needs no sampling or scaling."""
    import numpy as np
    from threadpoolctl import threadpool_limits

    from oracle import losa_oracle as O
    from paper_2608_12032_amd import workload as W
    tw = W.WORKLOADS["tiny"]
    q, k, v = (x.cpu().numpy().astype(np.float64) for x in W.make_inputs(tw))
    with threadpool_limits(limits=1):
        t0 = time.perf_counter()
        mbar, _ = O.block_masses(q, k, tw.N, tw.block, tw.bk, tw.scale)
        t1 = time.perf_counter()
        rp, ci, _ = O.select_blocks(mbar, tw.N, tw.block, tw.bk, tw.tau)
        t2 = time.perf_counter()
        O.sparse_attention(q, k, v, tw.N, tw.block, tw.bk, tw.scale, rp, ci)
        t3 = time.perf_counter()
    return {"threads": 1, "workload": "tiny: B=1 H=2 d=64 f32 N=1024 block 64 tau=0.99",
            "ms": {"calibrate": round((t1 - t0) * 1e3, 2), "select": round((t2 - t1) * 1e3, 2),
                   "sparse_fwd": round((t3 - t2) * 1e3, 2)}}


def _sclk_sampler():
    """Background sampler of the GPU shader clock (rocm-smi --showclocks), in MHz."""
    import re
    import shutil
    import subprocess
    import threading
    exe = shutil.which("rocm-smi") or ("/opt/rocm/bin/rocm-smi"
                                       if os.path.exists("/opt/rocm/bin/rocm-smi") else None)
    state = {"phase": None, "stop": False, "samples": []}

    def loop():
        while not state["stop"]:
            try:
                out = subprocess.run([exe, "--showclocks"], capture_output=True, text=True,
                                     timeout=5).stdout
                m = re.search(r"sclk clock level:\s*\d+:\s*\((\d+)\s*Mhz\)", out, re.I)
                if m and state["phase"]:
                    state["samples"].append((state["phase"], int(m.group(1))))
            except Exception:  # noqa: BLE001 - a missing or failing tool only loses samples
                pass
            time.sleep(0.2)

    th = None
    if exe:
        th = threading.Thread(target=loop, daemon=True)
        th.start()
    return state, th


def clock_context(torch, run_fwd, fwd_flop):
    """Shader clock while the sparse forward runs back to back, and a hipBLASLt
    bf16 GEMM (8192^3) with its clock, for context on the MFMA fraction: under
    sustained load the chip runs below the 2.4 GHz behind the 2.5 PFLOP/s peak."""
    state, th = _sclk_sampler()
    if th is None:
        return None

    def loop(fn, flop, secs, phase):
        fn()
        torch.cuda.synchronize()
        state["phase"] = phase
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        n, t0 = 0, time.perf_counter()
        a.record()
        while time.perf_counter() - t0 < secs:
            for _ in range(4):
                fn()
            n += 4
            torch.cuda.synchronize()
        b.record()
        torch.cuda.synchronize()
        state["phase"] = None
        return flop / (a.elapsed_time(b) / n * 1e-3) / 1e12

    fwd_tf = loop(run_fwd, fwd_flop, 2.5, "fwd")
    x = torch.randn(8192, 8192, device="cuda", dtype=torch.bfloat16)
    y = torch.randn(8192, 8192, device="cuda", dtype=torch.bfloat16)
    gemm_tf = loop(lambda: torch.mm(x, y), 2.0 * 8192 ** 3, 2.5, "gemm")
    del x, y
    state["stop"] = True
    th.join(timeout=10)

    def med(phase):
        v = sorted(c for p, c in state["samples"] if p == phase)
        return v[len(v) // 2] if v else None

    f_fwd, f_gemm = med("fwd"), med("gemm")
    out = {"sclk_mhz_sparse_fwd": f_fwd, "sparse_fwd_tflops_back_to_back": round(fwd_tf, 1),
           "gemm_bf16_8192_tflops": round(gemm_tf, 1), "sclk_mhz_gemm": f_gemm,
           "samples": len(state["samples"])}
    if f_fwd:
        out["sparse_fwd_frac_of_peak_at_its_sclk"] = round(
            fwd_tf / (MFMA_BF16_PEAK_TFLOPS * f_fwd / 2400.0), 4)
    if f_gemm:
        out["gemm_frac_of_peak_at_its_sclk"] = round(
            gemm_tf / (MFMA_BF16_PEAK_TFLOPS * f_gemm / 2400.0), 4)
    return out


def run_sweep(args):
    """Density sweep at the Wan shape: for each locality weight alpha one set of
    inputs and one calibration, then per tau the selection and the sparse
    forward (median of `reps` HIP-event-timed calls after warm-up), its
    coverage, MFMA fraction and the speedup over the full support (tau = 1)."""
    import torch

    from paper_2608_12032_amd import losa as L
    from paper_2608_12032_amd import workload as W

    pts = W.sweep_points()
    if args.block_k:
        pts = [W.rectangular(p, args.block_k) for p in pts]
    reps = max(3, args.steps * 5)
    out = []
    for alpha in W.SWEEP_ALPHAS:
        group = [p for p in pts if p.alpha == alpha]
        w = group[0]
        N, C, Ck, d = w.N, w.block, w.bk, w.d
        q, k, v = W.make_inputs(w, device="cuda")
        mass, _ = L.losa_calibrate_mass(q, k, N, C, Ck, want_lse=False)
        o = torch.empty_like(q)
        ws = torch.empty(L.workspace_bytes(2, 1, w.B, w.H, N, d, C, Ck), dtype=torch.uint8,
                         device="cuda")
        times = {}
        for p in group:
            rp, ci = L.losa_select_blocks(mass, N, C, Ck, p.tau)
            nnz = L.nnz(rp)
            for _ in range(max(1, args.warmup)):
                L.losa_sparse_attn_fwd(q, k, v, N, C, Ck, rp, ci, out=o, workspace=ws)
            evs = []
            for _ in range(reps):
                a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
                a.record()
                L.losa_sparse_attn_fwd(q, k, v, N, C, Ck, rp, ci, out=o, workspace=ws)
                b.record()
                evs.append((a, b))
            torch.cuda.synchronize()
            ms = sorted(a.elapsed_time(b) for a, b in evs)[reps // 2]
            flop = 4.0 * C * Ck * d * nnz
            times[p.tau] = ms
            out.append({"alpha": alpha, "tau": p.tau, "coverage": round(nnz / (rp.numel() - 1)
                                                                         / w.n_kblocks, 4),
                        "fwd_ms_median": round(ms, 4),
                        "mfma_frac": round(flop / (ms * 1e-3) / 1e12 / MFMA_BF16_PEAK_TFLOPS, 4)})
        for e in out:
            if e["alpha"] == alpha:
                e["speedup_vs_tau1"] = round(times[1.0] / e["fwd_ms_median"], 3)
        del q, k, v, mass, o, ws
    w0 = pts[0]
    print(json.dumps({"sweep": f"{w0.name}: Wan shape B={w0.B} H={w0.H} d={w0.d} N={w0.N} "
                               + (f"block {w0.block}" if w0.bk == w0.block
                                  else f"blocks {w0.block}x{w0.bk}"),
                      "unit": "ms/layer", "reps": reps, "points": out}), flush=True)


def main():
    args = parse()
    if args.sweep:
        run_sweep(args)
        return
    if args.record_traffic:
        record_traffic(*args.record_traffic, args.copy_reference_mib, args.workload)
        return
    world = int(os.environ.get("WORLD_SIZE", "1"))
    if args.gpus != 1 or world != 1:
        print(json.dumps({"error": "bench.py measures one GPU only: the LoSA path is built and "
                          "timed on a single MI355X; it would shard by (batch, head) with no "
                          "exchange between GPUs, so no multi-GPU figure is produced",
                          "n_gpus": args.gpus}),
              flush=True)
        sys.exit(2)

    import torch

    from paper_2608_12032_amd import losa as L
    from paper_2608_12032_amd import workload as W

    assert torch.cuda.is_available(), "bench.py needs a GPU"
    torch.cuda.set_device(0)
    w = W.WORKLOADS[args.workload]
    if args.block_k:
        w = W.rectangular(w, args.block_k)
    tau = w.tau if args.tau is None else args.tau
    reuse = w.reuse if args.reuse is None else args.reuse
    N, C, Ck, d = w.N, w.block, w.bk, w.d
    n_q, n_k = w.n_blocks, w.n_kblocks
    rows = w.B * w.H * n_q

    # ---- inputs resident in HBM before timing --------------------------------
    state = W.make_state(w, device="cuda")
    q0, k0, v0 = W.cast(state, w)
    reuse_inputs = []
    for t in range(1, reuse + 1):
        W.drift_(state, w, t)
        reuse_inputs.append(W.cast(state, w))
    del state
    dev = q0.device
    mass = torch.empty((w.B, w.H, n_q, n_k), dtype=torch.float32, device=dev)
    out0 = torch.empty_like(q0)
    ws_con = torch.empty(max(L.workspace_bytes(4, 1 if w.dtype == "bf16" else 0, w.B, w.H, N, d,
                                               C, Ck), 16), dtype=torch.uint8, device=dev)
    row_ptr = torch.empty(rows + 1, dtype=torch.int32, device=dev)
    col_idx = torch.empty(rows * n_k, dtype=torch.int32, device=dev)
    ws_sel = torch.empty(max(L.workspace_bytes(1, 0, w.B, w.H, N, 1, C, Ck), 16),
                         dtype=torch.uint8, device=dev)
    ws_fwd = torch.empty(max(L.workspace_bytes(2, 1 if w.dtype == "bf16" else 0, w.B, w.H, N, d,
                                               C, Ck), 16), dtype=torch.uint8, device=dev)
    out = torch.empty_like(q0)
    if args.copy_reference_mib > 0:
        nbytes = args.copy_reference_mib << 20
        src = torch.ones(nbytes // 4, dtype=torch.float32, device=dev)
        dst = torch.empty_like(src)
        torch.cuda.synchronize()
        dst.copy_(src)
        torch.cuda.synchronize()
        del src, dst
    torch.cuda.synchronize()

    def step():
        ev = [torch.cuda.Event(enable_timing=True) for _ in range(3 + 2 * reuse)]
        ev[0].record()
        L.losa_construct(q0, k0, v0, N, C, Ck, out=out0, mass=mass, workspace=ws_con)
        ev[1].record()
        L.losa_select_blocks(mass, N, C, Ck, tau, row_ptr=row_ptr, col_idx=col_idx,
                             workspace=ws_sel)
        ev[2].record()
        for t, (q, k, v) in enumerate(reuse_inputs):
            ev[3 + 2 * t].record()
            L.losa_sparse_attn_fwd(q, k, v, N, C, Ck, row_ptr, col_idx, out=out, workspace=ws_fwd)
            ev[4 + 2 * t].record()
        return ev

    for _ in range(args.warmup):
        step()
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    events = [step() for _ in range(args.steps)]
    torch.cuda.synchronize()
    wall = time.perf_counter() - t0

    con_ms = [e[0].elapsed_time(e[1]) for e in events]
    sel_ms = [e[1].elapsed_time(e[2]) for e in events]
    fwd_ms = [e[3 + 2 * t].elapsed_time(e[4 + 2 * t]) for e in events for t in range(reuse)]
    nnz = L.nnz(row_ptr)
    fwd = sum(fwd_ms) / len(fwd_ms)
    fwd_sorted = sorted(fwd_ms)
    retained_flop = 4.0 * C * Ck * d * nnz
    dense_flop = 4.0 * w.B * w.H * N * N * d
    achieved = retained_flop / (fwd * 1e-3) / 1e12
    peak = MFMA_BF16_PEAK_TFLOPS if w.dtype == "bf16" else FP32_VECTOR_PEAK_TFLOPS
    wkey = args.workload + (f"-c{Ck}" if Ck != C else "")
    traffic = measured_traffic(wkey)
    n_pad = w.N_pad
    # algorithmic bytes per launch
    elt = 2 if w.dtype == "bf16" else 4
    qkv = w.B * w.H * n_pad * d * elt
    mass_b = w.B * w.H * n_q * n_k * 4
    stat_b = w.B * w.H * n_k * n_pad * 4   # one-sweep block statistics, fp32 per (query, key block)
    lse_b = w.B * w.H * n_pad * 4
    alg = {"sparse_fwd": 4 * qkv + 4 * (rows + 1 + nnz),
           # one sweep (the timed scheme): Q, K read; statistics and lse written
           # by the sweep and read back by the reduction; masses written
           "calibrate": 2 * qkv + 2 * stat_b + 2 * lse_b + mass_b,
           # two sweeps: Q, K read, masses written (the second sweep's re-reads
           # of K are not algorithmic)
           "calibrate_two_sweep": 2 * qkv + mass_b,
           "select": mass_b + 4 * (rows + 1 + nnz)}
    qk_flop = 2.0 * w.B * w.H * n_pad * n_pad * d   # one Q K^T over every (query, key) pair
    con_t = sum(con_ms) / len(con_ms)
    sel_t = sum(sel_ms) / len(sel_ms)

    # ---- untimed comparisons: calibration alone, dense attention alone ------
    def timed(fn, reps=5):
        fn()
        evs = []
        for _ in range(reps):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            fn()
            b.record()
            evs.append((a, b))
        torch.cuda.synchronize()
        return sum(a.elapsed_time(b) for a, b in evs) / reps

    mass_cal = torch.empty_like(mass)
    ws_cal = torch.empty(max(L.workspace_bytes(0, 1 if w.dtype == "bf16" else 0, w.B, w.H, N, d,
                                               C, Ck), 16), dtype=torch.uint8, device=dev)
    cal_t = timed(lambda: L.losa_calibrate_mass(q0, k0, N, C, Ck, want_lse=False, mass=mass_cal,
                                                workspace=ws_cal))
    cal2_t = timed(lambda: L.losa_calibrate_mass(q0, k0, N, C, Ck, want_lse=False, mass=mass_cal,
                                                 two_sweep=True))
    dense_t = None
    if not args.no_dense_compare:
        rp_full, ci_full = L.losa_select_blocks(mass_cal, N, C, Ck, 1.0)
        dense_t = timed(lambda: L.losa_sparse_attn_fwd(q0, k0, v0, N, C, Ck, rp_full, ci_full,
                                                       out=out, workspace=ws_fwd))
        del rp_full, ci_full

    # ---- cold forward: a 512 MiB write before each call evicts L2 and the
    # 256 MB Infinity Cache (the write is outside the events) -------------------
    cold = None
    if not args.no_cold:
        scratch = torch.empty((512 << 20) // 4, dtype=torch.float32, device=dev)
        evs = []
        for t in range(8):
            q, k, v = reuse_inputs[t % len(reuse_inputs)] if reuse_inputs else (q0, k0, v0)
            scratch.fill_(float(t))
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            L.losa_sparse_attn_fwd(q, k, v, N, C, Ck, row_ptr, col_idx, out=out,
                                   workspace=ws_fwd)
            b.record()
            evs.append((a, b))
        torch.cuda.synchronize()
        ct = sorted(a.elapsed_time(b) for a, b in evs)
        cold = {"median": round(ct[len(ct) // 2], 4), "min": round(ct[0], 4), "calls": len(ct)}
        del scratch

    # ---- recall of the frozen support at later steps (Eq. (2)) --------------
    recall = {}
    for t in sorted({1, (reuse + 1) // 2, reuse}):
        if t < 1 or t > reuse:
            continue
        q, k, _ = reuse_inputs[t - 1]
        L.losa_calibrate_mass(q, k, N, C, Ck, want_lse=False, mass=mass_cal, workspace=ws_cal)
        _, rh = L.losa_block_recall(mass_cal, N, C, Ck, row_ptr, col_idx, want_rows=False)
        rh = rh.float().cpu()
        recall[f"step{t}"] = {"mean": round(float(rh.mean()), 5), "worst_head": round(float(rh.min()), 5)}
    kk = max(1, round(nnz / rows))
    rp_k, ci_k = L.losa_select_blocks_topk(mass, N, C, Ck, kk)
    _, rh_k = L.losa_block_recall(mass, N, C, Ck, rp_k, ci_k, want_rows=False)
    _, rh_t = L.losa_block_recall(mass, N, C, Ck, row_ptr, col_idx, want_rows=False)
    recall["construction_step"] = {
        "threshold_rule": {"coverage": round(nnz / (rows * n_k), 4),
                           "mean": round(float(rh_t.float().mean()), 5),
                           "worst_head": round(float(rh_t.float().min()), 5)},
        "topk_rule_same_coverage": {"k": kk, "coverage": round(L.nnz(rp_k) / (rows * n_k), 4),
                                    "mean": round(float(rh_k.float().mean()), 5),
                                    "worst_head": round(float(rh_k.float().min()), 5)}}
    del rp_k, ci_k, ws_cal
    hbm = {"calibrate": {"algorithmic_GBs": round(alg["calibrate"] / cal_t / 1e6, 1),
                         "qk_tflops": round(qk_flop / (cal_t * 1e-3) / 1e12, 1),
                         "qk_frac_of_mfma_peak": round(qk_flop / (cal_t * 1e-3) / 1e12
                                                       / MFMA_BF16_PEAK_TFLOPS, 4)},
           "calibrate_two_sweep": {"algorithmic_GBs": round(alg["calibrate_two_sweep"] / cal2_t
                                                            / 1e6, 1),
                                   "qk_tflops": round(2 * qk_flop / (cal2_t * 1e-3) / 1e12, 1)},
           "select": {"algorithmic_GBs": round(alg["select"] / sel_t / 1e6, 1)},
           "note": "algorithmic bytes / measured time; counted_GBs = rocprofv3 FETCH_SIZE + "
                   "WRITE_SIZE bytes (scaled by a reference copy) / measured time; qk_tflops "
                   "counts one Q K^T per sweep (2 N_pad^2 d per head), the calibration's only "
                   "matrix work"}
    if traffic:
        kb = traffic["kernels"]
        tot = lambda key: kb.get(key, {}).get("fetch_bytes", 0) + kb.get(key, {}).get("write_bytes", 0)  # noqa: E731
        hbm["calibrate"]["counted_GBs"] = round((tot("calibrate") + tot("stat_mass")) / cal_t / 1e6,
                                                1)
        hbm["select"]["counted_GBs"] = round((tot("select_rows") + tot("compact_rows")) / sel_t / 1e6, 1)

    res = {
        "metric": "ms/layer + fraction of bf16 MFMA peak, block-sparse attn fwd, Wan-shaped tau=0.99",
        "value": round(fwd, 4),
        "unit": "ms/layer",
        "n_gpus": 1,
        "steps": args.steps,
        "warmup": args.warmup,
        "ms_per_step": round(wall / args.steps * 1e3, 3),
        "higher_is_better": False,
        "scaling": "weak",
        "vs_baseline": None,
        "dtype": w.dtype,
        "data": "synthetic",
        "config": {
            "workload": f"{w.name}-shaped: B={w.B} H={w.H} d={d} N={N} (padded {w.N_pad}) "
                        f"grid {w.grid[0]}x{w.grid[1]}x{w.grid[2]} "
                        + (f"block {C}" if Ck == C else f"blocks {C}x{Ck}") + f" tau={tau}",
            "step": f"construct (dense output + block masses) + select + {reuse} reuse sparse "
                    "forwards",
            "reuse_steps": reuse,
            "nnz_blocks": nnz,
            "retained_fraction": round(nnz / (rows * n_k), 4),
        },
        "fwd_ms": {"mean": round(fwd, 4), "median": round(fwd_sorted[len(fwd_sorted) // 2], 4),
                   "min": round(fwd_sorted[0], 4)},
        "fwd_cold_ms": cold,
        "construct_ms": round(con_t, 3),
        "select_ms": round(sel_t, 3),
        "calibrate_alone_ms": round(cal_t, 3),
        "calibrate_two_sweep_ms": round(cal2_t, 3),
        "dense_attn_ms": round(dense_t, 3) if dense_t else None,
        "construct_over_dense": round(con_t / dense_t, 3) if dense_t else None,
        "kernel_speedup_vs_full_csr": round(dense_t / fwd, 3) if dense_t else None,
        "retained_tflops": round(achieved, 1),
        "dense_equiv_tflops": round(dense_flop / (fwd * 1e-3) / 1e12, 1),
        "kernel_speedup_vs_dense_flops": round(dense_flop / retained_flop, 3),
        "roofline": {
            "bound": "mfma" if w.dtype == "bf16" else "alu",
            "achieved": round(achieved, 1),
            "peak": peak,
            "unit": "TFLOP/s",
            "frac": round(achieved / peak, 4),
            "traffic": traffic["bytes_per_launch"] if traffic else None,
            "traffic_algorithmic": alg["sparse_fwd"],
        },
        "hbm": hbm,
        "recall": recall,
        # the paper's own figures (Sec. 5: Tables 1-3), quoted as context: other
        # hardware, end-to-end sampling on real latents, not this kernel-level metric
        "paper_context": {
            "hardware": "NVIDIA H200, precision not stated",
            "wan2.1_1.3b_end_to_end_speedup": 1.36,
            "theta_0.99": {"coverage": 0.661, "recall": 0.990, "end_to_end_speedup": 1.37},
            "topk_rule_at_same_coverage_recall": 0.965,
            "note": "end-to-end sampling latency, construction step and non-attention work "
                    "included; compare with kernel_speedup_vs_full_csr, recall and "
                    "construction_step above",
        },
    }
    if not args.no_clock_context and w.dtype == "bf16":
        q, k, v = reuse_inputs[-1] if reuse_inputs else (q0, k0, v0)
        res["clock_context"] = clock_context(
            torch, lambda: L.losa_sparse_attn_fwd(q, k, v, N, C, Ck, row_ptr, col_idx, out=out,
                                                  workspace=ws_fwd), retained_flop)
    if not args.no_cpu_baseline:
        q, k, v = reuse_inputs[-1] if reuse_inputs else (q0, k0, v0)
        res["cpu_baseline"] = cpu_baseline(w, q, k, v, mass, row_ptr, col_idx, args.cpu_seconds)
        res["cpu_baseline"]["tiny_single_thread"] = tiny_single_thread()
    print(json.dumps(res), flush=True)


if __name__ == "__main__":
    main()
