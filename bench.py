#!/usr/bin/env python
"""HGEMM benchmark: prints ONE JSON line.

    python bench.py [--gpus N] [--steps K] [--warmup W] [--impl ours|reference] [--no-grid] [--grid-csv PATH] [--detail PATH]

A "step" is one pass of the hot path over the square HGEMM sweep (M = N = K in
{1024, 2048, 4096, 8192}: one plan/launch per shape, fp16 operands uniform in [-1, 1]
seeded per shape, fp32 accumulation, fp16 result).  `value` is the whole-job TFLOP/s
(flops of the sweep / device time, max over ranks) with inputs resident in HBM; `e2e` is the
same metric through the host-buffer entry point with the copies inside the timed region.
Extra keys: per-shape TFLOP/s beside torch.matmul on the same box; a sustained comparison (phases
of about a second, ours and torch.matmul alternating, SM clock per phase); the 729-shape grid against
torch.matmul (single GPU only) in four regimes -- warm back-to-back calls, cold L2 (buffer sets
rotate), single calls after idle gaps, and the GPU-side duration of one call of each arm as the
profiler records it, which leaves the host path out --; the memory-bound projection shapes against
the HBM roofline; one line each for the row-major-B layout, the alpha/beta form and fp16
accumulators; the roofline of the dominant kernel; the CPU oracle timed on the machine's cores; SM clocks
sampled during the timed region.  The long per-shape arrays (50 KB: every shape of the grid and of the
projections) are not part of the line; --detail PATH writes them.

Timing follows the paper's listing (section 2.4): synchronise, record an event, launch, record
an event, synchronise; no side streams.  With N > 1 every rank runs the same sweep on its own
GPU (replicas: the path has no exchange step) and the slowest rank sets the time.
"""
from __future__ import annotations

import argparse
import json
import math
import os
import random
import statistics
import subprocess
import sys
import threading
import time

ROOT = os.path.dirname(os.path.abspath(__file__))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

SWEEP = [1024, 2048, 4096, 8192]
GRID = [64, 128, 256, 512, 1024, 2048, 4096, 8192, 12288]
L2_BYTES = 126 * (1 << 20)
SPEC_TFLOPS = 2250.0
SPEC_HBM_GBS = 8000.0
# dram__bytes_read.sum + dram__bytes_write.sum of one 8192^3 launch of the dominant kernel,
# from the ncu capture summarised in profiles/hgemm_umma_kernel_dual_8192x8192x8192.md
DOMINANT_KERNEL_DRAM_BYTES = 0.869897e9 + 0.121344e9
METRIC = "HGEMM TFLOP/s"
WORKLOAD = "square HGEMM sweep M=N=K in {1024,2048,4096,8192}, one launch per shape per step"


def measured_peaks() -> dict:
    path = os.path.join(ROOT, "MEASURED_PEAKS.json")
    if os.path.exists(path):
        with open(path) as f:
            d = json.load(f)
        return {"source": "measured", "hbm_gbs": d["hbm_gbs"], "tflops_burst": d["bf16_tflops"],
                "tflops_sustained": d.get("bf16_tflops_sustained", d["bf16_tflops"])}
    return {"source": "fallback", "hbm_gbs": 6650.0, "tflops_burst": 1590.0, "tflops_sustained": 1400.0}


class ClockSampler:
    """Samples nvidia-smi clocks and throttle reasons while the timed region runs."""
    FIELDS = ("clocks.sm,clocks.max.sm,power.draw,clocks_event_reasons.hw_slowdown,"
              "clocks_event_reasons.hw_thermal_slowdown,clocks_event_reasons.sw_thermal_slowdown,"
              "clocks_event_reasons.sw_power_cap")

    def __init__(self, index: int):
        self.index = index
        self.rows = []
        self.proc = None
        self.thread = None

    def start(self):
        try:
            self.proc = subprocess.Popen(
                ["nvidia-smi", f"--id={self.index}", f"--query-gpu={self.FIELDS}", "--format=csv,noheader,nounits", "-lms", "50"],
                stdout=subprocess.PIPE, stderr=subprocess.DEVNULL, text=True)
        except OSError:
            self.proc = None
            return
        self.thread = threading.Thread(target=self._read, daemon=True)
        self.thread.start()

    def _read(self):
        for line in self.proc.stdout:
            self.rows.append((time.time(), [c.strip() for c in line.split(",")]))

    def stop(self, t0: float, t1: float) -> dict:
        if self.proc is None:
            return {"sm_mhz": None, "sm_max_mhz": None, "reasons": ["nvidia-smi unavailable"]}
        time.sleep(0.15)
        self.proc.terminate()
        try:
            self.proc.wait(timeout=5)
        except subprocess.TimeoutExpired:
            self.proc.kill()
        rows = [r for (t, r) in self.rows if t0 <= t <= t1 + 0.2 and len(r) >= 7] or [r for (_, r) in self.rows if len(r) >= 7]
        sm, mx, pw, reasons = [], [], [], set()
        names = ["hw_slowdown", "hw_thermal_slowdown", "sw_thermal_slowdown", "sw_power_cap"]
        for r in rows:
            try:
                sm.append(float(r[0]))
                mx.append(float(r[1]))
                pw.append(float(r[2]))
            except ValueError:
                continue
            for name, v in zip(names, r[3:7]):
                if v.lower().startswith("active"):
                    reasons.add(name)
        return {"sm_mhz": statistics.median(sm) if sm else None, "sm_max_mhz": max(mx) if mx else None,
                "power_w_max": max(pw) if pw else None, "samples": len(sm), "reasons": sorted(reasons)}


def flops(M, N, K):
    return 2.0 * M * N * K


def compulsory_bytes(M, N, K):
    return 2.0 * (M * K + N * K + M * N)


# --------------------------------------------------------------------------------------------------
# the reference arm: the CPU oracle, as it stands, on bounded row slabs of the same sweep

def oracle_slab(oracle, inputs, S: int, rows: int):
    a = inputs.draw(inputs.shape_seed(S, S, S), inputs.TAG_A, S, S, "uniform", "cpu", row_index=list(range(rows)))
    b = inputs.draw(inputs.shape_seed(S, S, S), inputs.TAG_B, S, S, "uniform", "cpu")
    return inputs.bits(a), inputs.bits(b)


def run_reference(args) -> None:
    rank = int(os.environ.get("RANK", "0"))
    if rank != 0:
        return
    import oracle
    from paper_2512_02551_b200 import inputs
    oracle.build()
    # rows of C per shape per step, sized so that warm-up + steps end within about a minute
    per_row_macs = sum(S * S for S in SWEEP)
    rows = max(1, min(96, int(60.0 * 15e9 / ((args.steps + args.warmup) * per_row_macs))))
    slabs = [(S, *oracle_slab(oracle, inputs, S, rows)) for S in SWEEP]
    macs = sum(rows * S * S for S in SWEEP)
    for _ in range(max(args.warmup, 1) if args.warmup else 0):
        for S, a, b in slabs:
            oracle.hgemm_full(a, b)
    t0 = time.perf_counter()
    for _ in range(args.steps):
        for S, a, b in slabs:
            oracle.hgemm_full(a, b)
    dt = time.perf_counter() - t0
    value = 2.0 * macs * args.steps / dt / 1e12
    sample = f"per step: first {rows} rows of C for each sweep shape ({macs / 1e9:.1f} GMAC)"
    line = {
        "impl": "reference", "metric": METRIC, "value": value, "unit": "TFLOP/s", "n_gpus": args.gpus,
        "steps": args.steps, "warmup": args.warmup, "ms_per_step": dt / args.steps * 1e3,
        "higher_is_better": True, "scaling": "weak", "vs_baseline": None, "dtype": "f64", "data": "synthetic",
        "config": {"workload": WORKLOAD, "sample": sample},
        "cpu_baseline": {"value": value, "unit": "TFLOP/s", "cores": oracle.max_threads(), "kind": "oracle", "sample": sample},
        "e2e": {"value": value, "unit": "TFLOP/s", "h2d_bytes_per_step": 0, "d2h_bytes_per_step": 0},
        "gpu_launches": 0,
    }
    print(json.dumps(line), flush=True)


# --------------------------------------------------------------------------------------------------
# our arm

def emit(line: dict, detail: dict, path: str | None) -> None:
    """The JSON line to stdout; the long arrays, which would make it too long for some readers, to a file if one is named."""
    if path:
        with open(path, "w") as f:
            json.dump(detail, f)
    print(json.dumps(line), flush=True)


def run_ours(args) -> None:
    import torch
    from paper_2512_02551_b200 import build as hbuild
    from paper_2512_02551_b200 import hgemm, inputs, replicas

    world = int(os.environ.get("WORLD_SIZE", "1"))
    rank = int(os.environ.get("RANK", "0"))
    local = int(os.environ.get("LOCAL_RANK", "0"))
    if not torch.cuda.is_available():
        raise SystemExit("bench.py needs a GPU (there is no CPU fallback)")
    if rank == 0:
        hbuild.build()
    torch.cuda.set_device(local)
    dist = None
    if world > 1:
        import torch.distributed as dist
        dist.init_process_group("nccl", device_id=torch.device("cuda", local))
        dist.barrier()

    def barrier():
        replicas.barrier(dist)
        torch.cuda.synchronize()

    ctx = hgemm.Context(local)
    stream = torch.cuda.current_stream()

    def check_status(where: str):
        st, code = ctx.last_device_status()
        if st != hgemm.OK:
            raise SystemExit(f"device status {st} code {code:#x} after {where}")

    # ---- buffers: enough distinct (A, B, C) sets per shape that the footprint exceeds 2x L2 ----
    work = []
    for S in SWEEP:
        sets = max(1, math.ceil(2 * L2_BYTES / compulsory_bytes(S, S, S)))
        A0, B0 = inputs.make_ab(S, S, S, "uniform", "cuda")
        bufs = []
        for r in range(sets):
            A = A0 if r == 0 else A0.clone()
            B = B0 if r == 0 else B0.clone()
            bufs.append((A, B, torch.empty(S, S, dtype=torch.float16, device="cuda")))
        work.append({"S": S, "plan": ctx.plan(S, S, S), "bufs": bufs})
    step_flops = sum(flops(S, S, S) for S in SWEEP)

    # Inside the timed region only the dominant launch (the largest shape) is bracketed by events -- its duration is what the
    # roofline figure is computed from; events around every launch would put a record between each pair of kernels, which is
    # instrumentation, not workload.  The other shapes' durations come from a separate pass (`every=True`) after the timed one.
    def one_step(i, events=None, every=False):
        for w in work:
            A, B, C = w["bufs"][i % len(w["bufs"])]
            if events is not None and (every or w["S"] == SWEEP[-1]):
                e0 = torch.cuda.Event(enable_timing=True)
                e1 = torch.cuda.Event(enable_timing=True)
                e0.record(stream)
                w["plan"].run_ptr(A.data_ptr(), B.data_ptr(), C.data_ptr(), stream.cuda_stream)
                e1.record(stream)
                events.append((w["S"], e0, e1))
            else:
                w["plan"].run_ptr(A.data_ptr(), B.data_ptr(), C.data_ptr(), stream.cuda_stream)

    def torch_step(i, events=None, every=False):
        for w in work:
            A, B, C = w["bufs"][i % len(w["bufs"])]
            if events is not None and (every or w["S"] == SWEEP[-1]):
                e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
                e0.record(stream)
                torch.matmul(A, B.T, out=C)
                e1.record(stream)
                events.append((w["S"], e0, e1))
            else:
                torch.matmul(A, B.T, out=C)

    def timed(fn, steps, warmup, sampler=None, label="hgemm_timed_region"):
        for i in range(warmup):
            fn(i)
        barrier()
        t0w = time.time()
        if sampler:
            sampler.start()
            time.sleep(0.25)
            t0w = time.time()
        e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        torch.cuda.nvtx.range_push(label)
        e0.record(stream)
        for i in range(steps):
            fn(warmup + i)
        e1.record(stream)
        barrier()
        torch.cuda.nvtx.range_pop()
        t1w = time.time()
        ms = replicas.slowest_rank_ms(e0.elapsed_time(e1), dist, "cuda")
        return ms, t0w, t1w

    # ---- the timed region ---------------------------------------------------------------------
    sampler = ClockSampler(local) if rank == 0 else None
    events = []
    ms_total, t0w, t1w = timed(lambda i: one_step(i, events), args.steps, args.warmup, sampler)
    clocks = sampler.stop(t0w, t1w) if sampler else None
    check_status("the timed region")
    ms_per_step = ms_total / args.steps
    value = replicas.job_throughput(step_flops, world, ms_per_step) / 1e12
    per_launch = {}
    for S, e0, e1 in events[-args.steps:]:                       # the dominant launch, inside the timed region
        per_launch.setdefault(S, []).append(e0.elapsed_time(e1))
    side_events = []                                             # every shape, in a pass of its own (not part of `value`)
    for i in range(min(args.steps, 50)):
        one_step(args.warmup + args.steps + i, side_events, every=True)
    torch.cuda.synchronize()
    for S, e0, e1 in side_events:
        if S != SWEEP[-1]:
            per_launch.setdefault(S, []).append(e0.elapsed_time(e1))
    per_shape = {}
    for S, v in per_launch.items():
        ms = statistics.mean(v)
        per_shape[str(S)] = {"us": ms * 1e3, "tflops": flops(S, S, S) / (ms * 1e-3) / 1e12,
                             "config": work[SWEEP.index(S)]["plan"].config.as_dict()}

    roofline = None
    if rank == 0:
        peaks = measured_peaks()
        dom = per_shape[str(SWEEP[-1])]
        timed_s = ms_total * 1e-3
        # the burst figure for a short timed region (the default 20-step run lasts about 20 ms), the sustained one once the
        # region is long enough for the power cap to have settled the clock (the 1000-step run lasts about a second)
        long_region = timed_s > 0.5
        peak = peaks["tflops_sustained"] if long_region else peaks["tflops_burst"]
        roofline = {"bound": "tensor", "kernel": "hgemm_umma_kernel, 8192^3 launch", "achieved": dom["tflops"], "peak": peak,
                    "unit": "TFLOP/s", "frac": dom["tflops"] / peak,
                    "peak_source": f"{peaks['source']} cuBLAS bf16 {'sustained' if long_region else 'burst'} (fp16 dense = bf16 dense)",
                    "timed_region_s": timed_s,
                    "traffic": DOMINANT_KERNEL_DRAM_BYTES,
                    "traffic_source": "one ncu capture of this launch, profiles/hgemm_umma_kernel_dual_8192x8192x8192.md; not measured in this run",
                    "algorithmic_flops_per_launch": flops(8192, 8192, 8192),
                    "compulsory_bytes_per_launch": compulsory_bytes(8192, 8192, 8192),
                    "frac_of_spec_peak": dom["tflops"] / SPEC_TFLOPS}

    # ---- torch.matmul on the same buffers, same protocol (comparison point, single rank) --------
    torch_cmp = None
    if rank == 0:
        tev = []
        for i in range(args.warmup):
            torch_step(i)
        torch.cuda.synchronize()
        e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        e0.record(stream)
        for i in range(args.steps):
            torch_step(args.warmup + i, tev)
        e1.record(stream)
        torch.cuda.synchronize()
        tms = e0.elapsed_time(e1) / args.steps
        tside = []
        for i in range(min(args.steps, 50)):
            torch_step(args.warmup + args.steps + i, tside, every=True)
        torch.cuda.synchronize()
        tps = {}
        for S, a, b in tev + [t for t in tside if t[0] != SWEEP[-1]]:
            tps.setdefault(S, []).append(a.elapsed_time(b))
        torch_cmp = {"value": step_flops / (tms * 1e-3) / 1e12, "unit": "TFLOP/s",
                     "per_shape_tflops": {str(S): flops(S, S, S) / (statistics.mean(v) * 1e-3) / 1e12 for S, v in tps.items()}}

    # ---- sustained comparison: phases of about a second under the power cap, arms alternating ----------
    sustained = None
    if rank == 0 and world == 1 and not args.no_grid:
        sustained = sustained_report(torch, one_step, torch_step, step_flops, ms_per_step, local, stream)
        check_status("the sustained phases")

    # ---- end to end: host buffers, copies inside the timed region --------------------------------
    host = []
    for w in work:
        S = w["S"]
        A, B, _ = w["bufs"][0]
        hA = torch.empty(S, S, dtype=torch.float16).pin_memory()
        hB = torch.empty(S, S, dtype=torch.float16).pin_memory()
        hC = torch.empty(S, S, dtype=torch.float16).pin_memory()
        hA.copy_(A)
        hB.copy_(B)
        host.append((w["plan"], hA, hB, hC))
    h2d = sum(hA.numel() * 2 + hB.numel() * 2 for _, hA, hB, _ in host)
    d2h = sum(hC.numel() * 2 for *_, hC in host)

    def e2e_step(i):
        for plan, hA, hB, hC in host:
            plan.run_host(hA, hB, hC, stream.cuda_stream)
    e2e_steps = max(3, min(args.steps, 10))
    e2e_ms, _, _ = timed(e2e_step, e2e_steps, 2, label="hgemm_e2e_region")
    e2e_value = replicas.job_throughput(step_flops, world, e2e_ms / e2e_steps) / 1e12
    # the result that came back is the GEMM's (spot check against the device-resident run)
    if rank == 0:
        _, _, _, hC = host[0]
        _, _, C = work[0]["bufs"][0]
        work[0]["plan"].run(work[0]["bufs"][0][0], work[0]["bufs"][0][1], C)
        torch.cuda.synchronize()
        assert torch.equal(hC, C.cpu()), "host-buffer path returned a different result"
    del host

    variants = None
    if rank == 0 and world == 1 and not args.no_grid:
        variants = variant_lines(ctx, torch, hgemm, inputs, stream)
        check_status("the variant lines")
    for w in work:
        w["plan"].close()
    del work
    torch.cuda.empty_cache()

    # ---- the 729-shape grid against torch.matmul (single GPU) ------------------------------------
    grid = None
    if rank == 0 and world == 1 and not args.no_grid:
        grid = grid_sweep(ctx, torch, hgemm, inputs, stream, args.grid_csv)
        check_status("the grid sweep")

    if grid is not None:
        # the paper's full grid has ten values per dimension: the 271 shapes with a 16384 in them, warm regime
        extra = grid10_extra(ctx, torch, hgemm, inputs, stream)
        check_status("the shapes with 16384")
        logs = [math.log(tt / to) for (_, _, _, to, tt) in extra]
        warm_logs = [math.log(r[4] / r[3]) for r in grid["detail"]["rows"]]
        grid["paper_grid_1000"] = {
            "shapes": len(extra) + len(warm_logs), "regime": "warm back-to-back calls; the 271 shapes with a 16384: best of two interleaved rounds",
            "geomean_torch_time_over_ours": math.exp((sum(logs) + sum(warm_logs)) / (len(logs) + len(warm_logs))),
            "geomean_of_the_271_with_16384": math.exp(sum(logs) / len(logs)),
            "wins_among_the_271": sum(x > 0 for x in logs),
            "worst_of_the_271": min(({"shape": [M, N, K], "ratio": tt / to} for (M, N, K, to, tt) in extra), key=lambda e: e["ratio"])}
        torch.cuda.empty_cache()

    skinny = None
    if rank == 0 and world == 1 and not args.no_grid:
        skinny = skinny_report(ctx, torch, hgemm, inputs, stream)
        check_status("the projection shapes")

    # ---- the CPU oracle on the machine's cores, on a bounded sample -------------------------------------
    cpu = None
    if rank == 0 and world == 1:
        import oracle
        oracle.build()
        rows = 384
        a, b = oracle_slab(oracle, inputs, 8192, rows)
        t0 = time.perf_counter()
        oracle.hgemm_full(a, b)
        dt = time.perf_counter() - t0
        cpu = {"value": 2.0 * rows * 8192 * 8192 / dt / 1e12, "unit": "TFLOP/s", "cores": oracle.max_threads(), "kind": "oracle",
               "sample": f"first {rows} rows of C for 8192^3 ({rows * 8192 * 8192 / 1e9:.1f} GMAC, {dt:.2f} s wall)"}

    if rank == 0:
        grid_detail = grid.pop("detail") if grid else None
        skinny_shapes = skinny.pop("shapes") if skinny else None
        line = {
            "metric": METRIC, "value": value, "unit": "TFLOP/s", "n_gpus": world, "steps": args.steps, "warmup": args.warmup,
            "ms_per_step": ms_per_step, "higher_is_better": True, "scaling": "weak", "vs_baseline": None, "dtype": "f16",
            "data": "synthetic",
            "config": {"workload": WORKLOAD, "accumulate": "f32", "inputs": "uniform[-1,1) rounded to fp16, seeded per shape",
                       "l2": "inputs larger than L2: buffer sets rotate so that each shape's footprint exceeds 2x the 126 MB L2",
                       "events": "inside the timed region only the dominant launch (8192^3) is bracketed by CUDA events; the other shapes' "
                                 "durations in per_shape come from a separate pass after it; torch.matmul is timed the same way",
                       "parallelism": "replicas" if world > 1 else "single GPU"},
            "pct_of_spec_peak": 100.0 * value / world / SPEC_TFLOPS,
            "per_shape": per_shape, "variants": variants, "skinny": skinny, "grid": grid, "torch_matmul": torch_cmp, "sustained": sustained,
            "roofline": roofline, "cpu_baseline": cpu, "clocks": clocks,
            "e2e": {"value": e2e_value, "unit": "TFLOP/s", "h2d_bytes_per_step": h2d, "d2h_bytes_per_step": d2h, "steps": e2e_steps},
            "gpu_launches": args.steps * len(SWEEP),
        }
        emit(line, {"skinny_shapes": skinny_shapes, "grid_detail": grid_detail}, args.detail)
    ctx.close()
    if dist is not None:
        dist.destroy_process_group()


def sustained_report(torch, one_step, torch_step, step_flops, ms_per_step, gpu_index, stream) -> dict:
    """The square sweep under the power cap: four phases of about 0.8 s each, ours / torch.matmul / ours / torch.matmul,
    same rotating buffers, SM clock sampled per phase.  time x clock (device cycles per step) compares boxes whose
    power caps settle at different clocks."""
    n = max(20, min(2000, int(800.0 / max(ms_per_step, 1e-3))))
    phases = []
    for name, fn in (("ours", one_step), ("torch", torch_step), ("ours", one_step), ("torch", torch_step)):
        for i in range(3):
            fn(i)
        torch.cuda.synchronize()
        sampler = ClockSampler(gpu_index)
        sampler.start()
        time.sleep(0.1)
        t0 = time.time()
        e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        e0.record(stream)
        for i in range(n):
            fn(i)
        e1.record(stream)
        torch.cuda.synchronize()
        t1 = time.time()
        clk = sampler.stop(t0, t1)
        ms = e0.elapsed_time(e1) / n
        phases.append({"arm": name, "tflops": step_flops / (ms * 1e-3) / 1e12, "ms_per_step": ms, "sm_mhz": clk.get("sm_mhz"),
                       "mcycles_per_step": (ms * 1e-3 * clk["sm_mhz"]) if clk.get("sm_mhz") else None, "reasons": clk.get("reasons")})
    ours = statistics.mean(p["tflops"] for p in phases if p["arm"] == "ours")
    ref = statistics.mean(p["tflops"] for p in phases if p["arm"] == "torch")
    return {"regime": f"{n} steps per phase, ours and torch.matmul alternating, rotating buffers", "phases": phases,
            "ours_tflops": ours, "torch_tflops": ref, "ours_over_torch": ours / ref}


def variant_lines(ctx, torch, hgemm, inputs, stream) -> dict:
    """One figure each for the row-major-B layout, the alpha/beta form and fp16 accumulators, on 4096^3 (warm calls,
    torch's counterpart beside it where it has one)."""
    S = 4096
    A, B = inputs.make_ab(S, S, S, "uniform", "cuda")
    Bkn = B.T.contiguous()                                   # the K x N row-major operand
    C = torch.zeros(S, S, dtype=torch.float16, device="cuda")
    s = stream.cuda_stream

    def per_call_ms(fn, n=60):
        for _ in range(5):
            fn()
        e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        e0.record(stream)
        for _ in range(n):
            fn()
        e1.record(stream)
        e1.synchronize()
        return e0.elapsed_time(e1) / n

    def tf(ms):
        return flops(S, S, S) / (ms * 1e-3) / 1e12

    out = {"shape": [S, S, S], "regime": "warm back-to-back calls"}
    plan = ctx.plan(S, S, S)
    out["tn_plain"] = {"tflops": tf(per_call_ms(lambda: plan.run_ptr(A.data_ptr(), B.data_ptr(), C.data_ptr(), s))),
                       "torch_tflops": tf(per_call_ms(lambda: torch.matmul(A, B.T, out=C)))}
    nn = ctx.plan(S, S, S, layout=hgemm.LAYOUT_NN)
    out["nn_layout"] = {"tflops": tf(per_call_ms(lambda: nn.run_ptr(A.data_ptr(), Bkn.data_ptr(), C.data_ptr(), s))),
                        "torch_tflops": tf(per_call_ms(lambda: torch.matmul(A, Bkn, out=C))), "config": nn.config.as_dict()}
    nn.close()
    C.zero_()
    out["alpha_beta"] = {"tflops": tf(per_call_ms(lambda: plan.run_scaled(0.5, 0.25, A, B, C))),
                         "torch_tflops": tf(per_call_ms(lambda: torch.addmm(C, A, B.T, beta=0.25, alpha=0.5, out=C))),
                         "alpha": 0.5, "beta": 0.25}
    cfg = plan.config
    cfg.accumulate = hgemm.ACC_F16
    if cfg.tail_split >= 2 and cfg.tail_mode == hgemm.TAIL_K:
        cfg.tail_split = 0
    if plan.try_set_config(cfg) == hgemm.OK:
        entry = {"tflops": tf(per_call_ms(lambda: plan.run_ptr(A.data_ptr(), B.data_ptr(), C.data_ptr(), s)))}
        flag = getattr(torch.backends.cuda.matmul, "allow_fp16_accumulation", None)
        if flag is not None:
            torch.backends.cuda.matmul.allow_fp16_accumulation = True
            try:
                entry["torch_tflops"] = tf(per_call_ms(lambda: torch.matmul(A, B.T, out=C)))
            finally:
                torch.backends.cuda.matmul.allow_fp16_accumulation = flag
        out["fp16_accumulate"] = entry
    plan.close()
    return out


def device_durations(torch, calls) -> list:
    """GPU-side duration in microseconds of each call in `calls` (a list of callables): from the start of the first
    kernel the call launches to the end of the last, as the profiler's activity records give it.  The host path
    (argument checks, heuristics, launch) is not in it.  None entries where the profiler gave nothing."""
    from torch.profiler import ProfilerActivity, profile, record_function
    out = [None] * len(calls)
    CHUNK = 300
    for c0 in range(0, len(calls), CHUNK):
        part = calls[c0:c0 + CHUNK]
        with profile(activities=[ProfilerActivity.CPU, ProfilerActivity.CUDA]) as prof:
            for j, fn in enumerate(part):
                with record_function(f"hgemm_bench_call_{c0 + j}"):
                    fn()
                torch.cuda.synchronize()
        # the profiler mirrors every annotation on the GPU timeline: an event of the same name whose span runs from the
        # start of the first kernel launched inside the annotation to the end of the last one
        for ev in prof.events():
            name = ev.name
            if name.startswith("hgemm_bench_call_") and ev.device_type == torch.autograd.DeviceType.CUDA:
                dur = ev.time_range.end - ev.time_range.start            # microseconds
                if dur > 0:
                    out[int(name.rsplit("_", 1)[1])] = float(dur)
    return out


def grid_sweep(ctx, torch, hgemm, inputs, stream, csv_path=None) -> dict:
    """All 729 grid shapes, ours against torch.matmul on the same buffers, in four regimes.

    warm    back-to-back calls on one buffer set (the paper's offline mode): batches of n calls between two events,
            ours/torch batches interleaved in seeded random order, median over rounds
    cold    the same with the buffer sets rotating through more than 2x L2 of A/B/C, so that no call finds its
            operands in L2 (shapes whose single set already exceeds 2x L2 keep one set)
    server  single calls after idle gaps that are not timed (paper section 2.4): short gaps of 20-200 us on the warm
            buffers, and gaps of at least 2 ms on the rotating buffers (caches cool down, the clock governor reacts)
    device  the GPU-side duration of one warm call of each arm from the profiler's kernel records: no host path
    Buffers are dense prefixes (and, for the rotating sets, consecutive slices) of three pools."""
    mx = GRID[-1]
    pool = (max(mx * mx, int(2.2 * L2_BYTES) // 2 + mx * mx) + 4095) // 4096 * 4096   # elements: room for > 2x L2 of any one operand
    A_all = inputs.draw(1, inputs.TAG_A, pool // 4096, 4096, "uniform", "cuda").view(-1)
    B_all = inputs.draw(1, inputs.TAG_B, pool // 4096, 4096, "uniform", "cuda").view(-1)
    C_all = torch.empty(pool, dtype=torch.float16, device="cuda")
    rng = random.Random(729)
    peaks = measured_peaks()
    rows = []
    dev_calls, dev_meta = [], []
    plans = []

    def batch_ms(fn, n):
        e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        e0.record(stream)
        for i in range(n):
            fn(i)
        e1.record(stream)
        e1.synchronize()
        return e0.elapsed_time(e1) / n

    def idle(seconds):
        t = time.perf_counter() + seconds
        while time.perf_counter() < t:
            pass

    for M in GRID:
        for N in GRID:
            for K in GRID:
                foot = compulsory_bytes(M, N, K)
                sets = max(1, min(math.ceil(2 * L2_BYTES / foot), (pool - 1) // max(M * K, N * K, M * N)))
                bufs = []
                for r in range(sets):
                    A = A_all[r * M * K:(r + 1) * M * K].view(M, K)
                    B = B_all[r * N * K:(r + 1) * N * K].view(N, K)
                    C = C_all[r * M * N:(r + 1) * M * N].view(M, N)
                    bufs.append((A, B.T, C, A.data_ptr(), B.data_ptr(), C.data_ptr()))
                plan = ctx.plan(M, N, K)
                s = stream.cuda_stream
                A0, Bt0, C0, a0, b0, c0 = bufs[0]
                # (defaults bind this iteration's plan and buffers: the callables are used again after the loop)
                ours_w = lambda i, plan=plan, a0=a0, b0=b0, c0=c0: plan.run_ptr(a0, b0, c0, s)      # noqa: E731
                ref_w = lambda i, A0=A0, Bt0=Bt0, C0=C0: torch.matmul(A0, Bt0, out=C0)            # noqa: E731

                def ours_c(i, bufs=bufs, plan=plan):
                    b = bufs[i % len(bufs)]
                    plan.run_ptr(b[3], b[4], b[5], s)

                def ref_c(i, bufs=bufs):
                    b = bufs[i % len(bufs)]
                    torch.matmul(b[0], b[1], out=b[2])
                for fn in (ours_w, ref_w):
                    for i in range(3):
                        fn(i)
                est = max(batch_ms(ours_w, 3), 1e-3)
                n = max(3, min(200, int(1.0 / est)))
                t = {"ours": [], "torch": [], "ours_cold": [], "torch_cold": []}
                for _ in range(3):
                    order = [("ours", ours_w), ("torch", ref_w)]
                    rng.shuffle(order)
                    for name, fn in order:
                        t[name].append(batch_ms(fn, n))
                if sets > 1:
                    for fn in (ours_c, ref_c):                                       # tensor maps of every set encoded, kernels loaded
                        batch_ms(fn, sets)
                    nc = max(sets, min(200, int(1.0 / est)))
                    for _ in range(3):
                        order = [("ours_cold", ours_c), ("torch_cold", ref_c)]
                        rng.shuffle(order)
                        for name, fn in order:
                            t[name].append(batch_ms(fn, nc))
                else:
                    t["ours_cold"], t["torch_cold"] = t["ours"], t["torch"]
                to, tt = statistics.median(t["ours"]), statistics.median(t["torch"])
                toc, ttc = statistics.median(t["ours_cold"]), statistics.median(t["torch_cold"])
                # server mode, short gaps: single calls on the warm buffers, each bracketed by its own pair of events
                ts = {"ours": [], "torch": []}
                for _ in range(5):
                    order = [("ours", ours_w), ("torch", ref_w)]
                    rng.shuffle(order)
                    for name, fn in order:
                        idle(rng.uniform(20e-6, 200e-6))
                        ts[name].append(batch_ms(fn, 1))
                # server mode, long gaps: at least 2 ms of idle time, rotating buffers, 15 single calls per arm
                tl = {"ours": [], "torch": []}
                for j in range(15):
                    order = [("ours", ours_c), ("torch", ref_c)]
                    rng.shuffle(order)
                    for name, fn in order:
                        idle(rng.uniform(2.0e-3, 2.5e-3))
                        tl[name].append(batch_ms(lambda i, fn=fn, j=j: fn(j), 1))
                t_roof = max(flops(M, N, K) / (peaks["tflops_burst"] * 1e12), foot / (peaks["hbm_gbs"] * 1e9))
                rows.append({"shape": (M, N, K), "ours": to * 1e3, "torch": tt * 1e3, "ours_cold": toc * 1e3, "torch_cold": ttc * 1e3,
                             "srv_ours": statistics.median(ts["ours"]) * 1e3, "srv_torch": statistics.median(ts["torch"]) * 1e3,
                             "srvl_ours": statistics.median(tl["ours"]) * 1e3, "srvl_torch": statistics.median(tl["torch"]) * 1e3,
                             "roof_us": t_roof * 1e6, "sets": sets})
                dev_calls += [lambda f=ours_w: f(0), lambda f=ref_w: f(0)]
                dev_meta.append(len(rows) - 1)
                plans.append(plan)
    # device-side durations of one warm call per arm (the plans are still alive: the callables hold them)
    dev_error = None
    try:
        for fn in dev_calls:                                # every kernel loaded, every map encoded
            fn()
        torch.cuda.synchronize()
        dur = device_durations(torch, dev_calls)
        for j, ri in enumerate(dev_meta):
            rows[ri]["dev_ours"], rows[ri]["dev_torch"] = dur[2 * j], dur[2 * j + 1]
    except Exception as e:                                  # no profiler on this machine: the regime is reported as absent
        dev_error = f"{type(e).__name__}: {e}"
    for plan in plans:
        plan.close()

    def geo(pairs):
        pairs = [(a, b) for a, b in pairs if a and b]
        return math.exp(sum(math.log(b / a) for a, b in pairs) / len(pairs)) if pairs else None

    def summary(ko, kt, sel=lambda r: True):
        use = [r for r in rows if sel(r) and r.get(ko) and r.get(kt)]
        if not use:
            return None
        ratios = [r[kt] / r[ko] for r in use]
        return {"shapes": len(use), "geomean_torch_time_over_ours": geo([(r[ko], r[kt]) for r in use]),
                "mean_speedup_minus_1": sum(x - 1.0 for x in ratios) / len(ratios), "win_rate": sum(x > 1.0 for x in ratios) / len(ratios)}

    if csv_path:
        with open(csv_path, "w") as f:
            cols = ["ours", "torch", "ours_cold", "torch_cold", "srv_ours", "srv_torch", "srvl_ours", "srvl_torch", "dev_ours", "dev_torch"]
            f.write("M,N,K,sets," + ",".join(c + "_us" for c in cols) + "\n")
            for r in rows:
                f.write(",".join(str(v) for v in r["shape"]) + f",{r['sets']}," +
                        ",".join("" if r.get(c) is None else f"{r[c]:.3f}" for c in cols) + "\n")

    big = [r for r in rows if min(r["shape"]) >= 4096]
    worst = sorted(rows, key=lambda r: r["torch"] / r["ours"])[:5]
    worst_dev = sorted((r for r in rows if r.get("dev_ours") and r.get("dev_torch")), key=lambda r: r["dev_torch"] / r["dev_ours"])[:5]
    device = None
    if dev_error is None:
        device = summary("dev_ours", "dev_torch")
        if device:
            device["regime"] = "GPU-side duration of one warm call per arm (first kernel start to last kernel end), from the profiler"
            device["buckets_by_our_device_time"] = {
                "under_5us": summary("dev_ours", "dev_torch", lambda r: (r.get("dev_ours") or 0) < 5.0),
                "5_to_30us": summary("dev_ours", "dev_torch", lambda r: 5.0 <= (r.get("dev_ours") or 0) < 30.0),
                "over_30us": summary("dev_ours", "dev_torch", lambda r: (r.get("dev_ours") or 0) >= 30.0)}
    warm = summary("ours", "torch")
    out = {
        "detail": {"columns": ["M", "N", "K", "ours_us", "torch_us", "ours_cold_us", "torch_cold_us", "dev_ours_us", "dev_torch_us"],
                   "rows": [list(r["shape"]) + [round(r["ours"], 2), round(r["torch"], 2), round(r["ours_cold"], 2), round(r["torch_cold"], 2),
                                                None if r.get("dev_ours") is None else round(r["dev_ours"], 2),
                                                None if r.get("dev_torch") is None else round(r["dev_torch"], 2)] for r in rows],
                   "worst5_warm": [{"shape": list(r["shape"]), "ratio": r["torch"] / r["ours"], "ours_us": r["ours"], "torch_us": r["torch"]} for r in worst],
                   "worst5_device": [{"shape": list(r["shape"]), "ratio": r["dev_torch"] / r["dev_ours"], "ours_us": r["dev_ours"],
                                      "torch_us": r["dev_torch"]} for r in worst_dev]},
        "shapes": len(rows), "regime": "warm, back-to-back calls (the paper's offline mode)",
        "geomean_torch_time_over_ours": warm["geomean_torch_time_over_ours"], "wins": sum(r["torch"] > r["ours"] for r in rows),
        "mean_speedup_minus_1": warm["mean_speedup_minus_1"], "offline_win_rate": warm["win_rate"],
        "geomean_fraction_of_measured_roofline": math.exp(sum(math.log(r["roof_us"] / r["ours"]) for r in rows) / len(rows)),
        "geomean_fraction_of_measured_roofline_cold": math.exp(sum(math.log(r["roof_us"] / r["ours_cold"]) for r in rows) / len(rows)),
        "compute_bound_min_tflops": min(flops(*r["shape"]) / (r["ours"] * 1e-6) / 1e12 for r in big),
        "compute_bound_geomean_vs_torch": geo([(r["ours"], r["torch"]) for r in big]),
        "cold": dict(summary("ours_cold", "torch_cold"), regime="buffer sets rotate through more than 2x L2 (every call finds its operands cold)",
                     rotated_shapes=sum(r["sets"] > 1 for r in rows)),
        "server_mode": dict(summary("srv_ours", "srv_torch"), regime="single calls after random idle gaps of 20-200 us, gap not timed, median of 5, warm buffers"),
        "server_mode_long_gaps": dict(summary("srvl_ours", "srvl_torch"),
                                      regime="single calls after idle gaps of 2.0-2.5 ms, gap not timed, median of 15, rotating buffers"),
        "device_time": device, "device_time_error": dev_error,
    }
    return out


def grid10_extra(ctx, torch, hgemm, inputs, stream) -> list:
    """The 271 shapes that the paper's tenth grid value, 16384, adds to the 9 x 9 x 9 grid: warm back-to-back calls only,
    two interleaved rounds per arm (these are the largest shapes; each call streams far more than L2 anyway).
    Returns [(M, N, K, ours_us, torch_us)]."""
    g10 = GRID + [16384]
    mx = 16384
    A_all = inputs.draw(2, inputs.TAG_A, mx, mx, "uniform", "cuda").view(-1)
    B_all = inputs.draw(2, inputs.TAG_B, mx, mx, "uniform", "cuda").view(-1)
    C_all = torch.empty(mx * mx, dtype=torch.float16, device="cuda")
    out = []

    def batch_ms(fn, n):
        e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        e0.record(stream)
        for _ in range(n):
            fn()
        e1.record(stream)
        e1.synchronize()
        return e0.elapsed_time(e1) / n

    for M in g10:
        for N in g10:
            for K in g10:
                if 16384 not in (M, N, K):
                    continue
                A = A_all[:M * K].view(M, K)
                B = B_all[:N * K].view(N, K)
                C = C_all[:M * N].view(M, N)
                plan = ctx.plan(M, N, K)
                a, b, c, s = A.data_ptr(), B.data_ptr(), C.data_ptr(), stream.cuda_stream
                Bt = B.T
                ours = lambda: plan.run_ptr(a, b, c, s)               # noqa: E731
                ref = lambda: torch.matmul(A, Bt, out=C)              # noqa: E731
                ours()
                ref()
                est = max(batch_ms(ours, 2), 1e-3)
                n = max(2, min(100, int(0.5 / est)))
                t = {"ours": [], "torch": []}
                for rnd in range(2):
                    for name, fn in ((("ours", ours), ("torch", ref)) if rnd == 0 else (("torch", ref), ("ours", ours))):
                        t[name].append(batch_ms(fn, n))
                out.append((M, N, K, min(t["ours"]) * 1e3, min(t["torch"]) * 1e3))
                plan.close()
    return out


def skinny_report(ctx, torch, hgemm, inputs, stream) -> dict:
    """The memory-bound LLM-projection shapes, M in {64, 128, 256} tokens x (N, K) in {(4096, 4096), (12288, 4096),
    (4096, 12288)}, entries N(0, 1) * K^-1/2: achieved GB/s of compulsory traffic against the HBM roofline, with B
    (the weight matrix) rotated through enough copies that it never comes from L2, torch.matmul beside it."""
    peaks = measured_peaks()
    base = inputs.draw(3, inputs.TAG_B, 4096, 4096, "normal", "cpu").cuda()          # N(0,1) / sqrt(4096)
    out = []

    def batch_ms(fn, n):
        e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        e0.record(stream)
        for i in range(n):
            fn(i)
        e1.record(stream)
        e1.synchronize()
        return e0.elapsed_time(e1) / n

    for (N, K) in ((4096, 4096), (12288, 4096), (4096, 12288)):
        scale = (4096.0 / K) ** 0.5
        tile = (base.float() * scale).half()
        B0 = tile.repeat(N // 4096, K // 4096).contiguous()
        copies = max(2, math.ceil(2 * L2_BYTES / (2.0 * N * K)) + 1)
        Bs = [B0] + [B0.clone() for _ in range(copies - 1)]
        for M in (64, 128, 256):
            A = (base[:M].float() * scale).half().repeat(1, K // 4096).contiguous()
            C = torch.empty(M, N, dtype=torch.float16, device="cuda")
            plan = ctx.plan(M, N, K)
            a, c, s = A.data_ptr(), C.data_ptr(), stream.cuda_stream
            ours = lambda i: plan.run_ptr(a, Bs[i % copies].data_ptr(), c, s)       # noqa: E731
            ref = lambda i: torch.matmul(A, Bs[i % copies].T, out=C)                # noqa: E731
            for fn in (ours, ref):
                batch_ms(fn, copies)
            n = 8 * copies
            to = statistics.median(batch_ms(ours, n) for _ in range(3))
            tt = statistics.median(batch_ms(ref, n) for _ in range(3))
            # the same with the weights declared static (hgemm_plan_set_static_operands): their first loads leave before the
            # previous call has finished -- a promise the rotating copies of B keep, and one torch.matmul has no way to take
            plan.set_static_operands(b=True)
            batch_ms(ours, copies)
            ts = statistics.median(batch_ms(ours, n) for _ in range(3))
            plan.set_static_operands()
            by = compulsory_bytes(M, N, K)
            out.append({"shape": [M, N, K], "us": to * 1e3, "gbs": by / (to * 1e-3) / 1e9,
                        "frac_of_measured_hbm": by / (to * 1e-3) / 1e9 / peaks["hbm_gbs"],
                        "frac_of_spec_hbm": by / (to * 1e-3) / 1e9 / SPEC_HBM_GBS, "torch_us": tt * 1e3,
                        "torch_time_over_ours": tt / to, "us_static_weights": ts * 1e3,
                        "frac_of_measured_hbm_static_weights": by / (ts * 1e-3) / 1e9 / peaks["hbm_gbs"],
                        "config": plan.config.as_dict()})
            plan.close()
        del Bs, B0
    return {"regime": "B rotates through copies totalling more than 2x L2 (cold weights), A and C stay hot",
            "inputs": "N(0,1) * K^-1/2 rounded to fp16", "shapes": out,
            "per_shape_frac_of_measured_hbm": {"x".join(map(str, r["shape"])): round(r["frac_of_measured_hbm"], 4) for r in out},
            "per_shape_torch_time_over_ours": {"x".join(map(str, r["shape"])): round(r["torch_time_over_ours"], 4) for r in out},
            "per_shape_frac_static_weights": {"x".join(map(str, r["shape"])): round(r["frac_of_measured_hbm_static_weights"], 4) for r in out},
            "geomean_frac_of_measured_hbm_static_weights": math.exp(sum(math.log(r["frac_of_measured_hbm_static_weights"]) for r in out) / len(out)),
            "geomean_frac_of_measured_hbm": math.exp(sum(math.log(r["frac_of_measured_hbm"]) for r in out) / len(out)),
            "geomean_torch_time_over_ours": math.exp(sum(math.log(r["torch_time_over_ours"]) for r in out) / len(out))}


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--gpus", type=int, default=1)
    ap.add_argument("--steps", type=int, default=1000)
    ap.add_argument("--warmup", type=int, default=5)
    ap.add_argument("--impl", choices=["ours", "reference"], default="ours")
    ap.add_argument("--no-grid", action="store_true", help="skip everything but the timed sweep, torch.matmul beside it and the end-to-end leg")
    ap.add_argument("--grid-csv", metavar="PATH", help="also write the grid's per-shape times to this CSV file")
    ap.add_argument("--detail", metavar="PATH", help="write the long per-shape arrays of the grid and the projections to this JSON file")
    args = ap.parse_args()
    if args.warmup < 3 and args.impl == "ours":
        args.warmup = 3
    if args.impl == "reference":
        run_reference(args)
    else:
        run_ours(args)


if __name__ == "__main__":
    main()
