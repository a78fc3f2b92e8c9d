#!/usr/bin/env python3
"""Benchmark of carry-through-protected CNN inference on one or more GPUs.

One step = one batch through the whole inference path on each GPU:
carry-through convolutions, FC layers with the checksum neurons, per-image
verification, and re-execution of the flagged images (fault-free run: the
flagged images are the false alarms of the distribution-based threshold,
alpha = 1%).  The headline runs the K timed batches through one
ct_infer_batches call, which re-executes each batch's flagged images as
extra rows of the inference two batches later (the last two batches' at the
end of the call); the same steps with a separate re-run per batch
(ct_infer + ct_reexecute) are reported beside it.  The same model built
without carry-through filters gives the unprotected throughput and the
overhead.  The end-to-end figure runs the same batches from pinned host
memory through ct_run_host_batches (copies in and out inside the call,
overlapped with the inferences).

Prints ONE JSON line (rank 0).  Multi-GPU (torchrun): independent replicas,
each rank runs its own batch; only the barrier and the max-over-ranks timing
use a collective.

  python bench.py [--workload NAME] [--steps K] [--warmup W] [--gpus N]
  python bench.py --impl reference ...   # the CPU oracle on a bounded sample
"""
from __future__ import annotations

import argparse
import glob
import hashlib
import json
import re
import os
import statistics
import subprocess
import sys
import threading
import time

import numpy as np

ROOT = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, ROOT)

import synth  # noqa: E402
from paper_2609_16742_gb300 import replicas  # noqa: E402

METRIC = "protected images/sec and checksum overhead % vs unprotected; conv % of GB300 peak"
DEFAULT_WORKLOAD = "resnet18_imagenet"
# images a batch may carry for the previous batch's re-execution (more go
# through the synchronous path inside ct_infer_reexec)
REEXEC_ROOM = 32
# bounded oracle samples (images) per workload: roughly 10-30 s of CPU work
ORACLE_SAMPLE = {"lenet5": 4096, "resnet18_cifar": 512, "campaign_resnet18_cifar": 512,
                 "resnet18_imagenet": 256, "vgg16": 32}


def peaks():
    p = os.path.join(ROOT, "MEASURED_PEAKS.json")
    if os.path.exists(p):
        return json.load(open(p)), "measured"
    return {"hbm_gbs": 6800.0, "bf16_tflops": 1900.0, "bf16_tflops_sustained": 1700.0,
            "sm_max_mhz": 2070.0}, "fallback"


class ClockSampler:
    """nvidia-smi clocks and throttle reasons, sampled during the timed region."""

    Q = ("index,clocks.sm,clocks.max.sm,power.draw,clocks_event_reasons.active,"
         "clocks_event_reasons.hw_slowdown,clocks_event_reasons.hw_thermal_slowdown,"
         "clocks_event_reasons.sw_thermal_slowdown,clocks_event_reasons.sw_power_cap")

    def __init__(self, index: int):
        self.index = index
        self.rows = []
        self.proc = None

    def start(self):
        try:
            self.proc = subprocess.Popen(
                ["nvidia-smi", "-i", str(self.index), "--query-gpu=" + self.Q,
                 "--format=csv,noheader,nounits", "-lms", "200"],
                stdout=subprocess.PIPE, stderr=subprocess.DEVNULL, text=True)
            self.t = threading.Thread(target=self._read, daemon=True)
            self.t.start()
        except Exception:
            self.proc = None

    def _read(self):
        for line in self.proc.stdout:
            self.rows.append([c.strip() for c in line.split(",")])

    def stop(self):
        if self.proc is None:
            return {"sm_mhz": None, "sm_max_mhz": None, "reasons": ["nvidia-smi unavailable"]}
        time.sleep(0.25)
        self.proc.terminate()
        try:
            self.proc.wait(timeout=5)
        except Exception:
            self.proc.kill()
        ok = [r for r in self.rows if len(r) >= 9]
        sm = [float(r[1]) for r in ok if r[1].replace(".", "").isdigit()]
        mx = [float(r[2]) for r in ok if r[2].replace(".", "").isdigit()]
        names = ["hw_slowdown", "hw_thermal_slowdown", "sw_thermal_slowdown", "sw_power_cap"]
        reasons = set()
        for r in ok:
            for nm, v in zip(names, r[5:9]):
                if v.strip().lower() in ("active", "1"):
                    reasons.add(nm)
        return {"sm_mhz": statistics.median(sm) if sm else None,
                "sm_max_mhz": max(mx) if mx else None, "reasons": sorted(reasons),
                "samples": len(sm)}


def conv_flops(wl) -> float:
    sh = synth.shapes(wl.layers, wl.in_shape)
    f = 0.0
    for L in wl.layers:
        if L.op == "conv":
            _, P, Q = sh[L.dst]
            f += 2.0 * P * Q * L.cout * (L.cin // L.groups) * L.k * L.k
    return f * wl.batch


def oracle_rate(wl, n_img: int):
    """Oracle images/s on n_img images of the workload (CPU, as it stands)."""
    import oracle
    net = oracle.build_workload(wl)
    x = synth.make_input(wl, batch=n_img)
    t = time.perf_counter()
    oracle.forward(net, x)
    dt = time.perf_counter() - t
    return n_img / dt, oracle.get_threads(), dt


def run_reference(args, wl, rank, world):
    """--impl reference: the CPU oracle, timed on bounded samples of the workload."""
    if rank != 0:
        return
    import oracle
    n = max(1, ORACLE_SAMPLE.get(wl.name, 4) // max(1, args.steps))
    net = oracle.build_workload(wl)
    x = synth.make_input(wl, batch=n)
    for _ in range(min(args.warmup, 1)):
        oracle.forward(net, x[:1])
    times = []
    for _ in range(args.steps):
        t = time.perf_counter()
        oracle.forward(net, x)
        times.append(time.perf_counter() - t)
    total = sum(times)
    v = n * args.steps / total
    line = {"impl": "reference", "metric": METRIC, "value": v, "unit": "images/s",
            "n_gpus": world, "steps": args.steps, "warmup": args.warmup,
            "ms_per_step": 1e3 * total / args.steps, "higher_is_better": True,
            "scaling": "weak", "vs_baseline": None,
            "dtype": "f16" if wl.precision == "fp16" else "f32",
            "data": "synthetic", "config": {"workload": wl.name, "batch": n,
                                            "precision": wl.precision},
            "cpu_baseline": {"value": v, "unit": "images/s", "cores": oracle.get_threads(),
                             "kind": "oracle",
                             "sample": "%d steps x %d images of %s" % (args.steps, n, wl.name)},
            "e2e": {"value": v, "unit": "images/s", "h2d_bytes_per_step": 0,
                    "d2h_bytes_per_step": 0}}
    print(json.dumps(line), flush=True)


# sources of the operators that stand beside the networks: no inference launches one of their kernels
OPERATOR_SOURCES = ("fp8_matmul.cu", "fp8_quantize.cu", "fp8_quantize.cuh", "logprobs.cu", "ops.cu", "ops_common.cuh", "adapters.cu", "adapters.cuh",
                    "adapters_expand.cu", "adapters_outer.cu", "adapters_shrink.cu", "adapters_tc.cu", "clip.cu", "verify.cu")


def source_fingerprint(csrc=os.path.join(ROOT, "paper_2609_16742_gb300", "csrc")):
    """Hash of the CUDA sources of the networks' kernels; ties recorded counters to the kernels they measured."""
    h = hashlib.sha1()
    for f in sorted(glob.glob(os.path.join(csrc, "*"))):
        if f.endswith((".cu", ".cuh", ".h")) and os.path.basename(f) not in OPERATOR_SOURCES:
            with open(f, "rb") as fh:
                h.update(fh.read())
    return h.hexdigest()[:12]


def recorded_traffic(workload, batch):
    """DRAM bytes per launch of the tensor-core conv family from the committed
    ncu summary of this workload, or None when the kernels changed since."""
    path = os.path.join(ROOT, "profiles", "dram_traffic_%s_b%d.md" % (workload, batch))
    if not os.path.exists(path):
        return None, None
    txt = open(path).read()
    fp = re.search(r"source fingerprint: (\w+)", txt)
    val = re.search(r"tensor-core conv family: \d+ launches, DRAM bytes per launch: (\d+)", txt)
    if not fp or not val or fp.group(1) != source_fingerprint():
        return None, os.path.relpath(path, ROOT) + " (kernels changed since the capture)"
    return int(val.group(1)), os.path.relpath(path, ROOT)


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--gpus", type=int, default=1)
    ap.add_argument("--steps", type=int, default=100)
    ap.add_argument("--warmup", type=int, default=5)
    ap.add_argument("--impl", default="ours", choices=["ours", "reference"])
    ap.add_argument("--workload", default=DEFAULT_WORKLOAD, choices=sorted(synth.WORKLOADS))
    ap.add_argument("--simt-only", action="store_true")
    ap.add_argument("--no-cpu-baseline", action="store_true")
    ap.add_argument("--campaign-faults", type=int, default=1000,
                    help="faults per precision of the fault-injection campaign (0: skip)")
    args = ap.parse_args()

    rank = int(os.environ.get("RANK", "0"))
    world = int(os.environ.get("WORLD_SIZE", "1"))
    local = int(os.environ.get("LOCAL_RANK", "0"))
    wl = synth.workload(args.workload)

    if args.impl == "reference":
        run_reference(args, wl, rank, world)
        return

    import torch
    torch.cuda.set_device(local)
    dist = None
    if world > 1:
        import torch.distributed as dist
        dist.init_process_group("nccl")

    from paper_2609_16742_gb300 import build as _build
    if rank == 0:
        _build.build()
    if dist is not None:
        dist.barrier()
    import paper_2609_16742_gb300 as ct

    B = wl.batch
    params = synth.make_params(wl.layers, wl.seed)
    # room for the previous batch's flagged images riding along (deferred re-execution)
    mp = ct.ct_build_workload(wl, params, device=local, simt_only=args.simt_only, max_batch=B + REEXEC_ROOM)
    mu = ct.ct_build_workload(wl, params, device=local, simt_only=args.simt_only, protect=False)
    # the paper's prune-and-replace construction of the same network (not
    # built for networks with depthwise convolutions)
    try:
        mr = ct.ct_build_workload(wl, params, device=local, simt_only=args.simt_only, replace=True,
                                  max_batch=B + REEXEC_ROOM)
    except ct.CtError as e:
        if e.status != 6:                       # CT_EUNSUPPORTED
            raise
        mr = None

    # calibration (Sec. II-C, distribution-based, alpha = 1%) on seeded fault-free
    # images: 8 batches, because the 99th percentile of |S - r| taken from 2
    # (512 images) came out ~10% low, which doubled the false alarms
    calib_n = 8 * B
    xc = torch.from_numpy(synth.make_input(wl, batch=calib_n, seed=wl.calib_seed)).cuda()
    Sc = torch.empty(calib_n, device="cuda")
    lc = torch.empty(B, wl.n_classes, device="cuda")

    def calibrate(model):
        for i in range(0, calib_n, B):
            ct.ct_infer(model, xc[i:i + B], B, lc, Sc[i:i + B], None)
        torch.cuda.synchronize()
        rr, tt = ct.ct_calibrate(Sc.cpu().numpy(), 0.01)
        ct.ct_set_threshold(model, rr, tt)
        return rr, tt

    r, tau = calibrate(mp)
    r_rep, tau_rep = calibrate(mr) if mr is not None else (None, None)
    del xc
    # every re-execution graph is captured before anything is timed
    for model_ in (mp, mr):
        if model_ is not None:
            ct.ct_reexecute_prepare(model_, B + REEXEC_ROOM)

    # evaluation batches for this rank (distinct slices of the seeded set per
    # rank); two, alternating, so that each step's re-run images come from
    # the batch before it
    x_hosts = [synth.make_input(wl, batch=B, first=f) for f in replicas.input_slices(rank, B)]
    x_host = x_hosts[0]
    bufs = [{"x": torch.from_numpy(xh_).cuda(), "lg": torch.empty(B, wl.n_classes, device="cuda"),
             "S": torch.empty(B, device="cuda"), "fl": torch.empty(B, dtype=torch.uint8, device="cuda")}
            for xh_ in x_hosts]
    x, logits, S, flag = bufs[0]["x"], bufs[0]["lg"], bufs[0]["S"], bufs[0]["fl"]
    stream = torch.cuda.current_stream()

    def step_protected():
        # synchronous re-execution of this batch's flagged images (own small batch)
        ct.ct_infer(mp, x, B, logits, S, flag, stream)
        return ct.ct_reexecute(mp, x, B, flag, logits, S, stream)

    # outputs of the batch-list calls: four rotating sets (a batch's re-run rows
    # are written two batches after it)
    outs = [{"lg": torch.empty(B, wl.n_classes, device="cuda"), "S": torch.empty(B, device="cuda"),
             "fl": torch.empty(B, dtype=torch.uint8, device="cuda")} for _ in range(4)]

    def deferred_steps(steps, model=None):
        """`steps` protected steps in one ct_infer_batches call: each batch's
        flagged images are re-executed as extra rows of the inference two
        batches later, the last two batches' at the end of the call."""
        model = model or mp
        xs = [bufs[i % 2]["x"] for i in range(steps)]
        return ct.ct_infer_batches(model, xs, B, [outs[i % 4]["lg"] for i in range(steps)],
                                   [outs[i % 4]["S"] for i in range(steps)],
                                   [outs[i % 4]["fl"] for i in range(steps)], stream)

    def step_unprotected():
        ct.ct_infer(mu, x, B, logits, None, None, stream)
        return 0

    def barrier():
        if dist is not None:
            dist.barrier()
        torch.cuda.synchronize()

    def timed(fn, steps, loop=False):
        barrier()
        e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        e0.record(stream)
        n_re = 0
        if loop:
            n_re = fn(steps)
        else:
            for _ in range(steps):
                n_re += fn()
        e1.record(stream)
        barrier()
        ms = replicas.reduce_max(e0.elapsed_time(e1), dist, "cuda")
        return ms, n_re

    for _ in range(max(args.warmup, 3)):
        step_protected()
        step_unprotected()
    deferred_steps(max(args.warmup, 3))
    if mr is not None:
        deferred_steps(max(args.warmup, 3), mr)
    torch.cuda.synchronize()

    # unprotected reference (same kernels, no carry-through filters)
    ms_u, _ = timed(step_unprotected, args.steps)

    # protected inference alone (no re-execution): the cost of the filters
    def step_protected_infer():
        ct.ct_infer(mp, x, B, logits, S, flag, stream)
        return 0
    ms_pi, _ = timed(step_protected_infer, args.steps)

    # protected, timed (the headline), with clocks sampled; the library counts
    # the kernels it launches, graph-replayed re-executions included
    clk = ClockSampler(local if "CUDA_VISIBLE_DEVICES" not in os.environ else
                       int(os.environ["CUDA_VISIBLE_DEVICES"].split(",")[local]))
    ct.ct_kernel_count(mp)
    clk.start()
    ms_p, n_rerun = timed(deferred_steps, args.steps, loop=True)
    clocks = clk.stop()
    launches = ct.ct_kernel_count(mp)

    # synchronous re-execution (each batch's flagged images as their own
    # small batch, replayed from a CUDA graph), for comparison
    ms_ps, n_rerun_s = timed(step_protected, args.steps)

    # the paper's prune-and-replace construction: same steps, and its
    # inference alone
    replace_leg = None
    if mr is not None:
        ms_r, n_rerun_r = timed(lambda k: deferred_steps(k, mr), args.steps, loop=True)

        def step_replace_infer():
            ct.ct_infer(mr, x, B, logits, S, flag, stream)
            return 0
        ms_ri, _ = timed(step_replace_infer, args.steps)
        replace_leg = {
            "what": "Sec. II-A prune-and-replace (ct_build CT_PROTECT_REPLACE): the least important channel of "
                    "every tensor gives its place to the carry-through filter; no fine-tuning",
            "value": replicas.job_throughput(world, B, args.steps, ms_r / 1e3), "unit": "images/s",
            "overhead_pct": 100.0 * (ms_r / ms_u - 1.0),
            "overhead_filters_pct": 100.0 * (ms_ri / ms_u - 1.0),
            "reexecuted_images_per_step": n_rerun_r / args.steps,
            "threshold": {"reference": r_rep, "tau": tau_rep},
            "device_error": ct.ct_device_error(mr)}

    # the headline steps again with CUDA events around every kernel on the
    # launch stream: per-family launches, device time and FLOPs for the roofline
    ct.ct_profile_enable(mp, True)
    for fam in range(5):
        ct.ct_profile_read(mp, fam)
    ms_prof, _ = timed(deferred_steps, args.steps, loop=True)
    ct.ct_profile_enable(mp, False)
    fam_stats = {fam: ct.ct_profile_read(mp, fam) for fam in range(5)}
    err = ct.ct_device_error(mp)

    def max_over_ranks(v):
        return replicas.reduce_max(v, dist, "cuda")

    # end to end through the public API from pinned host memory: one
    # ct_run_host_batches call over the K batches copies each batch in on the
    # library's copy stream while earlier batches run, and copies each
    # batch's logits, S and flags out once its re-run rows are final
    xh2 = [torch.from_numpy(xh_).pin_memory() for xh_ in x_hosts]
    hout = [{"lg": torch.empty(B, wl.n_classes, dtype=torch.float32).pin_memory(),
             "S": torch.empty(B, dtype=torch.float32).pin_memory(),
             "fl": torch.empty(B, dtype=torch.uint8).pin_memory()} for _ in range(4)]

    def e2e_steps(steps):
        return ct.ct_run_host_batches(mp, [xh2[i % 2] for i in range(steps)], B,
                                      [hout[i % 4]["lg"] for i in range(steps)],
                                      [hout[i % 4]["S"] for i in range(steps)],
                                      [hout[i % 4]["fl"] for i in range(steps)], stream)

    e2e_steps(3)
    barrier()
    t0 = time.perf_counter()
    e2e_steps(args.steps)
    barrier()
    e2e_s = max_over_ranks(time.perf_counter() - t0)
    # what the host link gives one batch's input alone (pinned host -> device)
    xd_probe = torch.empty_like(bufs[0]["x"])
    ev0, ev1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    ev0.record(stream)
    for _ in range(5):
        xd_probe.copy_(xh2[0], non_blocking=True)
    ev1.record(stream)
    torch.cuda.synchronize()
    h2d_gbs = 5 * xh2[0].numel() * 4 / (ev0.elapsed_time(ev1) / 1e3) / 1e9
    del xd_probe

    # the same through the host-buffer entry point ct_run_host (H2D, infer,
    # synchronous re-execution, D2H inside the call)
    xh = torch.from_numpy(x_host).pin_memory()
    lh = torch.empty(B, wl.n_classes, dtype=torch.float32).pin_memory()
    sh = torch.empty(B, dtype=torch.float32).pin_memory()
    fh = torch.empty(B, dtype=torch.uint8).pin_memory()
    xn, ln, sn, fn_ = xh.numpy(), lh.numpy(), sh.numpy(), fh.numpy()
    for _ in range(2):
        ct.ct_run_host(mp, xn, ln, sn, fn_, stream)
    barrier()
    t0 = time.perf_counter()
    for _ in range(args.steps):
        ct.ct_run_host(mp, xn, ln, sn, fn_, stream)
    barrier()
    e2e_sync_s = max_over_ranks(time.perf_counter() - t0)

    if rank != 0:
        if dist is not None:
            dist.destroy_process_group()
        return

    pk, pk_kind = peaks()
    value = replicas.job_throughput(world, B, args.steps, ms_p / 1e3)
    value_u = replicas.job_throughput(world, B, args.steps, ms_u / 1e3)
    props = torch.cuda.get_device_properties(local)
    # dominant kernel: the convolution family that carries the FLOPs
    tc_n, tc_ms, tc_fl = fam_stats[0]
    si_n, si_ms, si_fl = fam_stats[1]
    if tc_ms >= si_ms and tc_n:
        roof = {"kernel": "tcgen05 convolution family: stem_pool, conv_tc_halo, conv_tc, conv_tc_pair "
                          "(fp16 in / fp32 acc)", "bound": "tensor",
                "achieved": tc_fl / (tc_ms / 1e3) / 1e12, "peak": pk["bf16_tflops"],
                "unit": "TFLOP/s",
                "peak_source": "%s bf16 dense burst; fp16 has the bf16 rate" % pk_kind,
                "launches": tc_n, "avg_launch_us": 1e3 * tc_ms / tc_n,
                "flops_per_launch": tc_fl / tc_n}
    else:
        clock = pk.get("sm_max_mhz", 2070.0) * 1e6
        peak = props.multi_processor_count * 128 * 2 * clock / 1e12
        roof = {"kernel": "conv_simt_kernel (FFMA)", "bound": "alu",
                "achieved": si_fl / (si_ms / 1e3) / 1e12 if si_ms else 0.0,
                "peak": peak, "unit": "TFLOP/s",
                "peak_source": "%d SMs x 128 FFMA/clk x 2 flop x %.0f MHz (%s max SM clock)"
                               % (props.multi_processor_count, clock / 1e6, pk_kind),
                "launches": si_n, "avg_launch_us": 1e3 * si_ms / max(si_n, 1),
                "flops_per_launch": si_fl / max(si_n, 1)}
    roof["frac"] = roof["achieved"] / roof["peak"]
    roof["traffic"], roof["traffic_source"] = recorded_traffic(wl.name, B)
    roof["conv_share_of_step"] = (tc_ms + si_ms) / ms_p if ms_p else None

    cpu = None
    if not args.no_cpu_baseline:
        n_img = ORACLE_SAMPLE.get(wl.name, 4)
        v, cores, dt = oracle_rate(wl, n_img)
        cpu = {"value": v, "unit": "images/s", "cores": cores, "kind": "oracle",
               "sample": "%d images of %s, one forward pass (%.1f s)" % (n_img, wl.name, dt)}

    # fault-injection campaign on the CIFAR ResNet-18 (FP32 and FP16): detected
    # fraction of critical faults and end-to-end time including re-execution
    camp = None
    if args.campaign_faults > 0:
        from paper_2609_16742_gb300 import campaign
        camp = {}
        for prec in ("fp32", "fp16"):
            c = campaign.run(prec, args.campaign_faults, seed=0, device=local)
            camp[prec] = {"faults": c["faults"], "batch": c["batch"],
                          "detected_fraction_of_critical": c["all"]["detected_fraction_of_critical"],
                          "critical": c["all"]["critical"], "trials": c["all"]["trials"],
                          "false_alarm_rate": c["all"]["false_alarm_rate"],
                          "weights": c["weights"]["detected_fraction_of_critical"],
                          "activations": c["activations"]["detected_fraction_of_critical"],
                          "wall_s": c["wall_s"], "time_relative_to_fault_free": c["time_relative_to_fault_free"],
                          "reexecuted_images": c["reexecuted_images"], "device_error": c["device_error"]}
        # LeNet-5 (FP32): 100,000 faults in one launch of the batched campaign kernel
        cb = campaign.run_batched(faults=100 * args.campaign_faults, seed=0, device=local)
        camp["lenet5_batched"] = {"faults": cb["faults"], "batch": cb["batch"], "wall_s": cb["wall_s"],
                                  "faults_per_s": cb["faults_per_s"],
                                  "detected_fraction_of_critical": cb["all"]["detected_fraction_of_critical"],
                                  "critical": cb["all"]["critical"], "trials": cb["all"]["trials"],
                                  "false_alarm_rate": cb["all"]["false_alarm_rate"],
                                  "device_error": cb["device_error"]}

    in_bytes = B * int(np.prod(wl.in_shape)) * 4
    out_bytes = B * (wl.n_classes * 4 + 4 + 1)
    line = {
        "metric": METRIC, "value": value, "unit": "images/s", "n_gpus": world,
        "steps": args.steps, "warmup": max(args.warmup, 3), "ms_per_step": ms_p / args.steps,
        "higher_is_better": True, "scaling": "weak", "vs_baseline": None,
        "dtype": "f16" if wl.precision == "fp16" else "f32", "data": "synthetic",
        "config": {"workload": wl.name, "batch_per_gpu": B, "in_shape": list(wl.in_shape),
                   "precision": wl.precision + (" storage, fp32 accumulate"
                                                if wl.precision == "fp16" else ""),
                   "parallelism": "replicas x%d" % world, "alpha": 0.01,
                   "l2": "inputs and activations larger than L2 (no flush)",
                   "simt_only": bool(args.simt_only)},
        "reexecution": "deferred by two batches (ct_infer_batches): each batch's flagged images ride as extra "
                       "rows of the inference two batches later; the last two batches' are re-run at the end of "
                       "the call, inside the timed region",
        "value_sync_reexec": replicas.job_throughput(world, B, args.steps, ms_ps / 1e3),
        "overhead_reexec_sync_pct": 100.0 * (ms_ps - ms_pi) / ms_u,
        "reexecuted_images_per_step_sync": n_rerun_s / args.steps,
        "replace_construction": replace_leg,
        "conv_tflop_per_batch": conv_flops(wl) / 1e12,
        "roofline": roof,
        "cpu_baseline": cpu,
        "e2e": {"value": replicas.job_throughput(world, B, args.steps, e2e_s), "unit": "images/s",
                "h2d_bytes_per_step": in_bytes, "d2h_bytes_per_step": out_bytes,
                "api": "ct_run_host_batches: one call over the K batches from pinned host memory, copies in "
                       "and out overlapped with the inferences, deferred re-execution",
                "h2d_gbs_alone": h2d_gbs,
                "h2d_bound_images_per_s": h2d_gbs * 1e9 / (in_bytes / B) * world},
        "e2e_sync_reexec": {"value": replicas.job_throughput(world, B, args.steps, e2e_sync_s), "unit": "images/s",
                            "api": "ct_run_host (host buffers, synchronous re-execution)"},
        "kernel_families": {nm: {"launches": fam_stats[i][0], "ms": fam_stats[i][1],
                                 "tflop": fam_stats[i][2] / 1e12}
                            for i, nm in enumerate(["conv_tc", "conv_simt", "fc", "pool", "other"])},
        "gpu_launches": launches,
        "ms_per_step_with_kernel_events": ms_prof / args.steps,
        "clocks": clocks,
        "device_error": err,
        "threshold": {"reference": r, "tau": tau},
        "campaign": camp,
    }
    # the headline figures last, so that a truncated tail of the line keeps them
    line["reexecuted_images_per_step"] = n_rerun / args.steps
    line["roofline_frac"] = roof["frac"]
    line["unprotected_value"] = value_u
    line["overhead_reexec_pct"] = 100.0 * (ms_p - ms_pi) / ms_u
    line["overhead_filters_pct"] = 100.0 * (ms_pi / ms_u - 1.0)
    line["overhead_pct"] = 100.0 * (ms_p / ms_u - 1.0)
    line["value_images_per_s"] = value
    print(json.dumps(line), flush=True)
    if dist is not None:
        dist.destroy_process_group()


if __name__ == "__main__":
    main()
