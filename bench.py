"""Benchmark of the QuantEase hot path on one MI355X.

One step = one layer of the 4096 x 4096 attention-projection workload, 4-bit,
inputs resident in HBM:  Sigma = X X^T + 0.01 mean(diag) I over 128 x 2048
heavy-tailed tokens -> per-row grid -> 10 CD sweeps (objective after each)
-> exact objective.  value = CD column updates per second of sweep time
(p x 10 / the 10 sweeps' time, HIP events); the whole step's rate is
layer_column_updates_per_s.  The headline roofline is the CD step kernel
(the block-update GEMM with the next panel), the Gram's is under
"rooflines"; each counts the method's own flops (2qp^2 per sweep,
p(p+1)n per Gram) against the peak of the matrix-core type the kernels
issue (bf16: the fp32 products are exact three-way bf16 splits, and once
the codes are valid the block update multiplies integer code differences,
exact in one bf16 plane, by Sigma's three planes).  The
outlier-aware path (3-bit, 1% outliers: lambda_max, P_s(W), outlier grid, 10
CD + IHT iterations) is timed in the same run under "outlier"; the CPU
oracle is timed under "cpu_baseline" (all sweeps on every row; its Gram on a
token sample, scaled).

    python bench.py [--gpus 1] [--steps K] [--warmup W]
"""
import argparse
import json
import os
import re
import sys
import time

import numpy as np

ROOT = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, ROOT)

METRIC = "CD sweep time per layer (s) and column-updates/s at 4096×4096 4-bit"
HBM_PEAK_GBS = 8000.0
FP32_MFMA_PEAK_TFLOPS = 157.3
BF16_MFMA_PEAK_TFLOPS = 2500.0
FP16_MFMA_PEAK_TFLOPS = 2500.0
GRAM_PRODUCTS = 3              # fp16 products per fp32 product (two-way split of scaled channels)
INT_DELTA_PRODUCTS = 3         # integer code difference x three bf16 planes of Sigma
TRAFFIC_PROFILE = os.path.join(ROOT, "profiles", "hbm_traffic_c2_4096x4096.md")
LAUNCH_PROFILE = os.path.join(ROOT, "profiles", "kernel_trace_gram_cd_step_c2_4096x4096.md")
PARITY_RECORD = os.path.join(ROOT, "profiles", "parity_c2_4096x4096.md")
CONFIG_PROFILE = os.path.join(ROOT, "profiles", "cd_step_per_configuration.md")
CALIB_COPY_BYTES = 256 << 20


# HIP sources each measured kernel is compiled from
KERNEL_SOURCES = {
    "gram_x3w_kernel": ["gram.hip", "nt_f2.h", "nt_x3.h", "qe_internal.h"],
    "cd_step_kernel": ["cd.hip", "nt_x3.h", "qe_internal.h"],
}


def kernel_source_hash(kernel):
    """sha256 over the HIP sources `kernel` is compiled from and what they use of the ABI header: the
    macros whose names they contain.  (Declarations and comments of other calls change no kernel.)"""
    import hashlib
    h = hashlib.sha256()
    text = ""
    for name in KERNEL_SOURCES[kernel]:
        with open(os.path.join(ROOT, "paper_2309_01885_amd", "csrc", name), encoding="utf-8") as f:
            body = f.read()
        h.update((name + "\n" + body).encode())
        text += body
    with open(os.path.join(ROOT, "include", "qe.h"), encoding="utf-8") as f:
        header = re.sub(r"/\*.*?\*/", " ", f.read(), flags=re.S).replace("\\\n", " ")
    used = set(re.findall(r"\bQE_\w+", text))
    for name, rest in re.findall(r"^[ \t]*#define[ \t]+(\w+)(.*)$", header, re.M):
        if name in used:
            h.update(f"{name} {' '.join(rest.split())}\n".encode())
    return h.hexdigest()


def _json_block(path):
    try:
        with open(path) as f:
            text = f.read()
    except OSError:
        return None
    m = re.search(r"```json\n(.*?)\n```", text, re.S)
    return json.loads(m.group(1)) if m else None


def measured_traffic():
    """HBM bytes per launch from the committed FETCH_SIZE / WRITE_SIZE summary
    (copy-calibrated), keyed by kernel; a kernel is left out when its sources
    changed since the counters were taken."""
    data = _json_block(TRAFFIC_PROFILE)
    if not data:
        return {}
    return {k: v["hbm_bytes_per_launch"] for k, v in data["kernels"].items()
            if k in KERNEL_SOURCES and v.get("source_sha256") == kernel_source_hash(k)}


def profiled_panel_launch():
    """Mean duration of the panel-only launch (the first step launch of each
    sweep) from the committed kernel trace, or None when the step kernel's
    sources changed since the trace was taken."""
    data = _json_block(LAUNCH_PROFILE)
    if not data or data.get("source_sha256") != kernel_source_hash("cd_step_kernel"):
        return None
    return data


def parity_record():
    """CD parity figures of the c2 workload from the committed record of the
    GPU parity tests (teacher-forced and free-running, 512 seeded rows)."""
    return _json_block(PARITY_RECORD)


def log(msg):
    print(f"[bench] {msg}", file=sys.stderr, flush=True)


CPU_GRAM_TOKENS = 8192       # oracle Gram sample (about 2 s on 16 host threads)
CPU_SWEEP_ROWS = 1024        # oracle sweep sample with --oracle-sample
CPU_ONE_THREAD_ROWS = 64     # single-thread sweep sample

# Child process for the single-thread figure: OpenMP's thread count is fixed
# when the oracle library loads, so it runs in a fresh interpreter.
_ONE_THREAD = """
import sys, numpy as np
sys.path.insert(0, sys.argv[1])
import oracle
d = sys.argv[2]
a = {k: np.load(d + "/" + k + ".npy") for k in ("W", "S", "scale", "zero")}
print(oracle.num_threads(), oracle.cd_sweep_timed(a["W"], a["S"], int(sys.argv[3]), a["scale"],
                                                  a["zero"]))
"""


def cpu_model():
    try:
        for line in open("/proc/cpuinfo"):
            if line.startswith("model name"):
                return line.split(":", 1)[1].strip()
    except OSError:
        pass
    return "unknown"


def one_thread_sweep(S, W, scale, zero, bits):
    """Seconds of one oracle sweep over W's rows with one OpenMP thread."""
    import subprocess
    import tempfile
    with tempfile.TemporaryDirectory(dir="/tmp") as d:
        for k, v in (("W", W), ("S", S), ("scale", scale), ("zero", zero)):
            np.save(os.path.join(d, k + ".npy"), np.ascontiguousarray(v))
        env = dict(os.environ, OMP_NUM_THREADS="1")
        out = subprocess.run([sys.executable, "-c", _ONE_THREAD, ROOT, d, str(bits)], env=env,
                             capture_output=True, text=True, timeout=600, check=True).stdout
    threads, secs = out.split()
    assert int(threads) == 1, out
    return float(secs)


def cpu_baseline(spec, X_head, W, scale, zero, sweeps, full=False):
    """The oracle as it stands on the host cores, on a bounded sample of the
    same step: one CD sweep on r seeded rows, scaled by q/r rows (the cost is
    exactly linear in the rows, which are independent) -- or, with full, all
    sweeps on every row, unscaled -- and the Gram on the first n' tokens
    (scaled by n/n'); plus the sweep on fewer rows with a single thread.
    value: column updates per second of sweeping, as the GPU's value."""
    import oracle
    q, p, n = spec.q, spec.p, spec.n
    n_s = X_head.shape[1]
    t0 = time.perf_counter()
    S = oracle.damp(oracle.gram(X_head), spec.damp)
    t_gram = time.perf_counter() - t0
    if full:
        rows = np.arange(q)
        t_sweeps = oracle.cd_sweep_timed(W, S, spec.bits, scale, zero, sweeps)
        sweep_all = t_sweeps / sweeps
        how = f"all {sweeps} sweeps over all {q} rows (not scaled)"
        measured = t_sweeps
    else:
        rows = __import__("synth").row_sample(q, CPU_SWEEP_ROWS, spec.cfg)
        t_sweep = oracle.cd_sweep_timed(W[rows], S, spec.bits, scale[rows], zero[rows])
        sweep_all = t_sweep * (q / len(rows))
        how = f"one Lemma-1 sweep over {len(rows)} of {q} rows (x{q / len(rows):.0f} rows)"
        measured = t_sweep
    t_step = t_gram * (n / n_s) + sweep_all * sweeps
    r1 = rows[:CPU_ONE_THREAD_ROWS]
    t_one = one_thread_sweep(S, W[r1], scale[r1], zero[r1], spec.bits)
    return {
        "value": p / sweep_all,
        "unit": "column-updates/s",
        "cores": oracle.num_threads(),
        "cpu_model": cpu_model(),
        "kind": "oracle",
        "sample": (f"{how}, measured {measured:.2f} s; Gram over {n_s} of {n} tokens "
                   f"(x{n / n_s:.0f}), measured {t_gram:.2f} s"),
        "sweep_s": sweep_all,
        "layer_s": t_step,
        "layer_column_updates_per_s": p * sweeps / t_step,
        "one_thread_sweep": {"rows": len(r1), "seconds": t_one,
                             "coordinate_updates_per_s": len(r1) * p / t_one},
    }


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--gpus", type=int, default=1)
    ap.add_argument("--steps", type=int, default=10)
    ap.add_argument("--warmup", type=int, default=2)
    ap.add_argument("--no-cpu", action="store_true", help="skip the CPU oracle baseline")
    ap.add_argument("--no-outlier", action="store_true", help="skip the outlier-aware timing")
    ap.add_argument("--no-peaks", action="store_true",
                    help="skip the matrix-core / copy peak checks (libqe_peak.so)")
    ap.add_argument("--oracle-sample", action="store_true",
                    help="time one oracle sweep on a 1024-row sample (scaled) instead of all "
                         "sweeps on every row (about 20 s on 16 host threads)")
    ap.add_argument("--calib-copy", action="store_true",
                    help="end with a plain 256 MiB device copy (HBM counter calibration)")
    ap.add_argument("--configs", action="store_true",
                    help="instead of the c2 step: Gram and CD timings of every workload "
                         "configuration at its full size (one JSON line)")
    ap.add_argument("--no-configs", action="store_true",
                    help="leave the per-configuration report out of the line")
    args = ap.parse_args()
    if args.gpus != 1:
        print(f"bench.py runs on exactly one GPU: --gpus {args.gpus} is not supported "
              "(the CD sweep would shard by rows with no communication)",
              file=sys.stderr)
        sys.exit(2)

    import torch
    import paper_2309_01885_amd as P
    import synth

    if args.configs:
        print(json.dumps(configs_bench(P, torch, synth, with_oracle=not args.no_cpu)), flush=True)
        return

    assert torch.cuda.is_available(), "bench.py needs a GPU"
    dev = torch.device("cuda:0")
    spec = synth.CONFIGS["c2"]
    q, p, n, bits, sweeps = spec.q, spec.p, spec.n, spec.bits, spec.sweeps
    block = 128

    log(f"generating inputs: W {q}x{p}, X {p}x{n} (X drawn on the device, seeded)")
    W_h = synth.weights(spec)
    X = torch.empty((p, n), dtype=torch.float32, device=dev)
    chunk = 32768
    for c in range(n // chunk):
        X[:, c * chunk:(c + 1) * chunk] = synth.activation_chunk_device(spec, c, chunk, dev)
    X_head = X[:, :CPU_GRAM_TOKENS].cpu().numpy()          # the oracle's token sample
    W = torch.from_numpy(W_h).to(dev)
    Sigma = torch.empty((p, p), dtype=torch.float32, device=dev)
    Wh = torch.empty_like(W)
    codes = torch.empty((q, p), dtype=torch.uint8, device=dev)
    R = torch.empty_like(W)
    obj = torch.zeros(sweeps, dtype=torch.float64, device=dev)
    ws_gram = P.workspace(P.load().qe_gram_workspace_size(p, n), dev)
    ws_cd = P.workspace(P.cd_workspace_size(q, p, block), dev)
    ws_obj = P.workspace(P.load().qe_objective_workspace_size(q, p), dev)
    stream = torch.cuda.current_stream()

    ev = {k: [torch.cuda.Event(enable_timing=True) for _ in range(2)]
          for k in ("gram", "grid", "cd", "exact")}

    def step(timed=False):
        def mark(k, i):
            if timed:
                ev[k][i].record(stream)
        mark("gram", 0)
        P.gram(X, Sigma=Sigma, damp=spec.damp, ws=ws_gram, check=False)
        mark("gram", 1)
        mark("grid", 0)
        scale, zero = P.grid_minmax(W, bits)
        mark("grid", 1)
        mark("cd", 0)
        P.cd_sweep(W, Sigma, bits, scale, zero, Wh, codes, R, sweeps, block=block,
                   flags=P.QE_INIT_FROM_W, obj=obj, ws=ws_cd, check=False)
        mark("cd", 1)
        mark("exact", 0)
        out = P.objective(W, Wh, Sigma, ws=ws_obj, check=False)
        mark("exact", 1)
        return scale, zero, out

    log(f"warmup x{args.warmup}")
    for _ in range(args.warmup):
        step()
    torch.cuda.synchronize()
    for w in (ws_gram, ws_cd, ws_obj):
        st = P.sync_status(w)
        assert st == 0, f"device status {st}"

    log(f"timing x{args.steps}")
    phase = {k: [] for k in ev}
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    for _ in range(args.steps):
        scale, zero, exact = step(timed=True)
        torch.cuda.synchronize()
        for k in ev:
            phase[k].append(ev[k][0].elapsed_time(ev[k][1]) * 1e-3)
    torch.cuda.synchronize()
    wall = time.perf_counter() - t0
    for w in (ws_gram, ws_cd, ws_obj):
        st = P.sync_status(w)
        assert st == 0, f"device status {st}"
    ms_per_step = wall / args.steps * 1e3
    cd_phase_t = float(np.median(phase["cd"]))           # the 10 sweeps of a step
    value = p * sweeps / cd_phase_t                      # column updates per second of sweeping
    f_sweeps = obj.cpu().numpy()
    exact = exact.cpu().numpy()

    # ---- dominant kernels, measured live on this stream
    # block-update step kernel: sweeps resumed from a valid R, no objective,
    # so the region holds only the step launches (+2 tiny setup kernels);
    # every block update on the matrix cores (QE_CD_DENSE), so that the
    # roofline does not count the exact zeros the default path skips
    super_w = max(256, block)                     # columns per step launch (super-block)
    nb = (p + super_w - 1) // super_w

    def resumed_sweeps(extra):
        e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        e0.record(stream)
        P.cd_sweep(W, Sigma, bits, scale, zero, Wh, codes, R, sweeps, block=block,
                   flags=P.QE_R_VALID | P.QE_CODES_VALID | extra, obj=None, ws=ws_cd,
                   check=False)
        e1.record(stream)
        torch.cuda.synchronize()
        return e0.elapsed_time(e1) * 1e-3

    t_steps = resumed_sweeps(P.QE_CD_DENSE)
    # the same sweeps on the default path: past convergence almost no code
    # moves, and the sweeps run row by row, with a rank-1 update per move
    t_converged = resumed_sweeps(0) / sweeps
    # one sweep per call from W = What: events around each of sweeps 2..K
    # (with its objective, carried from call to call as inside the step's
    # multi-sweep call), median
    per_sweep = []
    for k in range(sweeps):
        if k > 0:
            obj[k].copy_(obj[k - 1])                     # the incoming objective
        a0, a1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a0.record(stream)
        P.cd_sweep(W, Sigma, bits, scale, zero, Wh, codes, R, 1, block=block,
                   flags=(P.QE_INIT_FROM_W if k == 0
                          else P.QE_R_VALID | P.QE_CODES_VALID | P.QE_OBJ_IN),
                   obj=obj[k:], ws=ws_cd, check=False)
        a1.record(stream)
        per_sweep.append((a0, a1))
    torch.cuda.synchronize()
    sweep_times_single = [a.elapsed_time(b) * 1e-3 for a, b in per_sweep]
    sweep_median_2_k = float(np.median(sweep_times_single[1:]))
    launches = sweeps * (nb + 1)
    cd_avg = t_steps / launches
    gram_t = float(np.median(phase["gram"]))
    sweep_t = cd_phase_t / sweeps
    traffic = measured_traffic()

    def roofline(kernel, flops, seconds, cores, products, issued, extra):
        """The method's own flops (fp32 multiply-adds x 2) per launch over the
        launch time, against the peak of the matrix-core type issued (`cores`:
        bf16 or fp16, both 2.5 PFLOP/s dense); the issue rate (`products`
        exact products of that type per fp32 product) and the fp32-equivalent
        fraction are separate fields."""
        peak = BF16_MFMA_PEAK_TFLOPS if cores == "bf16" else FP16_MFMA_PEAK_TFLOPS
        achieved = flops / seconds / 1e12
        r = {"kernel": kernel, "bound": "mfma", "achieved": achieved,
             "peak": peak, "unit": "TFLOP/s",
             "frac": achieved / peak,
             "traffic": traffic.get(kernel.split("<")[0]),
             "flops_per_launch": flops,
             "flops_counted": "the method's: fp32 products of the algorithm, 2 flops each",
             "issued": issued,
             "matrix_cores": cores,
             "products_per_fp32_product": products,
             "issued_tflops": products * achieved,
             "issued_frac_of_peak": products * achieved / peak,
             "fp32_equivalent_frac": achieved / FP32_MFMA_PEAK_TFLOPS,
             "frac_of_split_ceiling": achieved / (peak / products)}
        r.update(extra)
        return r

    # 2qp^2 per sweep over its nb + 1 launches; p(p+1)n for the Gram (symmetric half).
    # The resumed sweeps start from valid codes, so the block update multiplies
    # integer code differences (one exact bf16 plane) by Sigma's three planes.
    roof_cd = roofline("cd_step_kernel<8>", 2.0 * q * p * p / (nb + 1), cd_avg, "bf16",
                       INT_DELTA_PRODUCTS,
                       "bf16 matrix cores: integer code differences (exact in bf16) times "
                       "the three bf16 planes of Sigma, 3 products per fp32 product",
                       {"avg_launch_s": cd_avg, "launches_per_sweep": nb + 1})
    roof_gram = roofline("gram_x3w_kernel", float(p) * (p + 1) * n, gram_t, "fp16", GRAM_PRODUCTS,
                         "fp16 matrix cores: each channel scaled by a power of two and split "
                         "into two fp16 values, 3 exact fp16 products per fp32 product "
                         "(the call includes the pass that finds the scales)",
                         {"call_s": gram_t})

    # the Gram from token-major activations (n x p, as a model produces them),
    # in one call and streamed in 32768-token chunks accumulated into Sigma
    XT = X.t().contiguous()
    S_np = torch.empty_like(Sigma)
    ws_np = P.workspace(max(P.load().qe_gram_workspace_size(p, n),
                            P.load().qe_gram_workspace_size(p, 32768)), dev)
    tm = {}
    for label, chunk in (("one_call_s", n), ("chunks_32768_s", 32768)):
        times = []
        for rep in range(3):
            g0, g1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            g0.record(stream)
            for c0 in range(0, n, chunk):
                P.gram(XT[c0:c0 + chunk], layout=P.QE_LAYOUT_NP, Sigma=S_np, accumulate=c0 > 0,
                       damp=spec.damp if c0 + chunk >= n else 0.0, ws=ws_np, check=False)
            g1.record(stream)
            torch.cuda.synchronize()
            times.append(g0.elapsed_time(g1) * 1e-3)
        tm[label] = float(np.median(times))
    assert P.sync_status(ws_np) == 0
    del XT, S_np, ws_np
    torch.cuda.empty_cache()

    # the column-sequential panel: a panel-only launch (256 columns x q rows)
    # moves 17 bytes per coordinate (R, What in; What, code, delta out)
    panel = None
    prof = profiled_panel_launch()
    if prof:
        bytes_panel = 17.0 * q * super_w
        t_panel = prof["panel_only_launch_us"] * 1e-6
        panel = {"launch_s": t_panel, "algorithmic_bytes": bytes_panel,
                 "achieved_GBps": bytes_panel / t_panel / 1e9,
                 "frac_of_hbm_peak": bytes_panel / t_panel / 1e9 / HBM_PEAK_GBS,
                 "source": os.path.relpath(LAUNCH_PROFILE, ROOT) + " (rocprofv3 kernel trace)"}

    result = {
        "metric": METRIC,
        "value": value,
        "unit": "column-updates/s",
        "n_gpus": 1,
        "steps": args.steps,
        "warmup": args.warmup,
        "ms_per_step": ms_per_step,
        "higher_is_better": True,
        "scaling": "weak",
        "vs_baseline": None,
        "dtype": "f32 (matrix products: Gram fp16x2 split of power-of-two-scaled channels, "
                 "CD bf16x3 split; f32 accumulate)",
        "data": "synthetic",
        "config": {"workload": spec.name, "q": q, "p": p, "n": n, "bits": bits,
                   "sweeps": sweeps, "block": block, "damp": spec.damp},
        "roofline": roof_cd,
        "rooflines": [roof_cd, roof_gram],
        "panel": panel,
        "breakdown_s": {"gram": gram_t, "grid": float(np.median(phase["grid"])),
                        "cd_10_sweeps": cd_phase_t,
                        "exact_objective": float(np.median(phase["exact"]))},
        "sweep_time_s": sweep_t,
        "sweep_time_median_2_to_k_s": sweep_median_2_k,
        "sweep_times_single_calls_s": sweep_times_single,
        "sweep_time_converged_s": t_converged,
        "cd_column_updates_per_s": value,
        "cd_coordinate_updates_per_s": q * value,
        "layer_time_s": ms_per_step / 1e3,
        "layer_column_updates_per_s": p * sweeps / (wall / args.steps),
        "objective_per_sweep": [float(x) for x in f_sweeps],
        "rel_calibration_error": float(exact[0] / exact[1]),
        "parity": parity_record(),
        "gram_token_major": tm,
    }

    if not args.no_outlier:
        log("outlier-aware path")
        result["outlier"] = outlier_bench(P, torch, synth, W, Sigma, dev, block)

    if not args.no_peaks:
        log("peak checks")
        from paper_2309_01885_amd import peaks
        mp = peaks.measure(torch)
        result["measured_peaks"] = mp
        for r in result["rooflines"]:
            key = {"bf16": "mfma_bf16_tflops", "fp16": "mfma_f16_tflops"}[r["matrix_cores"]]
            r["issued_frac_of_measured_peak"] = r["issued_tflops"] / mp[key]

    if not args.no_cpu:
        log("CPU oracle baseline")
        result["cpu_baseline"] = cpu_baseline(spec, X_head, W_h, scale.cpu().numpy(),
                                              zero.cpu().numpy(), sweeps,
                                              full=not args.oracle_sample)
        result["gpu_over_oracle"] = value / result["cpu_baseline"]["value"]
    if not args.no_configs:
        log("every workload configuration at full size")
        del X, W, Sigma, Wh, R, codes
        torch.cuda.empty_cache()
        result["configs"] = configs_report(configs_bench(P, torch, synth,
                                                         with_oracle=not args.no_cpu))
    if args.calib_copy:
        a = torch.ones(CALIB_COPY_BYTES // 4, dtype=torch.float32, device=dev)
        b = torch.empty_like(a)
        b.copy_(a)
        torch.cuda.synchronize()
    print(json.dumps(result), flush=True)


# oracle row sample per configuration for the --configs report (rows; Gram tokens)
CONFIG_ORACLE = {"c1": (512, 2048), "c2": (256, 2048), "c3up": (256, 2048),
                 "c3down": (128, 1024), "c5": (32, 256)}


def configs_bench(P, torch, synth, with_oracle=True):
    """Every workload configuration at its full size: the Gram over all
    n = 262144 device-drawn tokens (one call when X fits comfortably, else
    token chunks accumulated into Sigma), damping, the per-row grid and the
    configured number of CD sweeps from What = W.  Times from HIP events on
    the library's stream (c1 timed on its second pass, after the code objects
    are loaded).  With the oracle: one Lemma-1 sweep over a seeded row sample
    on the host cores (Sigma from a token prefix of the same X; the sweep's
    cost does not depend on Sigma's values), scaled by q / rows and by the
    sweep count (rows are independent, so the cost is linear in them)."""
    dev = torch.device("cuda:0")
    stream = torch.cuda.current_stream()
    out = {}
    # the first (c1) pass also loads the code objects; it is repeated and the
    # repeat is reported
    for key in ("c1", "c1", "c2", "c3up", "c3down", "c5"):
        spec = synth.CONFIGS[key]
        q, p, n = spec.q, spec.p, spec.n
        log(f"{key}: {q}x{p}, {n} tokens")
        chunk = n if p * n * 4 <= (16 << 30) else 32768
        Sigma = torch.empty((p, p), dtype=torch.float32, device=dev)
        gram_s = 0.0
        head = None
        for c in range(n // chunk):
            Xc = synth.activation_chunk_device(spec, c, chunk, dev)
            if c == 0 and with_oracle:
                head = Xc[:, :CONFIG_ORACLE[key][1]].cpu().numpy()
            e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            e0.record(stream)
            P.gram(Xc, Sigma=Sigma, accumulate=c > 0, damp=spec.damp if c == n // chunk - 1 else 0.0)
            e1.record(stream)
            torch.cuda.synchronize()
            gram_s += e0.elapsed_time(e1) * 1e-3
            del Xc
        torch.cuda.empty_cache()
        W_h = synth.weights(spec)
        W = torch.from_numpy(W_h).to(dev)
        scale, zero = P.grid_minmax(W, spec.bits)
        Wh = torch.empty_like(W)
        R = torch.empty_like(W)
        codes = torch.empty((q, p), dtype=torch.uint8, device=dev)
        ws = P.workspace(P.cd_workspace_size(q, p, 128), dev)
        e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        e0.record(stream)
        P.cd_sweep(W, Sigma, spec.bits, scale, zero, Wh, codes, R, spec.sweeps, block=128,
                   flags=P.QE_INIT_FROM_W, ws=ws, check=False)
        e1.record(stream)
        torch.cuda.synchronize()
        cd_s = e0.elapsed_time(e1) * 1e-3
        rec = {"q": q, "p": p, "n": n, "bits": spec.bits, "sweeps": spec.sweeps,
               "gram_s": gram_s, "gram_chunks": n // chunk,
               "gram_fp32_equivalent_tflops": float(p) * (p + 1) * n / gram_s / 1e12,
               "sweep_s": cd_s / spec.sweeps,
               "column_updates_per_s": p * spec.sweeps / cd_s,
               "cd_fp32_equivalent_tflops": 2.0 * q * p * p * spec.sweeps / cd_s / 1e12,
               "layer_s": gram_s + cd_s,
               "layer_column_updates_per_s": p * spec.sweeps / (gram_s + cd_s)}
        sc_h, ze_h = scale.cpu().numpy(), zero.cpu().numpy()
        del Sigma, W, Wh, R, codes, ws
        torch.cuda.empty_cache()
        if with_oracle and key in CONFIG_ORACLE and head is not None:
            import oracle
            rows_n, _ = CONFIG_ORACLE[key]
            S = oracle.damp(oracle.gram_blas(head, row_block=4096), spec.damp)
            rows = synth.row_sample(q, rows_n, spec.cfg)
            t = oracle.cd_sweep_timed(W_h[rows], S, spec.bits, sc_h[rows], ze_h[rows])
            del S
            sweep_oracle = t * q / len(rows)
            rec["oracle"] = {"sweep_s": sweep_oracle, "measured_s": t, "rows": len(rows),
                             "cores": oracle.num_threads(), "kind": "oracle",
                             "column_updates_per_s": p / sweep_oracle,
                             "extrapolated": len(rows) < q}
            rec["gpu_over_oracle"] = rec["column_updates_per_s"] / rec["oracle"]["column_updates_per_s"]
        out[spec.name] = rec
    return {"configs": out}


def configs_report(rep):
    """Per-configuration rows for the line: the timings of configs_bench plus,
    from the committed per-configuration kernel trace and counter profile
    (while the step kernel's sources match), the panel-only launch as HBM
    bandwidth (17 bytes per coordinate of a 256-column super-block) and the
    step kernel's matrix-core busy fraction."""
    prof = _json_block(CONFIG_PROFILE)
    valid = bool(prof) and prof.get("source_sha256") == kernel_source_hash("cd_step_kernel")
    rows = {}
    for name, rec in rep["configs"].items():
        row = dict(rec)
        pc = prof.get("configs", {}).get(name) if valid else None
        if pc:
            t = pc["panel_only_launch_us"] * 1e-6
            b = 17.0 * rec["q"] * min(256, rec["p"])
            row["panel"] = {"launch_s": t, "achieved_GBps": b / t / 1e9,
                            "frac_of_hbm_peak": b / t / 1e9 / HBM_PEAK_GBS}
            row["cd_step_mfma_busy"] = pc.get("mfma_busy")
        else:
            row["panel"] = None
            row["cd_step_mfma_busy"] = None
        rows[name] = row
    return rows


def outlier_bench(P, torch, synth, W, Sigma, dev, block):
    spec = synth.CONFIGS["c4"]
    q, p, bits, iters, s = spec.q, spec.p, spec.bits, spec.sweeps, spec.s_budget
    stream = torch.cuda.current_stream()
    ev = [torch.cuda.Event(enable_timing=True) for _ in range(6)]
    ws_o = P.workspace(P.outlier_workspace_size(q, p, block, s), dev)
    Wh = torch.empty_like(W)
    codes = torch.empty((q, p), dtype=torch.uint8, device=dev)
    E = torch.empty_like(W)
    obj = torch.zeros(2 * iters, dtype=torch.float64, device=dev)
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    lam = P.lambda_max(Sigma)
    t_lam = time.perf_counter() - t0

    def run(timed):
        if timed:
            ev[0].record(stream)
        H, sup, nnz = P.topk_abs(W, s, check=False)
        scale, zero = P.grid_minmax(W, bits, H)
        if timed:
            ev[1].record(stream)
        P.cd_outlier_sweep(W, Sigma, bits, scale, zero, Wh, codes, H, E, s, lam, sup, nnz, iters,
                           block=block, flags=P.QE_INIT_FROM_W, obj=obj, ws=ws_o, check=False)
        if timed:
            ev[2].record(stream)
        return nnz

    run(False)
    torch.cuda.synchronize()
    nnz = run(True)
    torch.cuda.synchronize()
    assert P.sync_status(ws_o) == 0
    g = obj.cpu().numpy()
    t_init = ev[0].elapsed_time(ev[1]) * 1e-3
    t_iters = ev[1].elapsed_time(ev[2]) * 1e-3
    res = {"workload": spec.name, "s": s, "lambda_max": lam, "lambda_time_s": t_lam,
           "init_time_s": t_init, "iter_time_s": t_iters / iters,
           "support_nnz": int(nnz.cpu().item()),
           "g_after_cd": [float(x) for x in g[0::2]], "g_after_iht": [float(x) for x in g[1::2]]}

    # structured outliers (Sec. 4.3): floor(s / q) whole columns
    ncols = s // q
    sup = torch.zeros(s, dtype=torch.int64, device=dev)

    def run_cols(timed):
        if timed:
            ev[3].record(stream)
        H, _, sup_c, n = P.topk_columns(W, ncols, check=False)
        sup[:q * ncols] = sup_c[:q * ncols]
        scale, zero = P.grid_minmax(W, bits, H)
        if timed:
            ev[4].record(stream)
        P.cd_outlier_sweep(W, Sigma, bits, scale, zero, Wh, codes, H, E, s, lam, sup, n, iters,
                           block=block, flags=P.QE_INIT_FROM_W | P.QE_OUTLIER_COLUMNS, obj=obj,
                           ws=ws_o, check=False)
        if timed:
            ev[5].record(stream)

    run_cols(False)
    torch.cuda.synchronize()
    run_cols(True)
    torch.cuda.synchronize()
    assert P.sync_status(ws_o) == 0
    g = obj.cpu().numpy()
    res["structured"] = {"columns": ncols, "init_time_s": ev[3].elapsed_time(ev[4]) * 1e-3,
                         "iter_time_s": ev[4].elapsed_time(ev[5]) * 1e-3 / iters,
                         "g_after_iht": [float(x) for x in g[1::2]]}
    return res


if __name__ == "__main__":
    main()
