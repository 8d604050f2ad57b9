"""Output error of the quantized linear against float64, on the synthetic
workloads: a symmetrization ablation and bit-width sweep standing in for the
paper's Table 6 (with and without symmetrization, Sec. 4.4) and Table 10
(W8A6, W6A6, W8A4, W4A4), plus the per-token path of Eq. (c) as the
baseline the paper argues against (Sec. 2.2), and the same linears on 4-bit
floating point (MX4) with and without the channels' shift and scale, and the
attention behind a qkv linear with its keys and values in an 8-bit cache.

The paper measures perplexity on checkpoints and datasets that are not used
here; this measures the error the method introduces in one linear, which is
what those numbers follow from.  Every step runs through libot: one
calibration pass (ot_calibrate) gives the minmax state, ot_scales_from_minmax
derives each configuration's z and s from it, then ot_fold_weights,
ot_quantize_act and ot_qlinear (or the per-token or mx4 entry points).  The
reference is X W^T + b in float64 (torch, on the GPU).
"""
from __future__ import annotations

import torch

from . import ot, synth

# (label, a_bits, w_bits, path): path "channel" is OutlierTune's per-channel
# path, "channel-nosym" the same without symmetrization, "token" Eq. (c)
CONFIGS = [
    ("W8A8", 8, 8, "channel"), ("W8A8 no-sym", 8, 8, "channel-nosym"),
    ("W8A6", 6, 8, "channel"), ("W8A6 no-sym", 6, 8, "channel-nosym"),
    ("W6A6", 6, 6, "channel"), ("W6A6 no-sym", 6, 6, "channel-nosym"),
    ("W8A4", 4, 8, "channel"), ("W8A4 no-sym", 4, 8, "channel-nosym"),
    ("W4A4", 4, 4, "channel"), ("W4A4 no-sym", 4, 4, "channel-nosym"),
    ("W8A8 per-token", 8, 8, "token"), ("W6A6 per-token", 6, 6, "token"),
]

# 4-bit floating point in blocks of 32: with the channels' shift and scale taken
# out first, with the scale alone, and with neither
MX4_CONFIGS = [("MX4", 4, 4, "mx4"), ("MX4 no-sym", 4, 4, "mx4-nosym"),
               ("MX4 plain", 4, 4, "mx4-plain")]


def layer_inputs(wl, li, rows, calib_rows, calib_batches, device="cuda"):
    """Device tensors of one layer: X [rows, K], W, b, and the calibration
    minmax state of ot_calibrate over the seeded calibration batches."""
    X = torch.from_numpy(synth.activations(wl, li, rows)).to(device)
    W = torch.from_numpy(synth.weight(wl, li)).to(device)
    b = torch.from_numpy(synth.bias(wl, li)).to(device)
    minmax, _, _, _ = ot.calibrate(synth.calibration_batches(wl, li, calib_rows, calib_batches),
                                   8, device)
    return X, W, b, minmax


def run_config(X, W, b, minmax, a_bits, w_bits, path):
    """The quantized linear's fp16 output for one configuration."""
    if path == "token":
        Xq, sX = ot.quantize_act_per_token(X, a_bits)
        Wq, sW, bp = ot.fold_weights_per_token(W, b, None, w_bits)
        return ot.qlinear_per_token(Xq, Wq, sX, sW, bp, a_bits, w_bits)
    if path.startswith("mx4"):
        # a block's own scale takes care of the magnitude, so any a_bits gives the
        # same channel-to-channel proportions
        z, s, inv_s = (None, None, None) if path == "mx4-plain" else \
            ot.scales_from_minmax(minmax, 8, path == "mx4")
        Wc, We, bp = ot.fold_weights_mx4(W, b, z, s)
        return ot.qlinear_mx4(*ot.quantize_act_mx4(X, z, inv_s), ot.pack_weights_mx4(Wc, We),
                              W.shape[0], bp, True)
    z, s, inv_s = ot.scales_from_minmax(minmax, a_bits, path == "channel")
    Wq, sW, bp = ot.fold_weights(W, b, w_bits, z, s)
    Xq = ot.quantize_act(X, a_bits, z, inv_s)
    return ot.qlinear(Xq, Wq, sW, bp, a_bits, w_bits)


def errors(Y, ref):
    """Relative Frobenius error, mean and max absolute error (float64)."""
    e = Y.double() - ref
    return dict(rel_fro=float(e.norm() / ref.norm()), mean_abs=float(e.abs().mean()),
                max_abs=float(e.abs().max()))


def sweep(workloads=("opt6.7b_w8a8", "opt13b_w6a6", "opt66b_w8a8"), rows=256, calib_rows=None,
          calib_batches=None, configs=None, device="cuda", log=None):
    """Errors of every configuration on every linear of the given workloads
    (calibration: the workload's own batches unless given).  Configurations:
    CONFIGS, and MX4_CONFIGS where the linear's channels are whole blocks of 32,
    unless given.  Returns a list of dicts (workload, layer, config, a_bits,
    w_bits, path, rel_fro, mean_abs, max_abs)."""
    out = []
    for name in workloads:
        wl = synth.WORKLOADS[name]
        for li, lay in enumerate(wl.layers):
            X, W, b, minmax = layer_inputs(wl, li, rows, calib_rows, calib_batches, device)
            ref = torch.matmul(X.double(), W.double().t()) + b.double()
            mx4 = MX4_CONFIGS if X.shape[1] % 32 == 0 else []
            for label, a_bits, w_bits, path in CONFIGS + mx4 if configs is None else configs:
                Y = run_config(X, W, b, minmax, a_bits, w_bits, path)
                rec = dict(workload=name, layer=lay.name, config=label, a_bits=a_bits,
                           w_bits=w_bits, path=path, **errors(Y, ref))
                out.append(rec)
                if log:
                    log(f"quality {name}/{lay.name} {label}: rel {rec['rel_fro']:.3e}")
            del X, W, b, minmax, ref
    return out


# Attention behind a workload's qkv linear: (label, path of the linear, None for float64,
# whether keys and values go through the 8-bit cache)
ATTENTION_CONFIGS = [("KV8", None, True), ("W8A8", "channel", False), ("W8A8 KV8", "channel", True)]


def head_channels(hidden):
    """Channels of a head: OPT's smaller sizes have 64, the others 128."""
    return 64 if hidden < 2048 else 128


def attention_ref(q, k, v):
    """Causal softmax(q k^T / sqrt(D)) v of one sequence [tokens, heads, D] in float64."""
    q, k, v = q.double(), k.double(), v.double()
    n, heads, D = q.shape
    hidden = torch.ones(n, n, dtype=torch.bool, device=q.device).triu(1)
    out = torch.empty_like(q)
    for h in range(heads):
        x = (q[:, h] @ k[:, h].t()) * D ** -0.5
        out[:, h] = x.masked_fill(hidden, float("-inf")).softmax(1) @ v[:, h]
    return out


def attention_kv8(q, k, v, singles=8):
    """The same through the cache (fp16): a prompt and then `singles` tokens one by one, each
    written with ot_kv8_append and read by ot_attn_kv8, as a server would."""
    n, heads, D = q.shape
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device=q.device)
    pages = -(-n // ot.KV8_PAGE)
    table = torch.randperm(pages, device=q.device).int()[None]
    cache = ot.kv8_cache(pages, heads, D, q.device)
    first = max(n - singles, 1)
    out = torch.empty(n, heads, D, dtype=torch.float16, device=q.device)
    for lo, hi in [(0, first)] + [(i, i + 1) for i in range(first, n)]:
        cu, length = ints(0, hi - lo), ints(hi)
        ot.kv8_append(k[lo:hi], v[lo:hi], cu, length, table, cache)
        out[lo:hi] = ot.attn_kv8(q[lo:hi], cu, length, table, cache)
    return out


def attention_sweep(workloads=("opt6.7b_w8a8", "opt13b_w6a6", "opt66b_w8a8"), rows=256,
                    calib_rows=None, calib_batches=None, configs=None, device="cuda", log=None):
    """Errors of attention over `rows` tokens behind each workload's qkv linear, against
    float64 attention on the float64 linear.  Returns a list of dicts (workload, config,
    rel_fro, mean_abs, max_abs)."""
    out = []
    for name in workloads:
        wl = synth.WORKLOADS[name]
        li = [lay.name for lay in wl.layers].index("qkv")
        X, W, b, minmax = layer_inputs(wl, li, rows, calib_rows, calib_batches, device)
        hidden = W.shape[0] // 3
        heads = lambda y: y.view(rows, 3, hidden // head_channels(hidden), -1).unbind(1)
        exact = torch.matmul(X.double(), W.double().t()) + b.double()
        ref = attention_ref(*heads(exact))
        for label, path, cached in ATTENTION_CONFIGS if configs is None else configs:
            y = exact.half() if path is None else run_config(X, W, b, minmax, 8, 8, path)
            Y = attention_kv8(*heads(y)) if cached else attention_ref(*heads(y))
            rec = dict(workload=name, config=label, **errors(Y, ref))
            out.append(rec)
            if log:
                log(f"quality {name}/attention {label}: rel {rec['rel_fro']:.3e}")
    return out
