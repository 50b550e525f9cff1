"""What is timed of the training-step operators: what a rank does with its two kinds of messages once
they are decoded.

"norm" and "norm_backward" are the join of a block's all-reduced output with the residual stream and
the norm before the next block; "clip" is the global norm over many gradient tensors and the clipped
gradients; "step" is a ZeRO-1 rank's clipped AdamW step on its shard.  Sizes are those of workloads.py
(hidden size 6144, 4 x 2048 tokens, four tensor-parallel ranks, 1.5e8 parameters), smaller models'
and ragged neighbours of both.
"""
import math

import torch

own = False                # False: the plain form; True: the framework's operators

DEVICE = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-5
LARGEST_ROWS, LARGEST_COLS = 4 * 2048, 6144
LARGEST_SHARD = 150_000_000
ADAM = dict(lr=1e-4, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.01, step=7)
WORLD = 8                  # data-parallel ranks: the reduced gradients are sums over them
MAX_NORM = 1.0


def listed():
    return [
        # Serving: one new token for each of four sequences; latency alone counts.
        dict(name="norm_four_tokens_bf16", kind="norm", rows=4, cols=6144, dtype="bf16", layer=False, post=True, gate="none", save=False),
        # Training with fp16 messages, LayerNorm with its bias, plain residual (no norm after the block);
        # one sequence of 2048 tokens but the last.
        dict(name="norm_sequence_f16", kind="norm", rows=2047, cols=6144, dtype="f16", layer=True, post=False, gate="none", save=True),
        # One micro-batch behind its tensor-parallel all-reduce: norms after and before, a learned gate per channel.
        dict(name="norm_microbatch_bf16", kind="norm", rows=8192, cols=6144, dtype="bf16", layer=False, post=True, gate="channel", save=True),
        # An odd hidden size in fp32 with a gate for every element: rows start anywhere.
        dict(name="norm_ragged_f32", kind="norm", rows=1021, cols=4099, dtype="f32", layer=True, post=True, gate="full", save=True),
        # The backward passes of the three training cases.
        dict(name="norm_backward_sequence_f16", kind="norm_backward", rows=2047, cols=6144, dtype="f16", layer=True, post=False, gate="none"),
        dict(name="norm_backward_microbatch_bf16", kind="norm_backward", rows=8192, cols=6144, dtype="bf16", layer=False, post=True, gate="channel"),
        dict(name="norm_backward_ragged_f32", kind="norm_backward", rows=301, cols=1025, dtype="f32", layer=True, post=True, gate="full"),
        # A small model's gradients (two layers, hidden size 256, 24 tensors): the calls cost more than the bytes.
        dict(name="clip_small_model_f32", kind="clip", hidden=256, layers=2, ranks=1, dtype="f32", out="f32"),
        # Four layers at hidden size 1025: every tensor's length is odd or its place in the bucket is; bf16
        # gradients are clipped into the fp32 bucket that is exchanged.
        dict(name="clip_into_bucket_bf16", kind="clip", hidden=1025, layers=4, ranks=1, dtype="bf16", out="f32"),
        # Two layers of the 6144 wide model on one of four tensor-parallel ranks (2.3e8 fp32 gradients).
        dict(name="clip_two_layers_f32", kind="clip", hidden=6144, layers=2, ranks=4, dtype="f32", out="f32"),
        # A small shard whose length is odd, bf16 gradients.
        dict(name="step_small_shard_bf16", kind="step", n=(1 << 20) + 3, dtype="bf16", half="bf16"),
        # The ZeRO-1 shard of workloads.py: 1.5e8 parameters, fp32 gradients, bf16 parameters for the all-gather.
        dict(name="step_zero_shard_f32", kind="step", n=LARGEST_SHARD, dtype="f32", half="bf16"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm_backward", "clip", "step"])
    case = dict(kind=kind)
    if kind in ("norm", "norm_backward"):
        case["rows"] = _log_uniform(rng, 1, LARGEST_ROWS)
        case["cols"] = _log_uniform(rng, 64, 8192)
        if rng.random() < 0.5:
            case["cols"] = max(64, case["cols"] // 64 * 64)
        case["rows"] = min(case["rows"], LARGEST_ROWS * LARGEST_COLS // 2 // case["cols"])
        case["dtype"] = rng.choice(["f32", "bf16", "bf16", "f16"])
        case["layer"], case["post"] = rng.random() < 0.5, rng.random() < 0.5
        case["gate"] = rng.choice(["none", "channel", "full"])
        if kind == "norm":
            case["save"] = rng.random() < 0.7
    elif kind == "clip":
        case["hidden"] = _log_uniform(rng, 64, 4096)
        case["layers"] = rng.randint(1, 4)
        case["ranks"] = rng.choice([1, 2, 4]) if case["hidden"] < 2048 else 4
        case["dtype"], case["out"] = rng.choice(["f32", "f32", "bf16", "f16"]), rng.choice(["f32", "f32", "bf16"])
    else:
        case["n"] = _log_uniform(rng, 5000, LARGEST_SHARD)
        case["dtype"], case["half"] = rng.choice(["f32", "f32", "bf16", "f16"]), rng.choice(["none", "bf16", "bf16", "f16"])
    return case


# ---- inputs --------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(1_000_003 * seed + 17)
    return g


def _sizes(case):
    """The tensors of a transformer's layers on one of `ranks` tensor-parallel ranks: query-key-value, attention's output, the two
    of the feed-forward network, each with its bias, and two norms."""
    h, r = case["hidden"], case["ranks"]
    layer = [3 * h * h // r, 3 * h // r, h * h // r, h, 4 * h * h // r, 4 * h // r, 4 * h * h // r, h, h, h, h, h]
    return layer * case["layers"]


def _norm_inputs(case, seed):
    """Activations with a few outlier channels, weights near one, gates below one."""
    rows, cols, t = case["rows"], case["cols"], DTYPES[case["dtype"]]
    g = _generator(seed)

    def activation(std, mean=0.0):
        v = torch.randn((rows, cols), generator=g, device=DEVICE).mul_(std).add_(mean)
        v[:, torch.randint(0, cols, (max(1, cols // 200),), generator=g, device=DEVICE)] *= 10.0
        return v.to(t)

    def weight(mean, std):
        return torch.randn(cols, generator=g, device=DEVICE).mul_(std).add_(mean).to(t)

    s = dict(case)
    s["b"] = activation(0.5, 0.1)
    s["pre_weight"] = weight(1.0, 0.1)
    s["pre_bias"] = weight(0.0, 0.1) if case["layer"] else None
    s["post_weight"] = weight(1.0, 0.1) if case["post"] else None
    s["post_bias"] = weight(0.0, 0.1) if case["post"] and case["layer"] else None
    if case["gate"] == "channel":
        s["gate"] = weight(0.5, 0.2)
    elif case["gate"] == "full":
        s["gate"] = torch.sigmoid(torch.randn((rows, cols), generator=g, device=DEVICE)).to(t)
    else:
        s["gate"] = None
    s["residual_scale"] = 0.75
    if case["kind"] == "norm":
        s["x"] = activation(2.0, 0.2)
        return s
    s["y"] = activation(2.0, 0.2)
    s["dy"], s["dh"] = activation(1e-3), activation(1e-3) * 3
    return s


def _gradients(case, seed):
    g = _generator(seed)
    t = DTYPES[case["dtype"]]
    # one draw for all of them, then a tensor each: gradients of the layers differ in size
    sizes = _sizes(case)
    flat = torch.randn(sum(sizes), generator=g, device=DEVICE).mul_(3e-2)
    return [(part * (0.2 + 0.1 * (i % 12))).to(t) for i, part in enumerate(torch.split(flat, sizes))]


def _shard(case, seed):
    g, n = _generator(seed), case["n"]
    s = dict(case)
    s["grad"] = torch.randn(n, generator=g, device=DEVICE).mul_(1e-2).to(DTYPES[case["dtype"]])
    s["param"] = torch.randn(n, generator=g, device=DEVICE).mul_(0.02)
    s["m"] = torch.randn(n, generator=g, device=DEVICE).mul_(1e-3)
    s["v"] = torch.randn(n, generator=g, device=DEVICE).mul_(1e-3).square_()
    s["half_param"] = None if case["half"] == "none" else torch.empty(n, dtype=DTYPES[case["half"]], device=DEVICE)
    return s


def _statistics(v, layer):
    """(mean, 1 / deviation) of each row, as a forward pass leaves them."""
    v = v.float()
    mean = v.mean(1) if layer else torch.zeros(v.shape[0], device=DEVICE)
    return mean, torch.rsqrt((v - mean[:, None]).square().mean(1) + EPS)


def prepare(case, seed):
    kind = case["kind"]
    if kind in ("norm", "norm_backward"):
        s = _norm_inputs(case, seed)
        if kind == "norm":
            s["y"], s["h"] = torch.empty_like(s["x"]), torch.empty_like(s["x"])
            s["stats"] = torch.empty((case["rows"], 4), device=DEVICE) if case["save"] else None
            return s
        # what the forward pass has saved: for each row the post norm's mean and 1 / deviation, then the pre norm's
        s["stats"] = torch.zeros((case["rows"], 4), device=DEVICE)
        if case["post"]:
            s["stats"][:, 0], s["stats"][:, 1] = _statistics(s["b"], case["layer"])
        s["stats"][:, 2], s["stats"][:, 3] = _statistics(s["y"], case["layer"])
        return s
    if kind == "clip":
        s = dict(case)
        s["grads"] = _gradients(case, seed)
        s["bucket"] = torch.empty(sum(_sizes(case)), dtype=DTYPES[case["out"]], device=DEVICE)
        s["out_grads"] = list(torch.split(s["bucket"], _sizes(case)))
        return s
    return _shard(case, seed)


# ---- the timed pass ------------------------------------------------------------------

def _normed(v, layer, weight, bias):
    """The norm of each row, and the row's mean and 1 / deviation."""
    mean = v.mean(1, keepdim=True) if layer else torch.zeros_like(v[:, :1])
    v = v - mean if layer else v
    r = torch.rsqrt((v * v).mean(1, keepdim=True) + EPS)
    v = v * r * weight.float()
    return (v if bias is None else v + bias.float()), mean, r


def _plain_norm(s):
    z, stats = s["b"].float(), ()
    if s["post"]:
        z, *stats = _normed(z, s["layer"], s["post_weight"], s["post_bias"])
    if s["gate"] is not None:
        z = s["gate"].float() * z
    y = s["residual_scale"] * s["x"].float() + z
    h, *pre = _normed(y, s["layer"], s["pre_weight"], s["pre_bias"])
    y, h = y.to(s["x"].dtype), h.to(s["x"].dtype)
    if not s["save"]:
        return y, h
    return y, h, torch.cat([*(stats or [torch.zeros_like(t) for t in pre]), *pre], 1)


def _norm_gradient(dn, v_hat, r, weight, layer):
    """Gradient of a norm's input from that of its output."""
    t = dn * weight.float()
    t_in = t - v_hat * (t * v_hat).mean(1, keepdim=True)
    if layer:
        t_in = t_in - t.mean(1, keepdim=True)
    return r * t_in


def _plain_norm_backward(s):
    layer, stats, t = s["layer"], s["stats"], s["y"].dtype
    dh, b = s["dh"].float(), s["b"].float()
    y_hat = (s["y"].float() - stats[:, 2:3]) * stats[:, 3:4]
    out = {"pre_weight": (dh * y_hat).sum(0)}
    if s["pre_bias"] is not None:
        out["pre_bias"] = dh.sum(0)
    d = s["dy"].float() + _norm_gradient(dh, y_hat, stats[:, 3:4], s["pre_weight"], layer)
    out["x"] = (s["residual_scale"] * d).to(t)
    z = b
    if s["post"]:
        b_hat = (b - stats[:, 0:1]) * stats[:, 1:2]
        z = b_hat * s["post_weight"].float()
        if s["post_bias"] is not None:
            z = z + s["post_bias"].float()
    if s["gate"] is not None:
        dg = d * z
        out["gate"] = dg.sum(0) if s["gate"].dim() == 1 else dg.to(t)
        d = d * s["gate"].float()
    if s["post"]:
        out["post_weight"] = (d * b_hat).sum(0)
        if s["post_bias"] is not None:
            out["post_bias"] = d.sum(0)
        d = _norm_gradient(d, b_hat, stats[:, 1:2], s["post_weight"], layer)
    out["b"] = d.to(t)
    return out


def _factor(total, max_norm):
    """The norm of the averaged gradients from the sum of squares of the summed ones, and what clipping multiplies these by."""
    norm = torch.sqrt(total) / WORLD
    return norm, torch.where(norm <= max_norm, torch.ones_like(norm), max_norm / norm) / WORLD


def _plain_clip(s):
    flat = torch.cat([g.reshape(-1) for g in s["grads"]]).float()
    norm, factor = _factor((flat * flat).sum(), MAX_NORM)
    s["bucket"].copy_(flat * factor)
    return {"norm": norm.reshape(1), "bucket": s["bucket"]}


def _plain_step(s):
    a, g = ADAM, s["grad"].float()
    norm, factor = _factor((g * g).sum(), MAX_NORM)
    g = g * factor
    s["m"].mul_(a["beta1"]).add_(g * (1 - a["beta1"]))
    s["v"].mul_(a["beta2"]).add_(g * g * (1 - a["beta2"]))
    m_hat = s["m"] / (1 - a["beta1"] ** a["step"])
    v_hat = s["v"] / (1 - a["beta2"] ** a["step"])
    s["param"].sub_(a["lr"] * (m_hat / (torch.sqrt(v_hat) + a["eps"]) + a["weight_decay"] * s["param"]))
    out = {"norm": norm.reshape(1), "param": s["param"], "m": s["m"], "v": s["v"]}
    if s["half_param"] is not None:
        out["half_param"] = s["half_param"].copy_(s["param"])
    return out


def run(s):
    kind = s["kind"]
    if not own:
        return {"norm": _plain_norm, "norm_backward": _plain_norm_backward, "clip": _plain_clip, "step": _plain_step}[kind](s)
    from paper_2409_02423_amd import zt
    if kind in ("norm", "norm_backward"):
        form = dict(kind=zt.ZT_LAYER if s["layer"] else zt.ZT_RMS, pre_weight=s["pre_weight"], pre_bias=s["pre_bias"], post=s["post"],
                    post_weight=s["post_weight"], post_bias=s["post_bias"], d_gate=s["gate"], residual_scale=s["residual_scale"])
        if kind == "norm":
            y, h = zt.zt_residual_norm(s["x"], s["b"], eps=EPS, d_y=s["y"], d_h=s["h"], d_stats=s["stats"], **form)
            return (y, h, s["stats"]) if s["save"] else (y, h)
        got = zt.zt_residual_norm_backward(s["dy"], s["dh"], s["y"], s["b"], s["stats"], **form)
        return {k: v for k, v in got.items() if v is not None}
    if kind == "clip":
        norm = zt.zt_clip(s["grads"], MAX_NORM, scale=1.0 / WORLD, d_out=s["out_grads"])
        return {"norm": norm, "bucket": s["bucket"]}
    slots = zt.zt_sum_squares([s["grad"]])
    norm = zt.zt_adamw(s["grad"], s["param"], s["m"], s["v"], d_half=s["half_param"], d_slots=slots, scale=1.0 / WORLD, max_norm=MAX_NORM, **ADAM)
    out = {"norm": norm, "param": s["param"], "m": s["m"], "v": s["v"]}
    if s["half_param"] is not None:
        out["half_param"] = s["half_param"]
    return out


def work(case):
    """Every input read once and every output written once."""
    kind = case["kind"]
    if kind in ("norm", "norm_backward"):
        n, e = case["rows"] * case["cols"], BYTES[case["dtype"]]
        full, channel = case["gate"] == "full", case["gate"] == "channel"
        weights = 1 + case["layer"] + (1 + case["layer"]) * case["post"] + channel
        if kind == "norm":
            return {"bytes": n * e * (4 + full) + weights * case["cols"] * e + 16 * case["rows"] * case["save"], "flops": n * (6 + 4 * case["layer"] + 6 * case["post"])}
        return {"bytes": n * e * (6 + 2 * full) + weights * case["cols"] * (e + 4) + 16 * case["rows"],
                "flops": n * (14 + 2 * case["layer"] + 14 * case["post"] + 2 * (full or channel))}
    if kind == "clip":
        n = sum(_sizes(case))
        return {"bytes": n * (BYTES[case["dtype"]] + BYTES[case["out"]]), "flops": 3 * n}
    half = 0 if case["half"] == "none" else BYTES[case["half"]]
    return {"bytes": case["n"] * (BYTES[case["dtype"]] + 24 + half), "flops": 18 * case["n"]}


# ---- in 64 bits, from the definition -------------------------------------------------

def _exact_norm_parts(v, layer):
    v = v.double()
    mean = v.mean(1, keepdim=True) if layer else torch.zeros((v.shape[0], 1), dtype=torch.float64, device=v.device)
    deviation = torch.sqrt(((v - mean) ** 2).mean(1, keepdim=True) + EPS)
    return (v - mean) / deviation, deviation


def _or_zero(v):
    return 0.0 if v is None else v.double()


def _exact_norm_vjp(grad, unit, deviation, layer):
    """Jacobian of v -> unit(v), transposed, times grad: (I - [1 1^T / d] - unit unit^T / d) grad / deviation."""
    d = unit.shape[1]
    out = grad - unit * (unit * grad).sum(1, keepdim=True) / d
    if layer:
        out = out - grad.sum(1, keepdim=True) / d
    return out / deviation


def exact(case, seed):
    kind = case["kind"]
    if kind == "norm":
        s = _norm_inputs(case, seed)
        z = s["b"].double()
        if case["post"]:
            z = _exact_norm_parts(s["b"], case["layer"])[0] * s["post_weight"].double() + _or_zero(s["post_bias"])
        y = s["residual_scale"] * s["x"].double() + (z if s["gate"] is None else z * s["gate"].double())
        unit, deviation = _exact_norm_parts(y, case["layer"])
        h = unit * s["pre_weight"].double() + _or_zero(s["pre_bias"])
        if not case["save"]:
            return y, h
        stats = torch.zeros((case["rows"], 4), dtype=torch.float64, device=y.device)
        for at, v in ((0, s["b"].double()), (2, y)):
            if at or case["post"]:
                stats[:, at] = v.mean(1) if case["layer"] else 0.0
                stats[:, at + 1] = 1.0 / _exact_norm_parts(v, case["layer"])[1][:, 0]
        return y, h, stats
    if kind == "norm_backward":
        s = _norm_inputs(case, seed)
        unit, deviation = _exact_norm_parts(s["y"], case["layer"])
        dh = s["dh"].double()
        out = {"pre_weight": (dh * unit).sum(0)}
        if case["layer"]:
            out["pre_bias"] = dh.sum(0)
        total = s["dy"].double() + _exact_norm_vjp(dh * s["pre_weight"].double(), unit, deviation, case["layer"])
        out["x"] = s["residual_scale"] * total
        z = s["b"].double()
        if case["post"]:
            unit, deviation = _exact_norm_parts(s["b"], case["layer"])
            z = unit * s["post_weight"].double() + _or_zero(s["post_bias"])
        if s["gate"] is not None:
            out["gate"] = (total * z).sum(0) if case["gate"] == "channel" else total * z
            total = total * s["gate"].double()
        if case["post"]:
            out["post_weight"] = (total * unit).sum(0)
            if case["layer"]:
                out["post_bias"] = total.sum(0)
            total = _exact_norm_vjp(total * s["post_weight"].double(), unit, deviation, case["layer"])
        out["b"] = total
        return out
    if kind == "clip":
        flat = torch.cat([g.double().reshape(-1) for g in _gradients(case, seed)])
        norm = torch.linalg.vector_norm(flat) / WORLD
        return {"norm": norm.reshape(1), "bucket": flat.mul_(min(1.0, MAX_NORM / norm.item()) / WORLD)}
    s, a = _shard(case, seed), ADAM
    g = s["grad"].double()
    norm = torch.linalg.vector_norm(g) / WORLD
    g.mul_(min(1.0, MAX_NORM / norm.item()) / WORLD)
    m = a["beta1"] * s["m"].double() + (1 - a["beta1"]) * g
    v = a["beta2"] * s["v"].double() + (1 - a["beta2"]) * g ** 2
    p = s["param"].double()
    p = p * (1 - a["lr"] * a["weight_decay"]) - a["lr"] * (m / (1 - a["beta1"] ** a["step"])) / (torch.sqrt(v / (1 - a["beta2"] ** a["step"])) + a["eps"])
    out = {"norm": norm.reshape(1), "param": p, "m": m, "v": v}
    if case["half"] != "none":
        out["half_param"] = p
    return out
