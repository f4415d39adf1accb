"""The optimizer side of a population's training step, as a set of timed cases.

A population is N copies of one model in stacks of N * padded_P elements (tensors start on multiples of eight
elements; padding is zero here).  The operators work on its gradients:

  op  "norm"   every model's gradient norm over all of its tensors
      "clip"   gradients of the models whose norm is above max_norm scaled down, in place
      "sgd"    the norms and one step of SGD with momentum that takes the clipping's factor as it reads the gradients
      "adamw"  the same with AdamW

  table    tensor table: "resnet18", "resnet50", "flat:P" or "ragged:COUNT:LARGEST" (COUNT tensors of 1 to LARGEST coordinates);
           weight decay applies to tensors of two and more dimensions, in a ragged table to every other one
  layout   "np" (one model's row after the other) or "pn" (a coordinate's N values side by side)
  weights, grads   element types; momentum and the second moment are fp32
  clipped  "norm", "clip": models whose gradient is made longer than max_norm; steps: the same, 0 models: no norm is taken and nothing clipped
  step     the training step, from 0 (AdamW's bias correction)
"""
from __future__ import annotations

import math
import random

import torch

own = False

MAX_NORM = 1.0
LR, MOMENTUM, DECAY = 0.1, 0.9, 5e-4                              # SGD, the small-image recipe
ADAM_LR, BETA1, BETA2, EPS, ADAM_DECAY = 1e-3, 0.9, 0.999, 1e-8, 0.05
_TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "bf16": 2}
_LARGEST = 255_570_560                                            # N * padded_P of the largest listed case
_ADAM_LARGEST_BYTES = 28 * _LARGEST


def _case(op, N, table, clipped, layout="np", weights="f32", grads="f32", nesterov=False, step=0, **name):
    return dict(name, op=op, N=N, table=table, clipped=clipped, layout=layout, weights=weights, grads=grads, nesterov=nesterov, step=step)


def listed():
    return [
        # one small layer's tensors, odd lengths: launch and host time count
        _case("norm", 3, "ragged:8:5003", 2, name="norm_ragged_n3"),
        # the large network, the population of the benchmark: one pass over 1 GB of gradients
        _case("norm", 10, "resnet50", 6, name="norm_resnet50_n10"),
        # bf16 gradients, coordinate-major
        _case("norm", 8, "resnet50", 4, layout="pn", grads="bf16", name="norm_resnet50_n8_bf16_pn"),
        # gradients clipped in place for an optimizer of the caller's own
        _case("clip", 5, "resnet18", 3, name="clip_resnet18_n5"),
        # a large population whose gradient norms exceed the bound in most models, an odd length
        _case("clip", 32, "flat:4194301", 24, layout="pn", grads="bf16", name="clip_flat_n32_bf16_pn"),
        # a few small tensors: launch and host time count
        _case("sgd", 5, "ragged:12:4001", 3, name="sgd_ragged_n5"),
        # the small-image network's training step
        _case("sgd", 5, "resnet18", 2, name="sgd_resnet18_n5"),
        # bf16 weights and gradients with fp32 momentum, Nesterov's form
        _case("sgd", 8, "resnet50", 3, weights="bf16", grads="bf16", nesterov=True, name="sgd_resnet50_n8_bf16"),
        # coordinate-major, without clipping
        _case("sgd", 16, "flat:4194305", 0, layout="pn", name="sgd_flat_n16_pn"),
        # a small fine-tuned part of a model, first step
        _case("adamw", 2, "ragged:6:9001", 1, step=0, name="adamw_ragged_n2"),
        # the large network's training step
        _case("adamw", 10, "resnet50", 4, step=999, name="adamw_resnet50_n10"),
        # bf16 weights and gradients, coordinate-major, an odd population
        _case("adamw", 7, "flat:16777213", 7, layout="pn", weights="bf16", grads="bf16", step=9, name="adamw_flat_n7_bf16_pn"),
    ]


def draw(rng):
    op = rng.choice(["norm", "clip", "sgd", "adamw"])
    N = int(round(math.exp(rng.uniform(math.log(2), math.log(64)))))
    kind = rng.choice(["flat", "flat", "ragged", "ragged", "network"])
    most = _LARGEST // N
    target = int(math.exp(rng.uniform(math.log(1500), math.log(most))))
    table = "flat:%d" % target
    if kind == "network":
        fits = [t for t in ("resnet18", "resnet50") if _padded(t)[1] <= most]
        if fits:
            table = rng.choice(fits)
    elif kind == "ragged":
        count = rng.randint(2, 160)
        largest = max(8, target // 4)
        while _padded("ragged:%d:%d" % (count, largest))[1] > most:
            largest = largest * 2 // 3
        table = "ragged:%d:%d" % (count, largest)
    half = rng.choice(["f32", "bf16"])
    c = _case(op, N, table, rng.randint(1 if op == "clip" else 0, N), layout=rng.choice(["np", "pn"]), weights=half,
              grads=half if rng.random() < 0.7 else rng.choice(["f32", "bf16"]), nesterov=op == "sgd" and rng.random() < 0.4,
              step=int(math.exp(rng.uniform(0, math.log(100000)))) - 1)
    return c


# ---- tensor tables ------------------------------------------------------------------------

def _network(blocks, expansion, classes, stem):
    """(coordinates, dimensions) of a residual network's learnable tensors, in definition order"""
    out = []

    def conv_bn(cout, cin, k):
        out.extend([(cout * cin * k * k, 4), (cout, 1), (cout, 1)])

    conv_bn(64, 3, stem)
    cin = 64
    for stage, count in enumerate(blocks):
        width = 64 << stage
        for b in range(count):
            if expansion == 1:
                conv_bn(width, cin, 3)
                conv_bn(width, width, 3)
            else:
                conv_bn(width, cin, 1)
                conv_bn(width, width, 3)
                conv_bn(width * expansion, width, 1)
            if b == 0 and cin != width * expansion:
                conv_bn(width * expansion, cin, 1)
            cin = width * expansion
    out.extend([(classes * cin, 2), (classes, 1)])
    return out


def _table(spec):
    if spec == "resnet18":
        return _network((2, 2, 2, 2), 1, 100, 3)
    if spec == "resnet50":
        return _network((3, 4, 6, 3), 4, 1000, 7)
    kind, *args = spec.split(":")
    if kind == "flat":
        return [(int(args[0]), 2)]
    count, largest = int(args[0]), int(args[1])
    rng = random.Random(count * 1000003 + largest)
    return [(int(math.exp(rng.uniform(0.0, math.log(largest)))), 1 + i % 2) for i in range(count - 1)] + [(largest, 2)]


def _padded(spec):
    """(table, elements of a padded row)"""
    table = _table(spec)
    return table, sum((d + 7) // 8 * 8 for d, _ in table)


# ---- inputs ---------------------------------------------------------------------------------

def _inputs(case, seed):
    """The stacks as [N, P] or [P, N] tensors, zero in the padding, and the norms of the gradients."""
    N, op = case["N"], case["op"]
    table, P = _padded(case["table"])
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 7919 + 17)
    real = torch.zeros(P, device="cuda")
    at = 0
    for d, _ in table:
        real[at:at + d] = 1.0
        at += (d + 7) // 8 * 8

    def laid(rows):
        return rows.t().contiguous() if case["layout"] == "pn" else rows

    def stack(scale, dtype):
        rows = torch.empty(N, P, device="cuda", dtype=dtype)
        for n in range(N):   # a model's row at a time
            rows[n] = (torch.randn(P, generator=gen, device="cuda") * (scale[n] if isinstance(scale, list) else scale) * real).to(dtype)
        return laid(rows)

    coordinates = sum(d for d, _ in table)
    length = random.Random(seed)
    order = list(range(N))
    length.shuffle(order)
    over = set(order[:case["clipped"]])
    # tiny models' norms scatter: lengths keep a distance from the bound
    scale = [(length.uniform(2.0, 6.0) if n in over else length.uniform(0.1, 0.4)) * MAX_NORM / math.sqrt(coordinates) for n in range(N)]
    out = {"grads": stack(scale, _TYPE[case["grads"]])}
    if op == "clip":
        rows = out["grads"] if case["layout"] == "np" else out["grads"].t()
        out["norm"] = torch.stack([rows[n].double().square().sum().sqrt() for n in range(N)])
    if op in ("sgd", "adamw"):
        out["params"] = stack(0.05, _TYPE[case["weights"]])
        first = op == "adamw" and case["step"] == 0
        out["m"] = stack(0.0 if first else [0.5 * s for s in scale], torch.float32)
        if op == "adamw":
            out["v"] = stack(0.0 if first else scale, torch.float32).square_()
    return out


def prepare(case, seed):
    state = dict(_inputs(case, seed), case=case)
    N = case["N"]
    table, P = _padded(case["table"])
    if own:
        from paper_2405_17517_b200 import binding as B
        pop = B.Population(N, [d for d, _ in table], B.WASH_LAYOUT_PN if case["layout"] == "pn" else B.WASH_LAYOUT_NP, torch.cuda.current_device())
        for role, name in ((B.WASH_STACK_GRADS, "grads"), (B.WASH_STACK_PARAMS, "params"), (B.WASH_STACK_OPT, "m"), (B.WASH_STACK_OPT2, "v")):
            if name in state:
                pop.bind(role, state[name])
        if case["op"] in ("sgd", "adamw"):
            B.wash_set_decay(pop.ctx, [1.0 if dims > 1 else 0.0 for _, dims in table])
        state.update(B=B, pop=pop)
    else:
        decays = torch.zeros(P, device="cuda")   # the parameter groups of a training program, laid out once
        at = 0
        for d, dims in table:
            decays[at:at + d] = float(dims > 1)
            at += (d + 7) // 8 * 8
        state["decays"] = decays if case["layout"] == "np" else decays[:, None]
    if case["op"] != "clip":
        state["norm"] = torch.zeros(N, dtype=torch.float64, device="cuda")
    return state


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(state):
    case, B, ctx = state["case"], state["B"], state["pop"].ctx
    op, norm = case["op"], state["norm"]
    if op == "clip":
        B.wash_clip_grads(ctx, MAX_NORM, norm)
        return {"grads": state["grads"]}
    clipping = op == "norm" or case["clipped"] > 0
    if clipping:
        B.wash_grad_norm(ctx, 0, state["pop"].numel.size, norm)
    if op == "norm":
        return {"norm": norm}
    max_norm, given = (MAX_NORM, norm) if clipping else (0.0, None)
    if op == "sgd":
        B.wash_sgd_step(ctx, LR, MOMENTUM, DECAY, B.WASH_STEP_NESTEROV if case["nesterov"] else 0, max_norm, given)
        out = {"params": state["params"], "m": state["m"]}
    else:
        B.wash_adamw_step(ctx, case["step"], ADAM_LR, BETA1, BETA2, EPS, ADAM_DECAY, 0, max_norm, given)
        out = {"params": state["params"], "m": state["m"], "v": state["v"]}
    return dict(out, norm=norm) if clipping else out


def _models(values, case):
    """One value a model, shaped to go with a stack"""
    return values[:, None] if case["layout"] == "np" else values[None, :]


def _factor(norm):
    return torch.clamp(MAX_NORM / (norm + 1e-6), max=1.0)


def _run_plain(state):
    case = state["case"]
    op, axis = case["op"], 1 if case["layout"] == "np" else 0
    if op == "clip":
        g = state["grads"]
        g.copy_(g.float() * _models(_factor(state["norm"]).float(), case))
        return {"grads": g}
    clipping = op == "norm" or case["clipped"] > 0
    norm = None
    if clipping:
        norm = state["grads"].double().square().sum(dim=axis).sqrt()
    if op == "norm":
        return {"norm": norm}
    g = state["grads"].float()
    if clipping:
        g = g * _models(_factor(norm).float(), case)
    params, m = state["params"], state["m"]
    p = params.float()
    if op == "sgd":
        d = g + (DECAY * state["decays"]) * p
        m.mul_(MOMENTUM).add_(d)
        params.copy_(p - LR * (d + MOMENTUM * m if case["nesterov"] else m))
        out = {"params": params, "m": m}
    else:
        v, t = state["v"], case["step"] + 1
        m.mul_(BETA1).add_((1.0 - BETA1) * g)
        v.mul_(BETA2).add_((1.0 - BETA2) * g * g)
        u = (m / (1.0 - BETA1 ** t)) / (v.sqrt() / math.sqrt(1.0 - BETA2 ** t) + EPS)
        params.copy_(p - ADAM_LR * (u + (ADAM_DECAY * state["decays"]) * p))
        out = {"params": params, "m": m, "v": v}
    return dict(out, norm=norm) if clipping else out


def exact(case, seed):
    """The operators' definitions in 64 bits, model by model."""
    given = _inputs(case, seed)
    N, op, rows = case["N"], case["op"], case["layout"] == "np"
    table, P = _padded(case["table"])
    decay = torch.zeros(P, dtype=torch.float64, device="cuda")
    at = 0
    for d, dims in table:
        if dims > 1:
            decay[at:at + d] = DECAY if op == "sgd" else ADAM_DECAY
        at += (d + 7) // 8 * 8
    names = {"norm": [], "clip": ["grads"], "sgd": ["params", "m"], "adamw": ["params", "m", "v"]}[op]
    out = {k: torch.empty(given[k].shape, dtype=torch.float64, device="cuda") for k in names}
    norms = []
    for n in range(N):
        def mine(name):
            return (given[name][n] if rows else given[name][:, n]).to(torch.float64)
        g = mine("grads")
        if op == "clip":
            norm = given["norm"][n].item()
        else:
            norm = math.sqrt((g * g).sum().item())
            norms.append(norm)
        new = {}
        if op != "norm" and case["clipped"] > 0 and norm + 1e-6 > MAX_NORM:
            g = g * (MAX_NORM / (norm + 1e-6))
        if op == "clip":
            new["grads"] = g
        elif op == "sgd":
            w = mine("params")
            d = g + decay * w
            new["m"] = MOMENTUM * mine("m") + d
            new["params"] = w - LR * (d + MOMENTUM * new["m"]) if case["nesterov"] else w - LR * new["m"]
        elif op == "adamw":
            t, w = case["step"] + 1, mine("params")
            new["m"] = BETA1 * mine("m") + (1 - BETA1) * g
            new["v"] = BETA2 * mine("v") + (1 - BETA2) * g ** 2
            # 1 - beta^t without the difference of two neighbours
            first, second = -math.expm1(t * math.log(BETA1)), -math.expm1(t * math.log(BETA2))
            hat = (new["m"] / first) / (torch.sqrt(new["v"] / second) + EPS)
            new["params"] = w - ADAM_LR * hat - ADAM_LR * decay * w
        for name, value in new.items():
            if rows:
                out[name][n] = value
            else:
                out[name][:, n] = value
    if op == "norm" or (op != "clip" and case["clipped"] > 0):
        out["norm"] = torch.tensor(norms, dtype=torch.float64, device="cuda")
    return out


def work(case):
    N, op = case["N"], case["op"]
    coordinates = sum(d for d, _ in _table(case["table"]))
    g, w = _BYTES[case["grads"]], _BYTES[case["weights"]]
    n = N * coordinates
    if op == "norm":
        return {"bytes": n * g + 8 * N, "flops": 2 * n}
    if op == "clip":   # the gradients of models within the bound need not be touched
        return {"bytes": 2 * g * case["clipped"] * coordinates + 8 * N, "flops": case["clipped"] * coordinates}
    norm = 2 * n if case["clipped"] > 0 else 0
    if op == "sgd":    # each input once, each output once
        return {"bytes": n * (g + 2 * w + 8), "flops": norm + 8 * n}
    return {"bytes": n * (g + 2 * w + 16), "flops": norm + 18 * n}
