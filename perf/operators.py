"""Timed cases of the operators on gradients: the global norm over many tensors
(grad_norm), clipping by it (clip_grads), clipping every row of a replica
tensor by its own norm (clip_rows), and the model update that applies the
clip as it reads the gradient (clipped_sgd, clipped_adamw).

Gradients are separate tensors, as a backward pass leaves them.  Parameters,
optimizer state and clipped results are views into one flat buffer each,
packed without padding, so most of them start off a 16-byte boundary.

A case holds
  op        "norm", "clip", "rows", "sgd" or "adamw"
  layout    the lists' tensor sizes: "softmax" (784 x 10 weights, 10 biases),
            "resnet" (ResNet-18 on 10 classes, 62 tensors), "blocks" (hidden,
            layers, vocab: a stack of transformer blocks), or "random" (total
            elements over `tensors` tensors of uneven sizes); for "rows":
            rows, d and pad (elements between one row's end and the next)
  dtype     the gradients' type: "float32", "bfloat16", "float16", or "mixed"
            (matrices bfloat16, vectors float32)
  max_norm  the bound (rows: 1.5 times an honest row's norm)
  each      norm: every tensor's norm too
  nesterov, decay, copy   the update's options (copy: the type of the
            parameters' low-precision copy, or "")
"""
import random
from math import exp, log, sqrt

import torch

own = False

TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
LR, MU, BETAS, EPS = 0.01, 0.9, (0.9, 0.95), 1e-8


def _case(name, op, **more):
    return {"name": name, "op": op, "dtype": "float32", **more}


def listed():
    blocks = {"layout": "blocks", "hidden": 2048, "layers": 16, "vocab": 32_003}
    return [
        # the softmax layer of a seven-worker run: only the call's own cost
        _case("norm_softmax", "norm", layout="softmax", each=False),
        # the headline's model, a ResNet-18, tensor by tensor
        _case("norm_resnet", "norm", layout="resnet", each=False),
        # a language model's gradients: matrices in bfloat16, vectors in
        # float32, every tensor's norm for the training log
        _case("norm_blocks", "norm", **{**blocks, "dtype": "mixed"}, each=True),
        _case("clip_softmax", "clip", layout="softmax", max_norm=0.5),
        # a worker's gradient of one batch, clipped
        _case("clip_resnet", "clip", layout="resnet", max_norm=1.0),
        # the largest list whose result is written out
        _case("clip_blocks", "clip", **{**blocks, "dtype": "mixed"}, max_norm=1.0),
        # one worker's upload in a seven-worker run: its 15 files
        _case("rows_softmax", "rows", rows=15, d=7_850, pad=0),
        # all replicas of 2,300 files, an odd length, uploaded in half precision
        _case("rows_many", "rows", rows=6_900, d=10_007, pad=0, dtype="float16"),
        # one worker's upload at the headline: 91 files of 11.2M coordinates
        _case("rows_headline", "rows", rows=91, d=11_200_000, pad=0),
        _case("sgd_softmax", "sgd", layout="softmax", max_norm=0.5, nesterov=False, decay=0.0,
              copy=""),
        # the headline's model updated from the aggregated gradient
        _case("sgd_resnet", "sgd", layout="resnet", max_norm=1.0, nesterov=True, decay=5e-4,
              copy=""),
        # a language model in mixed precision: master weights and state in
        # float32, gradients and the model's own weights in bfloat16
        _case("adamw_blocks", "adamw", **{**blocks, "dtype": "bfloat16"}, max_norm=1.0,
              decay=0.1, copy="bfloat16"),
    ]


def _log_int(rng, low, high):
    return int(exp(rng.uniform(log(low), log(high + 1))))


def draw(rng):
    op = rng.choice(["norm", "clip", "rows", "rows", "sgd", "adamw"])
    dtype = rng.choice(["float32", "float32", "bfloat16", "float16"])
    if op == "rows":
        d = _log_int(rng, 1, 11_200_000)
        rows = _log_int(rng, 1, min(100_000, max(1, 600_000_000 // d)))
        return {"op": op, "dtype": dtype, "rows": rows, "d": d,
                "pad": rng.choice([0, 0, rng.randint(1, 70)])}
    total = _log_int(rng, 1, 500_000_000)
    case = {"op": op, "layout": "random", "total": total, "dtype": dtype,
            "tensors": _log_int(rng, 1, min(400, total))}
    if op == "norm":
        return {**case, "each": rng.random() < 0.3}
    case["max_norm"] = rng.choice([0.5, 1.0, 5.0])
    if op == "sgd":
        case.update(nesterov=rng.random() < 0.5, decay=rng.choice([0.0, 5e-4]))
    if op == "adamw":
        case.update(decay=rng.choice([0.0, 0.1]))
    if op != "clip":
        case["copy"] = rng.choice(["", "bfloat16", "float16"])
    return case


# ------------------------------------------------------------------ inputs

def _numels(case):
    """The list's tensor sizes, and which of them are vectors."""
    if case["layout"] == "softmax":
        return [784 * 10, 10], [False, True]
    if case["layout"] == "random":
        r = random.Random(case["total"] * 1009 + case["tensors"])
        w = [exp(r.uniform(-5, 0)) for _ in range(case["tensors"])]
        left = case["total"] - case["tensors"]
        n = [1 + int(left * x / sum(w)) for x in w]
        n[-1] += case["total"] - sum(n)
        return n, [False] * len(n)
    if case["layout"] == "blocks":
        h, wide = case["hidden"], case["hidden"] * 8 // 3
        block = [h, 3 * h * h, h * h, h, 2 * h * wide, wide * h]
        n = [case["vocab"] * h] + block * case["layers"] + [h]
        return n, [x == h for x in n]
    n, at = [3 * 64 * 9, 64, 64], 64
    for width in (64, 128, 256, 512):
        for _ in range(2):
            n += [at * width * 9, width, width, width * width * 9, width, width]
            if at != width:
                n += [at * width, width, width]
            at = width
    n += [512 * 10, 10]
    return n, [x <= 512 for x in n]


def _grads(case, seed):
    """The gradients: N(0, 0.01^2), every tensor with a scale of its own
    between 0.3 and 3."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    numels, vector = _numels(case)
    scale = random.Random(seed)
    out = []
    for n, v in zip(numels, vector):
        kind = case["dtype"]
        kind = torch.float32 if kind == "mixed" and v else TYPES.get(kind, torch.bfloat16)
        x = torch.randn(n, generator=gen, device="cuda")
        out.append(x.mul_(0.01 * exp(scale.uniform(-1.2, 1.1))).to(kind))
    return out, gen


def _rows(case, seed):
    """Rows of N(0, 0.01^2); every fifth one, on average, an adversary's, a
    hundred times as long."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rows, d, pad = case["rows"], case["d"], case["pad"]
    x = torch.empty((rows, d + pad), dtype=TYPES[case["dtype"]], device="cuda")
    step = max(1, (1 << 28) // (d + pad))
    for i in range(0, rows, step):
        part = x[i:i + step]
        part.copy_(torch.randn(part.shape, generator=gen, device="cuda").mul_(0.01))
    bad = torch.rand(rows, generator=gen, device="cuda") < 0.2
    for i in bad.nonzero().flatten().tolist():
        x[i].mul_(100.0)
    return x[:, :d]


def _views(flat, numels):
    return list(flat.split(numels))


def prepare(case, seed):
    if case["op"] == "rows":
        x = _rows(case, seed)
        state = {"case": case, "x": x, "bound": 0.015 * sqrt(case["d"]),
                 "out": torch.empty(x.shape, dtype=x.dtype, device="cuda"),
                 "norms": torch.empty(case["rows"], device="cuda")}
        if own:   # the workspace a server keeps
            from paper_2108_02416_amd import aspis
            state["ws"] = aspis.row_workspace(x)
        return state
    grads, gen = _grads(case, seed)
    numels = [g.numel() for g in grads]
    state = {"case": case, "grads": grads, "lists": {}}
    lists = {"grads": grads}
    if case["op"] == "clip":
        # one flat buffer per type, the tensors' results packed in it
        kinds = list(dict.fromkeys(g.dtype for g in grads))
        state["out"] = [torch.empty(sum(g.numel() for g in grads if g.dtype == k), dtype=k,
                                    device="cuda") for k in kinds]
        views = {k: iter(_views(f, [g.numel() for g in grads if g.dtype == k]))
                 for k, f in zip(kinds, state["out"])}
        lists["out"] = [next(views[g.dtype]) for g in grads]
    if case["op"] in ("sgd", "adamw"):
        # a run some way in: state of the size that clipped gradients give it
        n = sum(numels)
        rms = case["max_norm"] / sqrt(n)
        flat = {"params": torch.randn(n, generator=gen, device="cuda").mul_(0.02),
                "mean": torch.randn(n, generator=gen, device="cuda").mul_(rms)}
        if case["op"] == "adamw":
            flat["square"] = torch.rand(n, generator=gen, device="cuda").add_(0.5).mul_(rms * rms)
        if case["copy"]:
            flat["copy"] = torch.empty(n, dtype=TYPES[case["copy"]], device="cuda")
        state.update(flat, step=1000)
        lists.update({k: _views(f, numels) for k, f in flat.items()})
    if own:   # the handles and buffers a training program makes once
        from paper_2108_02416_amd import aspis
        state["lists"] = {k: aspis.TensorList(v) for k, v in lists.items()}
        state["bufs"] = aspis.NormBuffers.empty(grads[0].device,
                                                each=len(grads) if case.get("each") else 0)
        state["ws"] = aspis.norm_workspace(state["lists"]["grads"])
    return state


# --------------------------------------------------------------- the calls

def run(state):
    return (_own if own else _plain)(state)


def _own(state):
    from paper_2108_02416_amd import aspis
    case = state["case"]
    if case["op"] == "rows":
        out, norms = aspis.clip_rows(state["x"], state["bound"], out=state["out"],
                                     norms=state["norms"], ws=state["ws"])
        return {"out": out, "norms": norms}
    lists, bufs = state["lists"], state["bufs"]
    keep = {"bufs": bufs, "ws": state["ws"]}
    if case["op"] == "norm":
        aspis.grad_norm(lists["grads"], each=case["each"], **keep)
        return {"norm": bufs.norm, "each": bufs.each} if case["each"] else {"norm": bufs.norm}
    if case["op"] == "clip":
        aspis.clip_grads(lists["grads"], case["max_norm"], out=lists["out"], **keep)
        return {"norm": bufs.norm, "out": state["out"]}
    keep.update(weight_decay=case["decay"], max_norm=case["max_norm"], copies=lists.get("copy"))
    state["step"] += 1
    if case["op"] == "sgd":
        aspis.clipped_sgd(lists["params"], lists["grads"], lists["mean"], lr=LR, momentum=MU,
                          nesterov=case["nesterov"], **keep)
    else:
        aspis.clipped_adamw(lists["params"], lists["grads"], lists["mean"], lists["square"],
                            step=state["step"], lr=LR, betas=BETAS, eps=EPS, **keep)
    return _updated(state, bufs.norm)


def _updated(state, norm):
    return {"norm": norm, **{k: state[k] for k in ("params", "mean", "square", "copy")
                             if k in state}}


def _coef(norm, bound):
    return torch.where(norm <= bound, torch.ones_like(norm), bound / norm)


def _plain(state):
    case = state["case"]
    if case["op"] == "rows":
        x = state["x"].float()
        norms = (x * x).sum(1).sqrt()
        state["out"].copy_(x * _coef(norms, state["bound"])[:, None])
        return {"out": state["out"], "norms": norms}
    grads = state["grads"]
    if case["op"] == "norm" and case["each"]:
        each = torch.stack([(g.float() * g.float()).sum() for g in grads])
        return {"norm": each.sum().sqrt().reshape(1), "each": each.sqrt()}
    kinds = list(dict.fromkeys(g.dtype for g in grads)) if case["op"] == "clip" else [None]
    flat = [torch.cat([g.reshape(-1) for g in grads if k in (None, g.dtype)]).float()
            for k in kinds]
    norm = sum((x * x).sum() for x in flat).sqrt().reshape(1)
    if case["op"] == "norm":
        return {"norm": norm}
    coef = _coef(norm, case["max_norm"])
    if case["op"] == "clip":
        return {"norm": norm, "out": [o.copy_(x * coef) for o, x in zip(state["out"], flat)]}
    state["step"] += 1
    p, m, decay = state["params"], state["mean"], case["decay"]
    g = flat[0] * coef
    if case["op"] == "sgd":
        if decay:
            g = g + decay * p
        m.mul_(MU).add_(g)
        p.sub_(LR * (g + MU * m if case["nesterov"] else m))
    else:
        v, t = state["square"], state["step"]
        if decay:
            p.mul_(1 - LR * decay)
        m.mul_(BETAS[0]).add_((1 - BETAS[0]) * g)
        v.mul_(BETAS[1]).add_((1 - BETAS[1]) * (g * g))
        p.sub_((LR / (1 - BETAS[0] ** t)) * m / ((v / (1 - BETAS[1] ** t)).sqrt() + EPS))
    if "copy" in state:
        state["copy"].copy_(p)
    return _updated(state, norm)


def work(case):
    size = {"float32": 4, "bfloat16": 2, "float16": 2}
    if case["op"] == "rows":
        n = case["rows"] * case["d"]
        return {"bytes": 2 * n * size[case["dtype"]] + 4 * case["rows"], "flops": 3 * n}
    numels, vector = _numels(case)
    n = sum(numels)
    grads = sum(x * size.get(case["dtype"], 4 if v else 2) for x, v in zip(numels, vector))
    if case["op"] == "norm":
        return {"bytes": grads + 4 + 4 * case["each"] * len(numels), "flops": 2 * n}
    if case["op"] == "clip":
        return {"bytes": 2 * grads + 4, "flops": 3 * n}
    state, flops = {"sgd": (16, 9), "adamw": (24, 16)}[case["op"]]
    return {"bytes": grads + (state + size.get(case["copy"], 0)) * n + 4, "flops": flops * n}


# -------------------------------------------------------------- reference

def exact(case, seed):
    """One pass from the definitions, in 64 bits."""
    if case["op"] == "rows":
        x = _rows(case, seed)
        norms = torch.empty(case["rows"], dtype=torch.float64, device="cuda")
        out = torch.empty(x.shape, dtype=torch.float64, device="cuda")
        for i in range(0, case["rows"], max(1, (1 << 27) // case["d"])):
            part = x[i:i + max(1, (1 << 27) // case["d"])].double()
            norms[i:i + len(part)] = part.square().sum(1).sqrt()
            ratio = 0.015 * sqrt(case["d"]) / norms[i:i + len(part)]
            out[i:i + len(part)] = part * ratio.clamp(max=1.0)[:, None]
        return {"out": out, "norms": norms}
    state = prepare(case, seed)
    grads = state["grads"]
    each = torch.stack([g.double().square().sum() for g in grads])
    norm = float(each.sum().sqrt())
    answer = {"norm": torch.tensor([norm], dtype=torch.float64)}
    if case["op"] == "norm":
        return {**answer, "each": each.sqrt()} if case["each"] else answer
    c = min(1.0, case["max_norm"] / norm) if norm > 0 else 1.0
    if case["op"] == "clip":
        kinds = list(dict.fromkeys(g.dtype for g in grads))
        return {**answer, "out": [torch.cat([c * g.double() for g in grads if g.dtype == k])
                                  for k in kinds]}
    p, m = state["params"].double(), state["mean"].double()
    g = torch.cat([c * x.double() for x in grads])
    if case["op"] == "sgd":
        g = g + case["decay"] * p
        m = MU * m + g
        p = p - LR * ((g + MU * m) if case["nesterov"] else m)
    else:
        t = state["step"] + 1
        v = BETAS[1] * state["square"].double() + (1 - BETAS[1]) * g.square()
        m = BETAS[0] * m + (1 - BETAS[0]) * g
        bent = (m / (1 - BETAS[0] ** t)) / ((v / (1 - BETAS[1] ** t)).sqrt() + EPS)
        p = p * (1 - LR * case["decay"]) - LR * bent
        answer["square"] = v
    answer.update(params=p, mean=m)
    if case["copy"]:
        answer["copy"] = p
    return answer
