"""Timed cases of the operators at both ends of a worker's step on token data:
the embedding lookup with scaling (embed) and its gradient by sorted tokens
(embed_grad), dropout from a counter-based generator (dropout, the same call
forward and backward), the log-probabilities of tokens under logits
(token_logps), and the clipped policy loss with a KL term and its gradient
(policy_loss).

Workers that hold the same file have to return the same bits, so none of these
may depend on a device's random state or on the order of atomic additions:
dropout's mask is a function of a seed and an element's position, a table row's
gradient is summed in the order of the tokens.

A case holds
  op       "embed", "embed_grad", "dropout", "logps" or "policy"
  dtype    the type of the table, the incoming gradient, x or the logits
  tokens, vocab, d   embed, embed_grad: tokens looked up, table rows and their length
  out      embed, embed_grad: the type of the result
  index    the tokens' type
  scaled   embed, embed_grad: rows are multiplied by sqrt(d)
  accumulate   embed_grad: the result is added to what the table's gradient holds
  rows, d, pad, p, residual, offset   dropout: x has `pad` elements between one
           row's end and the next; what it adds the result to; the first
           element's position
  rows, vocab, masked, kl, temperature   logps, policy: positions, `masked` of
           them without weight (a prompt's), the KL term's factor (0: none)
"""
import random
from functools import lru_cache
from math import exp, log, sqrt

import numpy as np
import torch

own = False

TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
INDEX = {"int64": torch.int64, "int32": torch.int32}
CLIP = (0.2, 0.25)


def _case(name, op, **more):
    return {"name": name, "op": op, **more}


def _embed(name, op, tokens, vocab, d, dtype, out, accumulate=False, scaled=False, index="int64"):
    case = _case(name, op, dtype=dtype, tokens=tokens, vocab=vocab, d=d, out=out, index=index,
                 scaled=scaled)
    return {**case, "accumulate": accumulate} if op == "embed_grad" else case


def _policy(name, op, rows, vocab, dtype, masked=0, kl=0.0, temperature=1.0):
    case = _case(name, op, dtype=dtype, rows=rows, vocab=vocab, temperature=temperature,
                 index="int64")
    return {**case, "masked": masked, "kl": kl} if op == "policy" else case


def listed():
    return [
        # one token while a model answers: only the call's own cost
        _embed("embed_token", "embed", 1, 32_003, 2048, "bfloat16", "bfloat16"),
        # a batch looked up in float32 master weights, scaled, in the model's type
        _embed("embed_batch", "embed", 16_384, 32_003, 2048, "float32", "bfloat16", scaled=True),
        # the table's gradient of one worker's file: few tokens, odd sizes
        _embed("embed_grad_file", "embed_grad", 515, 4_099, 257, "float32", "float32",
               scaled=True),
        # the same of a whole batch, written out for the upload, rows without
        # tokens as zeros
        _embed("embed_grad_batch", "embed_grad", 32_768, 32_003, 2048, "bfloat16", "float32"),
        # a table shared with the output layer: added to that layer's gradient
        _embed("embed_grad_tied", "embed_grad", 65_536, 128_003, 1024, "bfloat16", "float32",
               accumulate=True, index="int32"),
        # the hidden layer of a small classifier
        _case("dropout_small", "dropout", dtype="float32", rows=32, d=784, pad=0, p=0.5,
              residual=False, offset=0),
        # a block's output, dropped and added to the residual stream
        _case("dropout_residual", "dropout", dtype="bfloat16", rows=16_384, d=2048, pad=0, p=0.1,
              residual=True, offset=0),
        # the gradient of one rank's shard of a long activation, rows of a
        # wider buffer, an odd length and start
        _case("dropout_shard", "dropout", dtype="float16", rows=10_007, d=2_049, pad=63, p=0.2,
              residual=False, offset=20_504_347),
        # a few answers scored under a reference model, token by token
        _policy("logps_few", "logps", 4, 128_003, "bfloat16"),
        # a batch's log-probabilities under the policy that sampled it
        _policy("logps_batch", "logps", 4_096, 32_003, "float32", temperature=0.7),
        # one worker's file of a small vocabulary, no KL term
        _policy("policy_file", "policy", 96, 257, "float32", masked=31),
        # the largest: a batch of prompts (masked) and answers
        _policy("policy_batch", "policy", 8_192, 128_003, "bfloat16", masked=2_003, kl=0.05),
    ]


def _log_int(rng, low, high):
    return int(exp(rng.uniform(log(low), log(high + 1))))


def draw(rng):
    op = rng.choice(["embed", "embed_grad", "embed_grad", "dropout", "logps", "policy", "policy"])
    dtype = rng.choice(["float32", "bfloat16", "bfloat16", "float16"])
    index = rng.choice(["int64", "int64", "int32"])
    if op in ("embed", "embed_grad"):
        d = _log_int(rng, 1, 4096)
        vocab = _log_int(rng, 2, min(131_072, 134_217_728 // d))
        tokens = _log_int(rng, 1, min(131_072, 67_108_864 // d))
        case = {"op": op, "dtype": dtype, "tokens": tokens, "vocab": vocab, "d": d, "index": index,
                "out": rng.choice(["float32", dtype]), "scaled": rng.random() < 0.5}
        if op == "embed_grad":
            case["accumulate"] = rng.random() < 0.3
            if case["accumulate"]:
                case["out"] = "float32"
        return case
    if op == "dropout":
        d = _log_int(rng, 1, 16_384)
        return {"op": op, "dtype": dtype, "rows": _log_int(rng, 1, max(1, 67_108_864 // d)), "d": d,
                "pad": rng.choice([0, 0, rng.randint(1, 70)]), "p": rng.choice([0.05, 0.1, 0.3, 0.5]),
                "residual": rng.random() < 0.4,
                "offset": rng.choice([0, 0, _log_int(rng, 1, 1 << 40)])}
    vocab = _log_int(rng, 2, 131_072)
    rows = _log_int(rng, 1, min(16_384, max(1, 600_000_000 // vocab)))
    case = {"op": op, "dtype": dtype, "rows": rows, "vocab": vocab, "index": index,
            "temperature": rng.choice([1.0, 1.0, 0.7, 1.3])}
    if op == "policy":
        case.update(masked=int(rows * rng.choice([0.0, 0.3, 0.6])), kl=rng.choice([0.0, 0.05, 0.2]))
    return case


# ------------------------------------------------------------------ inputs

def _normal(shape, gen, kind, scale):
    x = torch.empty(shape, dtype=TYPES[kind], device="cuda")
    flat = x.view(-1)
    for i in range(0, flat.numel(), 1 << 28):
        part = flat[i:i + (1 << 28)]
        part.copy_(torch.randn(part.shape, generator=gen, device="cuda").mul_(scale))
    return x


def _tokens(case, gen):
    """Word frequencies: token k is drawn in proportion to 1 / k (near enough),
    so the commonest are a few percent of the batch; one position in 33 holds
    no token (-1, padding)."""
    n, vocab = case["tokens"], case["vocab"]
    u = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)
    ids = (u * log(vocab + 1)).exp().long().sub_(1).clamp_(0, vocab - 1)
    if n >= 33:
        ids[16::33] = -1
    return ids.to(INDEX[case["index"]])


def _scale(case):
    return sqrt(case["d"]) if case["scaled"] else 1.0


def _logps64(z, ids, temperature):
    """log p(ids) under the logits, in 64 bits."""
    out = torch.empty(len(z), dtype=torch.float64, device=z.device)
    step = max(1, (1 << 27) // z.shape[1])
    for i in range(0, len(z), step):
        part = z[i:i + step].double() / temperature
        at = part.gather(1, ids[i:i + step, None].long())[:, 0]
        top = part.amax(1)
        out[i:i + step] = at - top - (part - top[:, None]).exp().sum(1).log()
    return out


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op, kind = case["op"], case["dtype"]
    state = {"case": case}
    if op in ("embed", "embed_grad"):
        state["ids"] = _tokens(case, gen)
        n, vocab, d, out = case["tokens"], case["vocab"], case["d"], TYPES[case["out"]]
        if op == "embed":
            state["table"] = _normal((vocab, d), gen, kind, 0.02)
            state["out"] = torch.empty((n, d), dtype=out, device="cuda")
            return state
        state["grad"] = _normal((n, d), gen, kind, 0.01)
        if case["accumulate"]:
            state["out"] = _normal((vocab, d), gen, case["out"], 0.01)
        else:
            state["out"] = torch.empty((vocab, d), dtype=out, device="cuda")
        if own:   # the workspace a training program keeps
            from paper_2108_02416_amd import aspis
            state["ws"] = aspis.embed_workspace(state["grad"], state["ids"], vocab)
        return state
    if op == "dropout":
        rows, d = case["rows"], case["d"]
        state["x"] = _normal((rows, d + case["pad"]), gen, kind, 1.0)[:, :d]
        state["residual"] = _normal((rows, d), gen, kind, 1.0) if case["residual"] else None
        state["out"] = torch.empty((rows, d), dtype=TYPES[kind], device="cuda")
        state["seed"] = random.Random(seed).getrandbits(64)
        return state
    rows, vocab = case["rows"], case["vocab"]
    state["logits"] = _normal((rows, vocab), gen, kind, 2.0)
    # the likeliest of eight tokens: what a policy samples has a high probability
    eight = torch.randint(vocab, (rows, 8), generator=gen, device="cuda")
    best = state["logits"].gather(1, eight).float().argmax(1, keepdim=True)
    state["ids"] = eight.gather(1, best)[:, 0].to(INDEX[case["index"]])
    state["logps"] = torch.empty(rows, device="cuda")
    if own:
        from paper_2108_02416_amd import aspis
        state["ws"] = aspis.policy_workspace(state["logits"])
    if op == "logps":
        return state
    here = _logps64(state["logits"], state["ids"], case["temperature"])
    noise = torch.randn((3, rows), generator=gen, device="cuda", dtype=torch.float64)
    old = here + 0.15 * noise[0]
    # a ratio right at a border of the clip has a gradient on one side and none
    # on the other: those few are moved off it
    for border in (1.0 - CLIP[0], 1.0 + CLIP[1]):
        close = ((here - old).exp() / border - 1.0).abs() < 1e-3
        old = torch.where(close, old + 3e-3, old)
    state["old"] = old.float()
    state["ref"] = (here + 0.3 * noise[1]).float() if case["kl"] else None
    state["advantage"] = noise[2].float()
    weight = torch.full((rows,), 1.0 / max(1, rows - case["masked"]), device="cuda")
    weight[torch.randperm(rows, generator=gen, device="cuda")[:case["masked"]]] = 0.0
    state["weight"] = weight
    state["grad"] = torch.empty_like(state["logits"])
    # half precision: the loss is scaled so that small gradients stay in range
    state["grad_scale"] = 4096.0 if kind == "float16" else 1.0
    if own:
        state["bufs"] = aspis.PolicyBuffers.empty(rows, state["logits"].device)
    return state


# --------------------------------------------------------------- the calls

def run(state):
    return (_own if own else _plain)(state)


def _own(state):
    from paper_2108_02416_amd import aspis
    case = state["case"]
    if case["op"] == "embed":
        return aspis.embed(state["table"], state["ids"], scale=_scale(case), out=state["out"])
    if case["op"] == "embed_grad":
        return aspis.embed_grad(state["grad"], state["ids"], case["vocab"], scale=_scale(case),
                                out=state["out"], accumulate=case["accumulate"], ws=state["ws"])
    if case["op"] == "dropout":
        return aspis.dropout(state["x"], case["p"], state["seed"], offset=case["offset"],
                             residual=state["residual"], out=state["out"])
    if case["op"] == "logps":
        return aspis.token_logps(state["logits"], state["ids"], temperature=case["temperature"],
                                 logps=state["logps"], ws=state["ws"])
    bufs = aspis.policy_loss(state["logits"], state["ids"], state["old"], state["advantage"],
                             state["weight"], ref=state["ref"], clip=CLIP, kl=case["kl"],
                             temperature=case["temperature"], grad=state["grad"],
                             grad_scale=state["grad_scale"], bufs=state["bufs"], ws=state["ws"])
    return {"sums": bufs.sums, "logps": bufs.logps, "grad": state["grad"]}


def _plain(state):
    case = state["case"]
    if case["op"] == "embed":
        ids = state["ids"].long()
        rows = state["table"][ids.clamp(min=0)].float() * _scale(case)
        return state["out"].copy_(torch.where((ids >= 0)[:, None], rows, torch.zeros_like(rows)))
    if case["op"] == "embed_grad":
        ids = state["ids"].long()
        sums = torch.zeros((case["vocab"] + 1, case["d"]), device="cuda")
        ids = torch.where(ids >= 0, ids, torch.full_like(ids, case["vocab"]))
        sums.index_add_(0, ids, state["grad"].float())
        sums = sums[:-1] * _scale(case)
        return state["out"].copy_(sums + state["out"].float() if case["accumulate"] else sums)
    if case["op"] == "dropout":
        keep, scale = _kept(case, state["seed"])
        x = state["x"].float() * scale
        x = torch.where(keep, x, torch.zeros_like(x))
        if case["residual"]:
            x = x + state["residual"].float()
        return state["out"].copy_(x)
    z = state["logits"].float() * (1.0 / case["temperature"])
    ids = state["ids"].long()[:, None]
    z = z - z.amax(1, keepdim=True)
    e = z.exp()
    total = e.sum(1, keepdim=True)
    lp = z.gather(1, ids)[:, 0] - total[:, 0].log()
    if case["op"] == "logps":
        return state["logps"].copy_(lp)
    weight, adv = state["weight"], state["advantage"]
    used = weight != 0
    ratio = (lp - state["old"]).exp()
    cut = torch.where(adv > 0, ratio > 1.0 + CLIP[1], (adv < 0) & (ratio < 1.0 - CLIP[0]))
    bound = torch.where(adv > 0, torch.full_like(adv, 1.0 + CLIP[1]),
                        torch.full_like(adv, 1.0 - CLIP[0]))
    loss = -torch.where(cut, bound, ratio) * adv
    slope = -torch.where(cut, torch.zeros_like(ratio), ratio) * adv
    kl = torch.zeros_like(lp)
    if case["kl"]:
        up = (state["ref"] - lp).exp()
        kl = up - 1.0 - (state["ref"] - lp)
        loss = loss + case["kl"] * kl
        slope = slope + case["kl"] * (1.0 - up)
    sums = torch.stack([(weight.double() * x.double()).sum() for x in (loss, kl, cut)])
    coef = weight * slope * (state["grad_scale"] / case["temperature"])
    grad = e.mul_((-coef / total[:, 0])[:, None])
    grad.scatter_add_(1, ids, coef[:, None])
    state["grad"].copy_(torch.where(used[:, None], grad, torch.zeros_like(grad)))
    return {"sums": sums.float(), "logps": torch.where(used, lp, torch.zeros_like(lp)),
            "grad": state["grad"]}


def _kept(case, seed):
    """Which elements stay, and the factor of those: element i of position
    q = offset + i takes the 16-bit half q mod 8 of Philox4x32-10 (Salmon,
    Moraes, Dror, Shaw, SC'11) with key `seed` and counter q div 8, and stays
    unless it is below the threshold p * 2^16, rounded."""
    rows, d, offset = case["rows"], case["d"], case["offset"]
    limit = round(case["p"] * 65536)
    low = 0xFFFFFFFF
    first, last = offset // 8, (offset + rows * d + 7) // 8
    block = torch.arange(first, last, device="cuda")
    c = [block & low, block >> 32, torch.zeros_like(block), torch.zeros_like(block)]
    k = [seed & low, seed >> 32]
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57   # modulo 2^64
        c = [(b >> 32 & low) ^ c[1] ^ k[0], b & low, (a >> 32 & low) ^ c[3] ^ k[1], a & low]
        k = [k[0] + 0x9E3779B9 & low, k[1] + 0xBB67AE85 & low]
    halves = torch.stack([w >> s & 0xFFFF for w in c for s in (0, 16)], dim=1).view(-1)
    at = offset - 8 * first
    return (halves[at:at + rows * d] >= limit).view(rows, d), 65536.0 / (65536 - limit)


# -------------------------------------------------------------------- work

@lru_cache(maxsize=None)
def _distinct(tokens, vocab):
    """Expected number of different tokens in a batch (see _tokens)."""
    edge = np.log(np.arange(1, vocab + 2)) / log(vocab + 1)
    return float((1.0 - (1.0 - np.diff(edge)) ** tokens).sum())


def work(case):
    size = {"float32": 4, "bfloat16": 2, "float16": 2}
    of = size[case["dtype"]]
    if case["op"] in ("embed", "embed_grad"):
        n, d = case["tokens"], case["d"]
        used = n - (len(range(16, n, 33)) if n >= 33 else 0)
        met = _distinct(used, case["vocab"])
        ids = n * (8 if case["index"] == "int64" else 4)
        to = size[case["out"]]
        if case["op"] == "embed":
            return {"bytes": ids + d * (met * of + n * to), "flops": n * d}
        written = 2 * met if case["accumulate"] else case["vocab"]
        return {"bytes": ids + d * (used * of + written * to), "flops": used * d}
    if case["op"] == "dropout":
        n = case["rows"] * case["d"]
        return {"bytes": n * of * (2 + case["residual"]), "flops": n * (1 + case["residual"])}
    n, vocab = case["rows"], case["vocab"]
    ids = 8 if case["index"] == "int64" else 4
    if case["op"] == "logps":
        return {"bytes": n * (vocab * of + ids + 4), "flops": 4 * n * vocab}
    used = n - case["masked"]
    return {"bytes": (used + n) * vocab * of + n * (ids + 16 + 4 * bool(case["kl"])),
            "flops": 7 * used * vocab}


# -------------------------------------------------------------- reference

def _philox_keeps(seed, offset, n, limit):
    """The same generator, in numpy's unsigned words."""
    u32, keeps = np.uint64(0xFFFFFFFF), np.empty(n, dtype=bool)
    for at in range(0, n, 1 << 24):
        pos = np.arange(offset + at, offset + min(n, at + (1 << 24)), dtype=np.uint64)
        blocks = np.arange(int(pos[0]) >> 3, (int(pos[-1]) >> 3) + 1, dtype=np.uint64)
        x0, x1 = blocks & u32, blocks >> np.uint64(32)
        x2, x3 = np.zeros_like(x0), np.zeros_like(x0)
        for r in range(10):
            ka = np.uint64((seed + r * 0x9E3779B9) & 0xFFFFFFFF)
            kb = np.uint64(((seed >> 32) + r * 0xBB67AE85) & 0xFFFFFFFF)
            p, q = x0 * np.uint64(0xD2511F53), x2 * np.uint64(0xCD9E8D57)
            x0, x1, x2, x3 = ((q >> np.uint64(32)) ^ x1 ^ ka, q & u32,
                              (p >> np.uint64(32)) ^ x3 ^ kb, p & u32)
        words = np.stack([x0, x1, x2, x3], axis=1).astype("<u4")
        halves = words.view("<u2").reshape(-1)
        start = int(pos[0]) - 8 * int(blocks[0])
        keeps[at:at + len(pos)] = halves[start:start + len(pos)] >= limit
    return keeps


def exact(case, seed):
    """One pass from the definitions, in 64 bits."""
    state = prepare(case, seed)
    op = case["op"]
    if op == "embed":
        ids = state["ids"].long()
        out = torch.zeros((case["tokens"], case["d"]), dtype=torch.float64, device="cuda")
        there = (ids >= 0).nonzero()[:, 0]
        out[there] = state["table"].double().index_select(0, ids[there]) * _scale(case)
        return out
    if op == "embed_grad":
        there = (state["ids"] >= 0).nonzero()[:, 0]
        ids = state["ids"][there].long()
        out = state["out"].double() if case["accumulate"] else torch.zeros(
            (case["vocab"], case["d"]), dtype=torch.float64, device="cuda")
        return out.index_add_(0, ids, state["grad"][there].double(), alpha=_scale(case))
    if op == "dropout":
        n, limit = case["rows"] * case["d"], round(case["p"] * 65536)
        keeps = torch.from_numpy(_philox_keeps(state["seed"], case["offset"], n, limit))
        out = state["x"].double().masked_fill(~keeps.cuda().view(case["rows"], case["d"]), 0.0)
        out *= 65536 / (65536 - limit)
        return out + state["residual"].double() if case["residual"] else out
    t, ids = case["temperature"], state["ids"].long()
    lp = _logps64(state["logits"], ids, t)
    if op == "logps":
        return lp
    w, adv = state["weight"].double(), state["advantage"].double()
    lp = torch.where(w == 0, torch.zeros_like(lp), lp)
    r = torch.exp(lp - state["old"].double())
    gain = torch.minimum(r * adv, r.clamp(1 - CLIP[0], 1 + CLIP[1]) * adv)
    free = gain == r * adv
    kl, by_kl = torch.zeros_like(lp), torch.zeros_like(lp)
    if case["kl"]:
        diff = state["ref"].double() - lp
        kl, by_kl = diff.expm1() - diff, -diff.expm1()
    sums = torch.stack([(w * (case["kl"] * kl - gain)).sum(), (w * kl).sum(),
                        (w * ~free).sum()])
    coef = state["grad_scale"] * w / t * (case["kl"] * by_kl - free * adv * r)
    grad = torch.empty(state["logits"].shape, dtype=torch.float64, device="cuda")
    step = max(1, (1 << 27) // case["vocab"])
    for i in range(0, case["rows"], step):
        part = state["logits"][i:i + step].double() / t
        p = torch.exp(part - part.gather(1, ids[i:i + step, None]) + lp[i:i + step, None])
        grad[i:i + step] = -coef[i:i + step, None] * p
    grad[torch.arange(case["rows"], device="cuda"), ids] += coef
    # a position without weight has the gradient 0 (its lp above is no log-probability)
    grad[w == 0] = 0.0
    return {"sums": sums, "logps": lp, "grad": grad}
