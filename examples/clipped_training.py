"""Training under attack with clipped gradients, end to end on one GPU.

A softmax layer (784 inputs, 10 classes, 7,850 parameters) is trained on
synthetic data by K = 7 workers, two of them adversaries; or, with --model
tokens, a policy on tokens (an embedding, dropout, and logits over the
vocabulary), whose gradients every worker computes for itself: each of its
files' replicas by calls of its own, in its own order, which agree bit for bit
with the other workers'.  Every iteration
- the samples are split into f = C(7,3) = 35 files, each given to three
  workers;
- every honest worker clips each of its files' gradients and uploads them;
  the adversaries upload -100 times theirs;
- the server clips the replicas (so that none can carry more than the bound),
  finds the adversaries, and averages the files the others agree on;
- the aggregated gradient's global norm is clipped and an SGD step with
  momentum (or an AdamW step) applied, in one call.

  python examples/clipped_training.py [--iterations N] [--optimizer adamw] [--model tokens]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2108_02416_amd import aspis  # noqa: E402

K, R, Q = 7, 3, 2
ADVERSARIES = (0, 1)
INPUTS, CLASSES, SAMPLES = 784, 10, 32
FILE_NORM = 2.0      # bound on one file's gradient
STEP_NORM = 0.5      # bound on the aggregated gradient


def make_data(files: int, device):
    gen = torch.Generator(device=device).manual_seed(428)
    x = torch.randn((files, SAMPLES, INPUTS), generator=gen, device=device)
    teacher = torch.randn((INPUTS, CLASSES), generator=gen, device=device)
    return x, (x @ teacher).argmax(-1)


def file_gradients(weight, bias, x, y):
    """Mean cross-entropy over all samples, and every file's gradient [f, d]."""
    logp = torch.log_softmax(x @ weight + bias, dim=-1)
    loss = -logp.gather(-1, y[..., None]).mean()
    delta = logp.exp()
    delta.scatter_add_(-1, y[..., None], torch.full_like(delta[..., :1], -1.0))
    delta /= SAMPLES
    by_weight = (x.transpose(1, 2).contiguous() @ delta).flatten(1)
    return loss, torch.cat([by_weight, delta.sum(1)], dim=1)


def train(iterations: int, optimizer: str = "sgd", device="cuda:0", say=print):
    device = torch.device(device)
    files = aspis.num_files(K, R)
    x, y = make_data(files, device)
    weight = torch.zeros((INPUTS, CLASSES), device=device)
    bias = torch.zeros(CLASSES, device=device)
    d = weight.numel() + bias.numel()
    # what the server keeps from one iteration to the next
    upload = torch.empty((K, files * R // K, d), device=device)
    rows = torch.from_numpy(aspis.worker_rows(K, R).reshape(-1)).long().to(device)
    grad = torch.empty(d, device=device)
    params = aspis.TensorList([weight, bias])
    grads = aspis.TensorList(list(grad.split([weight.numel(), bias.numel()])))
    mean, square = (aspis.TensorList([torch.zeros_like(weight), torch.zeros_like(bias)])
                    for _ in range(2))
    bufs, ws = aspis.NormBuffers.empty(device, each=len(grads)), aspis.norm_workspace(grads)
    losses, found = [], []
    for it in range(iterations):
        loss, g = file_gradients(weight, bias, x, y)
        # replica (i, s) is row rows[i * R + s] of the uploads
        upload.view(-1, d)[rows] = g.repeat_interleave(R, 0)
        for worker in range(K):
            if worker in ADVERSARIES:
                upload[worker].mul_(-100.0)
            else:
                aspis.clip_rows(upload[worker], FILE_NORM)
        # the server: no replica longer than the bound, whoever sent it
        _, norms = aspis.clip_rows(upload, FILE_NORM)
        res = aspis.detect_aggregate(upload, K, R, Q, mode="paper", layout="worker", out=grad)
        common = {"max_norm": STEP_NORM, "skip_nonfinite": True, "bufs": bufs, "ws": ws}
        if optimizer == "sgd":
            aspis.clipped_sgd(params, grads, mean, lr=0.5, momentum=0.9, **common)
        else:
            aspis.clipped_adamw(params, grads, mean, square, step=it + 1, lr=0.02,
                                weight_decay=0.0, **common)
        losses.append(float(loss))
        found.append(res["clique"].as_dict(K)["detected"])
        if it % 10 == 0 or it == iterations - 1:
            each = aspis.grad_norm(grads, each=True, bufs=bufs, ws=ws).each.tolist()
            say(f"iteration {it:3d}  loss {losses[-1]:.4f}  gradient norm {float(bufs.norm):.4f} "
                f"(weight {each[0]:.4f}, bias {each[1]:.4f})  longest upload "
                f"{float(norms.max()):.1f}  detected {sorted(found[-1])}")
    return losses, found


VOCAB, HIDDEN = 101, 48
DROP, KL, SCALE = 0.1, 0.02, HIDDEN ** 0.5


def policy_logits(table, head, tokens, seed):
    """What a worker keeps of a forward pass, and the logits."""
    hidden = aspis.dropout(aspis.embed(table, tokens, scale=SCALE), DROP, seed)
    return hidden, hidden @ head


def policy_gradient(table, head, batch, seed, out):
    """One file's loss and its gradient (of the table, then of the head) into
    the row `out` of the upload."""
    hidden, logits = policy_logits(table, head, batch["tokens"], seed)
    bufs = aspis.policy_loss(logits, batch["actions"], batch["old"], batch["advantage"],
                             batch["weight"], ref=batch["ref"], kl=KL, grad=logits)
    by_table, by_head = out.split([table.numel(), head.numel()])
    by_head.view_as(head).copy_(hidden.t().contiguous() @ logits)
    by_hidden = logits @ head.t().contiguous()
    aspis.dropout(by_hidden, DROP, seed, out=by_hidden)
    aspis.embed_grad(by_hidden, batch["tokens"], VOCAB, scale=SCALE, out=by_table.view_as(table))
    return bufs.sums


def rollouts(table, head, reference, files: int, it: int, device):
    """What the files hold: tokens, the actions that the policy answers them
    with, how good those are (a token's right answer is 7 t + 3 modulo the
    vocabulary) and their log-probabilities now and under the reference."""
    gen = torch.Generator().manual_seed(1000 + it)
    batches = []
    for _ in range(files):
        tokens = torch.randint(VOCAB, (SAMPLES,), generator=gen)
        tokens[::9] = -1                       # padding
        tokens = tokens.to(device)
        _, logits = policy_logits(table, head, tokens, 0)
        # an action drawn with the policy's probabilities
        noise = -torch.log(-torch.log(torch.rand((SAMPLES, VOCAB), generator=gen).clamp(1e-9, 1 - 1e-7)))
        actions = (logits + noise.to(device)).argmax(-1)
        reward = (actions == (7 * tokens + 3) % VOCAB).float()
        weight = (tokens >= 0).float()
        batches.append({
            "tokens": tokens, "actions": actions, "advantage": reward - 1.0 / VOCAB,
            "weight": weight / weight.sum(), "old": aspis.token_logps(logits, actions),
            "ref": aspis.token_logps(policy_logits(*reference, tokens, 0)[1], actions)})
    return batches


def train_tokens(iterations: int, optimizer: str = "sgd", device="cuda:0", say=print):
    """The same with a policy on tokens.  Returns the files' losses, who was
    found, and whether every honest worker's replicas were the same bits."""
    device = torch.device(device)
    files = aspis.num_files(K, R)
    gen = torch.Generator().manual_seed(428)
    table = (0.3 * torch.randn((VOCAB, HIDDEN), generator=gen)).to(device)
    head = (0.05 * torch.randn((HIDDEN, VOCAB), generator=gen)).to(device)
    reference = table.clone(), head.clone()
    subsets, rows = aspis.assign(K, R), aspis.worker_rows(K, R)
    d = table.numel() + head.numel()
    upload = torch.empty((K, files * R // K, d), device=device)
    grad = torch.empty(d, device=device)
    split = list(grad.split([table.numel(), head.numel()]))
    params, grads = aspis.TensorList([table, head]), aspis.TensorList(split)
    mean, square = (aspis.TensorList([torch.zeros_like(table), torch.zeros_like(head)])
                    for _ in range(2))
    bufs, ws = aspis.NormBuffers.empty(device), aspis.norm_workspace(grads)
    losses, found, agreed = [], [], []
    for it in range(iterations):
        batches = rollouts(table, head, reference, files, it, device)
        sums = {}
        for worker in range(K):
            # a worker's own order: its files from the last to the first
            for i in reversed(range(files)):
                if worker not in subsets[i]:
                    continue
                row = rows[i, list(subsets[i]).index(worker)]
                # dropout by file and iteration: the same for all who hold it
                sums[i] = policy_gradient(table, head, batches[i], it * files + i,
                                          upload.view(-1, d)[row])
            if worker in ADVERSARIES:
                upload[worker].mul_(-100.0)
            else:
                aspis.clip_rows(upload[worker], FILE_NORM)
        honest = [[upload.view(-1, d)[rows[i, s]] for s, w in enumerate(subsets[i])
                   if w not in ADVERSARIES] for i in range(files)]
        agreed.append(all(torch.equal(a, h[0]) for h in honest for a in h[1:]))
        aspis.clip_rows(upload, FILE_NORM)
        res = aspis.detect_aggregate(upload, K, R, Q, mode="paper", layout="worker", out=grad)
        common = {"max_norm": STEP_NORM, "skip_nonfinite": True, "bufs": bufs, "ws": ws}
        if optimizer == "sgd":
            aspis.clipped_sgd(params, grads, mean, lr=1.0, momentum=0.9, **common)
        else:
            aspis.clipped_adamw(params, grads, mean, square, step=it + 1, lr=0.02,
                                weight_decay=0.0, **common)
        losses.append(float(torch.stack(list(sums.values()))[:, 0].mean()))
        found.append(res["clique"].as_dict(K)["detected"])
        if it % 10 == 0 or it == iterations - 1:
            right = torch.stack([b["advantage"] for b in batches]).mean() + 1.0 / VOCAB
            say(f"iteration {it:3d}  loss {losses[-1]:.4f}  right answers {float(right):.3f}  "
                f"gradient norm {float(bufs.norm):.4f}  honest replicas equal {agreed[-1]}  "
                f"detected {sorted(found[-1])}")
    return losses, found, agreed


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__,
                                 formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--iterations", type=int, default=60)
    ap.add_argument("--optimizer", choices=("sgd", "adamw"), default="sgd")
    ap.add_argument("--model", choices=("softmax", "tokens"), default="softmax")
    args = ap.parse_args()
    (train if args.model == "softmax" else train_tokens)(args.iterations, args.optimizer)
