"""Training under attack with clipped gradients, end to end on one GPU.

A softmax layer (784 inputs, 10 classes, 7,850 parameters) is trained on
synthetic data by K = 7 workers, two of them adversaries.  Every iteration
- the samples are split into f = C(7,3) = 35 files, each given to three
  workers;
- every honest worker clips each of its files' gradients and uploads them;
  the adversaries upload -100 times theirs;
- the server clips the replicas (so that none can carry more than the bound),
  finds the adversaries, and averages the files the others agree on;
- the aggregated gradient's global norm is clipped and an SGD step with
  momentum (or an AdamW step) applied, in one call.

  python examples/clipped_training.py [--iterations N] [--optimizer adamw]
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


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__,
                                 formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--iterations", type=int, default=60)
    ap.add_argument("--optimizer", choices=("sgd", "adamw"), default="sgd")
    args = ap.parse_args()
    train(args.iterations, args.optimizer)
