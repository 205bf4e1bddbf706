"""The example's policy on tokens: it runs, every worker's replicas of a file
are the same bits, so that the adversaries are found in every iteration, and a
file's gradient is that of its loss in 64 bits."""
import importlib.util
import os

import numpy as np
import pytest

from paper_2108_02416_amd import aspis

from _helpers import device
from _tokens import kept

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                    "clipped_training.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("clipped_training", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("optimizer", ["sgd", "adamw"])
def test_token_training(example, optimizer):
    losses, found, agreed = example.train_tokens(5, optimizer, device(), say=lambda line: None)
    assert np.isfinite(losses).all()
    assert all(agreed)
    assert all(f == frozenset(example.ADVERSARIES) for f in found)


def test_a_files_gradient(example):
    """Against the chain in 64 bits by automatic differentiation on the host.
    The products of f32 matrices add at most HIDDEN and VOCAB roundings each to
    sums whose terms are bounded by the largest gradient and hidden values."""
    import torch
    gen = torch.Generator().manual_seed(1)
    table = (0.3 * torch.randn((example.VOCAB, example.HIDDEN), generator=gen)).to(device())
    head = (0.05 * torch.randn((example.HIDDEN, example.VOCAB), generator=gen)).to(device())
    reference = table + 0.05, head * 1.1
    batch = example.rollouts(table, head, reference, 1, 3, device())[0]
    batch["old"] = batch["old"] + 0.1
    d = table.numel() + head.numel()
    out = torch.full((d,), 7.0, device=device())
    sums = example.policy_gradient(table, head, batch, 17, out)

    t64, h64 = (x.double().cpu().requires_grad_() for x in (table, head))
    tokens = batch["tokens"].cpu()
    there = (tokens >= 0).double()[:, None]
    x = example.SCALE * t64[tokens.clamp(min=0)] * there
    keep = torch.from_numpy(kept(x.numel(), example.DROP, 17, 0).reshape(x.shape)).double()
    limit = round(example.DROP * 65536)
    logits = x * keep * (65536 / (65536 - limit)) @ h64
    lp = torch.log_softmax(logits, 1).gather(1, batch["actions"].cpu()[:, None])[:, 0]
    host = {k: v.double().cpu() for k, v in batch.items() if v.is_floating_point()}
    r = torch.exp(lp - host["old"])
    gap = host["ref"] - lp
    loss = (host["weight"] * (example.KL * (gap.exp() - 1 - gap) - torch.minimum(
        r * host["advantage"], r.clamp(0.8, 1.2) * host["advantage"]))).sum()
    loss.backward()
    want = torch.cat([t64.grad.reshape(-1), h64.grad.reshape(-1)])
    assert abs(float(sums[0]) - float(loss.detach())) <= 1e-5
    bound = 4 * (example.HIDDEN + example.VOCAB) * 2.0 ** -24
    for got, exact in ((out[:table.numel()], want[:table.numel()]),
                       (out[table.numel():], want[table.numel():])):
        assert float((got.double().cpu() - exact).abs().max()) <= bound * float(exact.abs().max()) * 4
