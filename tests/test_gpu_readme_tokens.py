"""The README's lines on token data, run in their order: the log-probabilities
are those of the logits, and the table's gradient is that of the loss."""
import os
import re

import numpy as np
import pytest

from paper_2108_02416_amd import aspis

from _helpers import device
from _tokens import Policy, f64, kept

pytestmark = pytest.mark.gpu

README = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")


def _lines():
    with open(README) as f:
        blocks = re.findall(r"```python\n(.*?)```", f.read(), re.S)
    found = [b for b in blocks if "aspis.embed_grad" in b]
    assert len(found) == 1
    return found[0]


def test_the_lines_on_token_data():
    import torch
    n, vocab, d, seed = 90, 70, 33, 5
    gen = torch.Generator().manual_seed(1)
    table, head = 0.1 * torch.randn((vocab, d), generator=gen), 0.3 * torch.randn((d, vocab), generator=gen)
    tokens, actions = (torch.randint(vocab, (n,), generator=gen) for _ in range(2))
    keep = torch.from_numpy(kept(n * d, 0.1, seed, 0).reshape(n, d)).double()

    def logits_of(t):   # in 64 bits
        return 8.0 * t[tokens] * keep * (65536 / (65536 - round(0.1 * 65536))) @ head.double()

    sampled = (logits_of(table.double()) + 0.1 * torch.randn((n, vocab), generator=gen)).float()
    host = {"advantage": torch.randn(n, generator=gen), "weight": torch.full((n,), 1.0 / n),
            "ref": Policy(f64(sampled), actions.numpy(), temperature=0.7).logps}
    host["ref"] = torch.from_numpy(host["ref"]).float() + 0.1
    space = {"aspis": aspis, "seed": seed, "vocab": vocab, "dtable": torch.empty_like(table).to(device()),
             **{k: v.to(device()) for k, v in {**host, "table": table, "head": head, "tokens": tokens,
                                               "actions": actions, "sampled": sampled}.items()}}
    space["head_t"] = space["head"].t().contiguous()
    exec(_lines(), space)

    Policy(f64(sampled), actions.numpy(), temperature=0.7).check_logps(space["old"])
    t64 = table.double().requires_grad_()
    lp = torch.log_softmax(logits_of(t64) / 0.7, 1).gather(1, actions[:, None])[:, 0]
    r = torch.exp(lp - space["old"].double().cpu())
    gap, adv = host["ref"].double() - lp, host["advantage"].double()
    loss = (host["weight"].double() * (0.02 * (gap.exp() - 1 - gap)
                                       - torch.minimum(r * adv, r.clamp(0.8, 1.2) * adv))).sum()
    loss.backward()
    # the f32 products of matrices add d and vocab roundings to what they sum
    assert abs(float(space["bufs"].sums[0]) - float(loss.detach())) <= 1e-5
    want = t64.grad.numpy()
    got = f64(space["dtable"])
    assert np.abs(got - want).max() <= 4 * (d + vocab) * 2.0 ** -24 * np.abs(want).max()
