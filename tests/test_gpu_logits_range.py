"""The operators on logits where |logit / temperature| is large: masks by a
finite constant, rows and parts of rows far from 0, temperatures to both ends
of what is accepted.  Against the formulas in 64 bits, with the bounds of
_tokens.Policy, which hold for any size of the logits."""
import math

import numpy as np
import pytest

from paper_2108_02416_amd import aspis

from _helpers import device
from _tokens import Policy, f64

pytestmark = pytest.mark.gpu

KINDS = ["float32", "bfloat16", "float16"]
LOG2E = 1.0 / math.log(2.0)


def _cuda(*arrays):
    import torch
    return [torch.from_numpy(np.ascontiguousarray(a)).to(device()) for a in arrays]


def _bits(t):
    import torch
    return t.contiguous().view(torch.int32 if t.dtype == torch.float32 else torch.int16).cpu().numpy()


def _check(z, t, temperature=1.0, grad_scale=1.0, repeat=0):
    """Log-probabilities, loss, gradient (beside the logits and in place) of the
    rows z for tokens t that have a probability; with `repeat` the same bits
    where every row is there so often, which other kernels take."""
    import torch
    rows = len(z)
    kind = str(z.dtype).split(".")[1]
    lp = Policy(f64(z), t, temperature=temperature).logps
    old = (lp - 0.05).astype(np.float32)
    ref = (lp + 0.1).astype(np.float32)
    adv = np.where(np.arange(rows) % 2, 1.0, -1.0).astype(np.float32)
    w = np.full(rows, 1.0 / rows, np.float32)
    plain = Policy(f64(z), t, old, adv, w, ref, kl=0.05, temperature=temperature,
                   grad_scale=grad_scale)
    logits = z.to(device())
    tokens, old, adv, w, ref = _cuda(t, old, adv, w, ref)
    plain.check_logps(aspis.token_logps(logits, tokens, temperature=temperature))
    grad = torch.empty_like(logits)
    more = dict(kl=0.05, temperature=temperature, grad_scale=grad_scale)
    bufs = aspis.policy_loss(logits, tokens, old, adv, w, ref=ref, grad=grad, **more)
    plain.check_logps(bufs.logps)
    plain.check_sums(bufs.sums)
    plain.check_grad(grad, kind)
    if repeat:
        many = [x.repeat_interleave(repeat, 0) for x in (logits, tokens, old, adv, w, ref)]
        all_grad = torch.empty_like(many[0])
        all_bufs = aspis.policy_loss(*many[:5], ref=many[5], grad=all_grad, **more)
        for i in (0, repeat - 1):
            assert (_bits(all_grad[i::repeat]) == _bits(grad)).all()
            assert (_bits(all_bufs.logps[i::repeat]) == _bits(bufs.logps)).all()
        logps = aspis.token_logps(many[0], many[1], temperature=temperature)
        assert (_bits(logps[::repeat]) == _bits(bufs.logps)).all()
    aspis.policy_loss(logits, tokens, old, adv, w, ref=ref, grad=logits, **more)
    assert (_bits(logits) == _bits(grad)).all()


def _mask_rows(vocab, mask, kind, temperature=1.0, seed=0):
    """Rows with `mask` in most places, and a token of each."""
    import torch
    gen = torch.Generator().manual_seed(seed)
    z = (temperature * torch.randn((8, vocab), generator=gen, dtype=torch.float64))
    z[0, 5:] = mask                      # five answers allowed, at the front
    z[1, :-3] = mask                     # three, at the end
    z[2] = mask                          # none: all alike
    z[3] = -mask
    z[4, vocab // 2:] = mask             # half the row
    z[5] = mask
    z[5, vocab // 3] = -mask             # one far above the others
    z[6] = abs(mask) * (2.0 * torch.rand(vocab, generator=gen, dtype=torch.float64) - 1.0)
    z[7, ::2] = mask                     # every other
    z = z.to(getattr(torch, kind))
    t = np.array([3, vocab - 2, vocab // 2, vocab - 1, 1, vocab // 3, 0, 1])
    # a token without a probability has a log-probability whose steps in f32
    # are as large as the mask's: its ratio to another one says nothing
    lp = Policy(f64(z), t, temperature=temperature).logps
    return z, np.where(lp > -20.0, t, z.double().argmax(1).numpy())


@pytest.mark.parametrize("mask", [-1e5, -1e6, -1e9, 1e9, -1e10, -1e12, -1e18, -1e20, -1e30, -1e38])
@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
@pytest.mark.parametrize("vocab", [9, 300, 5003, 40_003])
def test_masks_by_a_constant(vocab, kind, mask):
    z, t = _mask_rows(vocab, mask, kind)
    _check(z, t, repeat=20 if vocab > 40_000 else 0)


@pytest.mark.parametrize("temperature", [1.0, 0.05, 1e-4, 1e-5, 1e-6])
@pytest.mark.parametrize("mask", [-1e4, -65504.0, 3e4])
@pytest.mark.parametrize("vocab", [300, 5003, 90_001])
def test_masks_by_a_constant_in_half_precision(vocab, mask, temperature):
    """(Its range takes a low temperature to get as far.)"""
    z, t = _mask_rows(vocab, mask, "float16", temperature)
    _check(z, t, temperature, grad_scale=temperature, repeat=20 if vocab > 90_000 else 0)


@pytest.mark.parametrize("mask", [-1e10, -1e20])
@pytest.mark.parametrize("kind,vocab", [("float32", 140_003), ("bfloat16", 300_001)])
def test_masks_in_rows_of_many_units(kind, vocab, mask):
    z, t = _mask_rows(vocab, mask, kind)
    _check(z, t)


@pytest.mark.parametrize("side", [-1.0, 1.0])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("vocab", [300, 5003, 40_003, 140_003])
def test_rows_around_a_power_of_two(vocab, kind, side):
    """Maxima m with |m| log2(e) / temperature just below and above powers of
    two from 2^17 to 2^24, so that the units of a row lie on both sides."""
    import torch
    gen = torch.Generator().manual_seed(3)
    for log in (17, 19, 20, 21, 24):
        for by in (0.999, 0.99999, 1.0, 1.00001, 1.001):
            top = 1024.0
            temperature = by * top * LOG2E / 2.0 ** log
            noise = 3.0 * temperature * torch.randn((6, vocab), generator=gen, dtype=torch.float64)
            noise[3:5] -= temperature * torch.arange(vocab) / vocab * 20.0   # a slope
            noise[5, vocab // 2:] -= top / 8
            z = (side * top + noise).to(getattr(torch, kind))
            t = z.double().argmax(1).numpy()
            _check(z, t, temperature, grad_scale=temperature)


@pytest.mark.parametrize("side", [-1.0, 1.0])
@pytest.mark.parametrize("vocab", [1030, 5003, 40_003, 140_003])
def test_units_on_both_sides_of_a_power_of_two(vocab, side):
    """Groups of 64 vectors, which a unit never cuts, whose maxima lie some
    powers of two apart around it: each has a share in the sum."""
    import torch
    top = 1024.0
    gen = torch.Generator().manual_seed(9)
    for log in (19, 20, 21):
        temperature = top * LOG2E / 2.0 ** log
        group = torch.arange(vocab) // 256
        steps = torch.tensor([-4.0, -1.0, 1.5, 0.0, 3.0, -2.0, -6.0])[group % 7]
        z = (side * top + temperature * (steps + 0.2 * torch.randn((4, vocab), generator=gen))).float()
        tops = torch.tensor([float(z[0, group == g].max()) for g in range(int(group[-1]) + 1)])
        powers = (tops / temperature * LOG2E).abs()
        assert powers.min() < 2.0 ** log < powers.max()
        t = np.array([0, 300, 700, vocab - 1])
        _check(z, t, temperature, grad_scale=temperature, repeat=40 if vocab == 40_003 else 0)


@pytest.mark.parametrize("temperature", [1e-30, 1e-20, 1e-9, 1e-4, 1e4, 1e9, 1e20, 1e30])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("vocab", [9, 300, 5003, 40_003])
def test_temperatures(vocab, kind, temperature):
    """Logits of ordinary size, and logits of the temperature's size where the
    type holds them."""
    import torch
    gen = torch.Generator().manual_seed(5)
    for size in (20.0, temperature):
        z = size * torch.randn((6, vocab), generator=gen, dtype=torch.float64)
        z[5] = size                      # all alike
        if size > 6e3 and kind == "float16":
            continue
        z = z.to(getattr(torch, kind))
        _check(z, z.double().argmax(1).numpy(), temperature, grad_scale=temperature)


def test_a_difference_beyond_f32():
    """From the lowest to the highest f32 at the highest temperature: the
    log-probability is finite, though the logits' difference is not."""
    import torch
    z = torch.zeros((2, 700))
    z[:, 0], z[:, 1] = torch.finfo(torch.float32).max, torch.finfo(torch.float32).min
    t = np.array([0, 1])
    got = aspis.token_logps(z.to(device()), _cuda(t)[0], temperature=1e30)
    Policy(f64(z), t, temperature=1e30).check_logps(got)
    assert torch.isfinite(got).all()


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
@pytest.mark.parametrize("vocab", [300, 5003, 40_003])
def test_masked_tokens_have_a_log_probability(vocab, kind):
    """That of a token at the mask: the mask itself, near enough."""
    for mask in (-1e9, -1e10, -1e20, -1e30):
        z, t = _mask_rows(vocab, mask, kind)
        t[:2] = vocab // 2
        t[4], t[7] = vocab - 1, vocab // 2 // 2 * 2
        plain = Policy(f64(z), t)
        plain.check_logps(aspis.token_logps(z.to(device()), _cuda(t)[0]))
        assert (plain.logps[[0, 1, 4, 7]] < mask / 2).all()
