"""The token operators' ways for long and large calls, against the formulas in
64 bits with the bounds of test_gpu_tokens.py, or against smaller calls, whose
results those tests hold: sorted gradients of all types, rows of logits of many
units, sums over many positions, calls of several launches, rows past 2^32
elements, calls at once and graphs that share a workspace."""
import math

import numpy as np
import pytest

from paper_2108_02416_amd import aspis

from _helpers import device
from _tokens import Policy, f64, kept
from test_gpu_tokens import (KINDS, _bits, _check_embed_grad, _cuda, _equal, _model, _padded, _randn,
                             _results, _same, _step, _tokens, _type)

pytestmark = pytest.mark.gpu


# ------------------------------------------------- gradients by sorted tokens

def _with_a_common_one(n, vocab, seed):
    """Half of the tokens are one: its rows are summed in many pieces."""
    t, tokens = _tokens(n, vocab, seed=seed, how="uniform")
    rng = np.random.default_rng(seed)
    common = rng.permutation(n)[:n // 2]
    t[common] = vocab // 3
    tokens[_cuda(common)[0]] = vocab // 3
    return t, tokens


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("kind,to", [(k, t) for k in KINDS for t in KINDS])
@pytest.mark.parametrize("n,vocab,d", [(1100, 60, 37), (1100, 2000, 130), (17_000, 60, 130),
                                       (17_000, 9000, 37)])
def test_sorted_gradients_of_all_types(n, vocab, d, kind, to, accumulate):
    grad, _ = _padded(_randn((n, d), kind, seed=d), 3, 1)
    t, tokens = _with_a_common_one(n, vocab, seed=n + vocab)
    out, buf = _padded(_randn((vocab, d), to, seed=9), 5, 1)
    _check_embed_grad(grad, t, tokens, vocab, out, 0.7, accumulate, to)
    out.fill_(7.0)
    assert (f64(buf) == 7.0).all()


@pytest.mark.parametrize("n", [300, 2000, 20_000, 40_000])
@pytest.mark.parametrize("kind", KINDS)
def test_rows_without_a_token_are_not_read(n, kind):
    """NaN in the rows of tokens outside the table and where rows end."""
    import torch
    vocab, d = 20, 75
    grad, _ = _padded(_randn((n, d), kind, seed=1), 9, fill=math.nan)
    t, tokens = _with_a_common_one(n, vocab, seed=2)
    plain = grad.clone()
    grad[(tokens < 0) | (tokens >= vocab)] = math.nan
    got = aspis.embed_grad(grad, tokens, vocab)
    assert torch.isfinite(got).all()
    assert _same(got, aspis.embed_grad(plain, tokens, vocab))


# -------------------------------------------- long rows and many of them

@pytest.mark.parametrize("kind,vocab", [("float32", 140_003), ("float32", 400_001), ("bfloat16", 300_001),
                                        ("float16", 300_007), ("float32", 1 << 24), ("bfloat16", 1 << 24)])
def test_rows_of_many_units(kind, vocab):
    """More units than a wave has lanes: each lane joins several first."""
    import torch
    gen = torch.Generator().manual_seed(vocab)
    rows = 6 if vocab < 1 << 24 else 3
    z = (2.0 * torch.randn((rows, vocab), generator=gen)).to(_type(kind))
    z[0, : 3 * vocab // 4] = -math.inf
    z[1, vocab // 5] = 90.0
    z[2, vocab - 3] = 300.0              # far above all others, in the last unit
    if rows > 3:
        z[3, 1000:] = -math.inf
        z[4, vocab // 2:] += 60.0
    t = z.float().argmax(1).numpy()
    t[0] = vocab - 1
    lp = Policy(f64(z), t).logps
    old, ref = (lp - 0.05).astype(np.float32), (lp + 0.1).astype(np.float32)
    adv, w = np.linspace(-1, 1, rows).astype(np.float32), np.full(rows, 0.25, np.float32)
    plain = Policy(f64(z), t, old, adv, w, ref, kl=0.05)
    logits, tokens, old, adv, w, ref = _cuda(z, t, old, adv, w, ref)
    plain.check_logps(aspis.token_logps(logits, tokens))
    grad = torch.empty_like(logits)
    bufs = aspis.policy_loss(logits, tokens, old, adv, w, ref=ref, kl=0.05, grad=grad)
    plain.check_logps(bufs.logps)
    plain.check_sums(bufs.sums)
    plain.check_grad(grad, kind)
    aspis.policy_loss(logits, tokens, old, adv, w, ref=ref, kl=0.05, grad=logits)
    assert _same(logits, grad)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("kind,vocab", [("float32", 140_003), ("bfloat16", 300_001)])
def test_nan_and_infinity_in_any_unit(kind, vocab, bad):
    import torch
    places = [0, vocab // 3, vocab // 2 + 1, vocab - 1]
    z = torch.zeros((5, vocab), dtype=_type(kind), device=device())
    for i, at in enumerate(places):
        z[i, at] = bad
    got = aspis.token_logps(z, torch.full((5,), 7, device=device())).tolist()
    assert all(math.isnan(g) for g in got[:4]) and abs(got[4] + math.log(vocab)) < 1e-5


@pytest.mark.parametrize("rows", [8192, 8193, 12_289, 20_000, 262_144, 300_001])
def test_sums_over_many_positions(rows):
    import torch
    rng = np.random.default_rng(rows)
    z = torch.from_numpy(rng.standard_normal((rows, 3))).float()
    t = rng.integers(0, 3, rows)
    lp = Policy(f64(z), t).logps
    ratio = np.exp(rng.normal(0, 0.2, rows))
    for border in (0.8, 1.2):            # off the clip's borders
        ratio = np.where(np.abs(ratio / border - 1) < 1e-3, ratio * 1.01, ratio)
    old, ref = (lp - np.log(ratio)).astype(np.float32), (lp + 0.2).astype(np.float32)
    adv = rng.standard_normal(rows).astype(np.float32)
    w = np.where(rng.random(rows) < 0.3, 0.0, rng.random(rows) / rows).astype(np.float32)
    plain = Policy(f64(z), t, old, adv, w, ref, kl=0.1)
    logits, tokens, old, adv, w, ref = _cuda(z, t, old, adv, w, ref)
    grad = torch.empty_like(logits)
    bufs = aspis.policy_loss(logits, tokens, old, adv, w, ref=ref, kl=0.1, grad=grad)
    plain.check_sums(bufs.sums)
    plain.check_logps(bufs.logps)
    plain.check_grad(grad, "float32")


# --------------------------------------------- several launches, far rows

def _window(x, a, b, p, seed, offset, residual=None):
    """The rows a to b of a call, by a call of their own."""
    return aspis.dropout(x[a:b], p, seed, offset=offset + a * x.shape[1],
                         residual=None if residual is None else residual[a:b])


def test_dropout_in_several_launches():
    """More than 2^30 rows that are not one after the other."""
    import torch
    rows, offset = (1 << 30) + 77, 3
    buf = torch.empty((rows, 2), dtype=torch.bfloat16, device=device())
    words, step = buf.view(torch.int16).view(-1), 1 << 28
    for a in range(0, len(words), step):     # positive and finite, many kinds
        part = words[a:a + step]
        part.copy_(torch.arange(a, a + len(part), device=device()) % 16_001)
    x, residual = buf[:, :1], buf[:, 1:]
    for res in (None, residual):
        out = aspis.dropout(x, 0.3, 5, offset=offset, residual=res)
        for a in range(0, rows, 1 << 27):
            b = min(rows, a + (1 << 27))
            assert torch.equal(out[a:b], _window(x, a, b, 0.3, 5, offset, res)), a
        del out
    ones = torch.ones_like(x)
    out = aspis.dropout(ones, 0.3, 5, offset=offset)
    for a in (0, (1 << 30) - 50, rows - 60):
        keep = kept(60, 0.3, 5, offset + a)
        assert ((out[a:a + 60, 0] != 0).cpu().numpy() == keep).all()


def test_dropout_of_more_than_2_to_33_elements_in_a_row():
    import torch
    n, offset = (1 << 33) + 11, 5
    x = torch.ones((1, n), dtype=torch.bfloat16, device=device())
    aspis.dropout(x, 0.25, -3, offset=offset, out=x)
    for a in (0, (1 << 31) - 9, (1 << 32) - 9, (1 << 33) - 9, n - 20):
        b = min(n, a + 20)
        assert ((x[0, a:b] != 0).cpu().numpy() == kept(b - a, 0.25, -3, offset + a)).all(), a
    for a in ((1 << 31) - 12_345, (1 << 33) - 54_321):
        one = torch.ones((1, 54_332), dtype=torch.bfloat16, device=device())
        assert torch.equal(x[:, a:a + 54_332], aspis.dropout(one, 0.25, -3, offset=offset + a))


def _far(x, ld):
    """The rows of x, ld elements apart; what is between them is not touched."""
    import torch
    to = torch.empty((len(x) - 1) * ld + x.shape[1], dtype=x.dtype, device=x.device)
    view = to.as_strided((len(x), x.shape[1]), (ld, 1))
    return view.copy_(x)


@pytest.mark.parametrize("n,vocab,d", [(5, 5, 300), (300, 5, 130), (300, 300, 37)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradients_of_rows_past_32_bits(n, vocab, d, accumulate):
    """In one launch, and sorted; rows of the gradient and of the table."""
    x, before = _randn((n, d), "bfloat16", seed=1), _randn((vocab, d), seed=2)
    t = np.arange(n) % vocab
    tokens, = _cuda(t)
    far, out = _far(x, (1 << 32) // (n - 1) + 8), _far(before, (1 << 32) // (vocab - 1) + 12)
    want = before.clone()
    aspis.embed_grad(x, tokens, vocab, scale=0.5, out=want, accumulate=accumulate)
    aspis.embed_grad(far, tokens, vocab, scale=0.5, out=out, accumulate=accumulate)
    assert _same(out, want)


def test_lookups_and_dropout_of_rows_past_32_bits():
    import torch
    n, d = 300, 1003
    ld = (1 << 32) // (n - 1) + 9
    table = _randn((n, d), "float16", seed=1)
    tokens = torch.randperm(n, generator=torch.Generator().manual_seed(1)).to(device())
    out = _far(torch.zeros_like(table), ld)
    aspis.embed(table, tokens, out=out)
    assert torch.equal(out, table[tokens])
    want = aspis.dropout(table[tokens], 0.4, 8, offset=1, residual=table)
    assert _same(aspis.dropout(out, 0.4, 8, offset=1, residual=table, out=out), want)


@pytest.mark.parametrize("kind,rows,vocab", [("bfloat16", 300, 515), ("float16", 300, 9001),
                                             ("float32", 9, 70_003), ("bfloat16", 9, 90_001)])
def test_logits_of_rows_past_32_bits(kind, rows, vocab):
    import torch
    z = _randn((rows, vocab), kind, seed=3)
    tokens = torch.arange(rows, device=device()) * 7 % vocab
    old, v = torch.full((rows,), -7.0, device=device()), torch.ones(rows, device=device())
    want = torch.empty_like(z)
    bufs = aspis.policy_loss(z, tokens, old, v, v, ref=old, kl=0.1, clip=(0.2, 1e4), grad=want)
    far = _far(z, (1 << 32) // (rows - 1) + 11)
    assert _same(aspis.token_logps(far, tokens), bufs.logps)
    got = aspis.policy_loss(far, tokens, old, v, v, ref=old, kl=0.1, clip=(0.2, 1e4), grad=far)
    assert _same(far, want) and _same(got.logps, bufs.logps) and _same(got.sums, bufs.sums)


# ------------------------------------------------- calls at once, graphs

def test_steps_on_two_streams_at_once():
    """With workspaces and results of their own."""
    import torch
    models = [_model(n=2500, vocab=3000, d=72, seed=s) for s in (0, 20)]
    for s in models:
        _step(s, 3)
    want = [_results(s) for s in models]
    streams = [torch.cuda.Stream() for _ in models]
    for turn in range(3):
        for stream in streams:
            stream.wait_stream(torch.cuda.current_stream())
        for _ in range(4):
            for s, stream in zip(models, streams):
                with torch.cuda.stream(stream):
                    _step(s, 3)
        torch.cuda.synchronize()
        assert all(_equal(_results(s), w) for s, w in zip(models, want)), turn


def test_graphs_that_share_workspaces():
    """Replayed one after the other on a stream, eager work in between: no
    call leaves anything in a workspace for another."""
    import torch
    models = [_model(seed=0), _model(n=2500, vocab=400, d=64, seed=50)]
    for key in ("pw", "ew"):
        ws = max((s[key] for s in models), key=lambda w: w.numel())
        for s in models:
            s[key] = ws
    seeds = [torch.tensor([5], device=device()), torch.tensor([6], device=device())]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for s, seed in zip(models, seeds):
            _step(s, seed)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graphs = []
    for s, seed in zip(models, seeds):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            _step(s, seed)
        graphs.append(g)
    for turn in range(4):
        for i, s in enumerate(models):
            s["tokens"].copy_(_tokens(len(s["tokens"]), s["vocab"], seed=10 * turn + i)[1])
            seeds[i].fill_(100 * turn + i)
        for g in (*graphs, *graphs[::-1]):
            g.replay()
        torch.cuda.synchronize()
        got = [_results(s) for s in models]
        for i, s in enumerate(models):
            for key in ("pw", "ew"):
                s[key].fill_(255)
            _step(s, 100 * turn + i)
            torch.cuda.synchronize()
            assert _equal(_results(s), got[i]), (turn, i)
