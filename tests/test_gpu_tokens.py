"""The token operators on the GPU against plain formulas in 64 bits.

Tolerances, from the formulas (U = 2^-24, half an f32 ulp relative to the
value):
- embed: the scale's rounding and the product's, then the result's type.
- embed_grad: a sum of k terms in f32, whatever its order, is off by at most
  k U of the sum of their magnitudes; the scale, the product and the addition
  to what was there add U each, then the result's type.
- dropout: the same f32 operations on the host, bit for bit.
- log-probabilities and the policy loss: _tokens.Policy.
"""
import math

import numpy as np
import pytest

from paper_2108_02416_amd import aspis

from _helpers import device
from _tokens import (HALF_ULP, TINY, U, Policy, embed_sums, embedded, f64, kept, policy_inputs,
                     softmax_loss)

pytestmark = pytest.mark.gpu

KINDS = ["float32", "bfloat16", "float16"]


def _type(kind):
    import torch
    return getattr(torch, kind)


def _randn(shape, kind="float32", seed=0, scale=1.0):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=gen, device=device()).mul_(scale).to(_type(kind))


def _padded(x, pad, before=0, fill=7.0):
    """x as rows of a wider buffer, `before` elements into it; the buffer."""
    import torch
    rows, d = x.shape
    buf = torch.full((before + rows * (d + pad),), fill, dtype=x.dtype, device=x.device)
    view = buf[before:].view(rows, d + pad)[:, :d]
    view.copy_(x)
    return view, buf


def _tokens(n, vocab, seed=0, how="zipf", kind="int64"):
    import torch
    rng = np.random.default_rng(seed)
    if how == "zipf":
        t = np.floor(np.exp(rng.random(n) * math.log(vocab + 1))).astype(np.int64) - 1
    elif how == "uniform":
        t = rng.integers(0, vocab, n)
    elif how == "one":
        t = np.full(n, vocab // 2)
    elif how == "none":
        t = np.full(n, -1)
    elif how == "distinct":
        t = rng.permutation(vocab)[:n]
    if how in ("zipf", "uniform") and n > 4:
        t[rng.random(n) < 0.1] = -1
        t[n // 2] = vocab
        t[n // 3] = 2 ** 31 - 1 if kind == "int32" else 2 ** 40 + 1
        t[n // 4] = -(2 ** 31) if kind == "int32" else -(2 ** 62)
    return t, torch.from_numpy(t.astype(kind)).to(device())


def _bits(t):
    import torch
    return t.detach().contiguous().view(
        torch.int32 if t.dtype == torch.float32 else torch.int16).cpu().numpy()


# ------------------------------------------------------------------ embed

@pytest.mark.parametrize("index", ["int64", "int32"])
@pytest.mark.parametrize("kind,to", [(k, t) for k in KINDS for t in KINDS])
@pytest.mark.parametrize("n,vocab,d", [(1, 5, 64), (3, 1, 1), (7, 100, 3), (33, 50, 257),
                                       (130, 37, 2048), (5, 9, 2501), (1000, 300, 8), (1, 3, 4100)])
def test_embed(n, vocab, d, kind, to, index):
    import torch
    table, _ = _padded(_randn((vocab, d), kind, seed=d), 3, 1)
    t, tokens = _tokens(n, vocab, seed=n, kind=index, how="uniform")
    scale = math.sqrt(d)
    out, buf = _padded(torch.zeros((n, d), dtype=_type(to), device=device()), 5, 1)
    got = aspis.embed(table, tokens, scale=scale, out=out)
    assert got is out
    want = embedded(f64(table), t, scale)
    tol = np.abs(want) * (2 * U + HALF_ULP[to]) * 1.01 + TINY[to]
    assert (np.abs(f64(out) - want) <= tol).all()
    out.fill_(7.0)
    assert (f64(buf) == 7.0).all()   # nothing outside the rows was written


@pytest.mark.parametrize("kind", KINDS)
def test_embed_without_scale_copies(kind):
    table = _randn((40, 100), kind, seed=1)
    t, tokens = _tokens(60, 40, seed=2, how="uniform")
    got = aspis.embed(table, tokens.view(3, 20))
    assert got.shape == (3, 20, 100) and got.dtype == table.dtype
    want = embedded(f64(table), t, 1.0)
    assert (f64(got).reshape(60, 100) == want).all()


def test_embed_beyond_32_bits():
    """Rows whose first element's index is past 2^32 in the table."""
    import torch
    d, vocab = 1 << 20, 4200
    table = torch.empty((vocab, d), dtype=torch.bfloat16, device=device())
    rows = [0, 4095, 4096, 4199]
    for r in rows:
        table[r] = float(r % 251)
    tokens = torch.tensor([*rows, -1], device=device())
    got = aspis.embed(table, tokens)
    for i, r in enumerate(rows):
        assert (got[i] == float(r % 251)).all()
    assert (got[4] == 0).all()


# ------------------------------------------------------------- embed_grad

def _check_embed_grad(grad, t, tokens, vocab, out, scale=1.0, accumulate=False, to="float32"):
    before = f64(out)
    got = aspis.embed_grad(grad, tokens, vocab, scale=scale, out=out, accumulate=accumulate)
    assert got is out
    sums, sizes, count = embed_sums(f64(grad).reshape(-1, grad.shape[-1]), t, vocab)
    want = scale * sums + (before if accumulate else 0.0)
    tol = abs(scale) * sizes * U * (count[:, None] + 3) * 1.01 + np.abs(want) * (
        U * accumulate + HALF_ULP[to]) * 1.01 + TINY[to]
    if accumulate:   # rows without a token are left alone, bit for bit
        tol[count == 0] = 0.0
    else:
        assert (want[count == 0] == 0).all()
        tol[count == 0] = 0.0
    bad = ~(np.abs(f64(out) - want) <= tol)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist(), f64(out)[bad][:4],
                           want[bad][:4])


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("kind,to", [(k, t) for k in KINDS for t in KINDS])
@pytest.mark.parametrize("n,vocab,d", [(1, 5, 64), (3, 1, 1), (7, 100, 3), (9, 50, 257),
                                       (515, 99, 300), (130, 200, 2048), (70, 9, 2501)])
def test_embed_grad_types(n, vocab, d, kind, to, accumulate):
    grad, _ = _padded(_randn((n, d), kind, seed=d), 3, 1)
    t, tokens = _tokens(n, vocab, seed=n)
    out, buf = _padded(_randn((vocab, d), to, seed=9), 5, 1)
    _check_embed_grad(grad, t, tokens, vocab, out, math.sqrt(d), accumulate, to)
    out.fill_(7.0)
    assert (f64(buf) == 7.0).all()


@pytest.mark.parametrize("how", ["zipf", "uniform", "one", "none", "distinct"])
@pytest.mark.parametrize("n", [1, 8, 9, 16, 17, 64, 255, 257, 767, 768, 769, 1024, 1025, 2047, 2048, 2049, 4096, 4097, 5000, 32_768,
                               33_000, 40_001])
def test_embed_grad_tokens(n, how):
    import torch
    vocab, d = 40_003 if how == "distinct" else 3001, 5
    grad = _randn((n, d), seed=n)
    t, tokens = _tokens(n, vocab, seed=n, how=how, kind="int32")
    out = torch.full((vocab, d), 7.0, device=device())
    _check_embed_grad(grad, t, tokens, vocab, out)


@pytest.mark.parametrize("n", [100, 700, 1024, 1500, 6000])
@pytest.mark.parametrize("vocab,d", [(7, 513), (300, 1030), (20_001, 257), (130_000, 520)])
@pytest.mark.parametrize("how", ["zipf", "uniform", "one"])
def test_embed_grad_shapes(n, vocab, d, how):
    """Every number of rows a workgroup takes, several slabs of columns, and
    columns after the last vector."""
    import torch
    for kind, accumulate in (("bfloat16", False), ("float32", True)):
        grad = _randn((n, d), kind, seed=n)
        t, tokens = _tokens(n, vocab, seed=n + d, how=how)
        out = _randn((vocab, d), seed=1) if accumulate else torch.full((vocab, d), 7.0,
                                                                       device=device())
        _check_embed_grad(grad, t, tokens, vocab, out, 0.7, accumulate)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("n,vocab", [(256, 1), (257, 1), (256, 32), (257, 32), (257, 33), (768, 95),
                                     (768, 96), (16_384, 4), (16_384, 900), (16_385, 4), (16_385, 900)])
def test_embed_grad_where_another_way_begins(n, vocab, accumulate):
    import torch
    d = 130
    grad = _randn((n, d), "bfloat16", seed=n)
    t, tokens = _tokens(n, vocab, seed=n + vocab, how="uniform")
    out = _randn((vocab, d), seed=1) if accumulate else torch.full((vocab, d), 7.0, device=device())
    _check_embed_grad(grad, t, tokens, vocab, out, 0.7, accumulate)


@pytest.mark.parametrize("how", ["zipf", "one"])
def test_embed_grad_of_three_rounds_of_merging(how):
    """More than 16 * 16 runs of 2,048 tokens."""
    import torch
    n, vocab, d = 530_011, 77, 2
    grad = _randn((n, d), "bfloat16", seed=3)
    t, tokens = _tokens(n, vocab, seed=4, how=how)
    _check_embed_grad(grad, t, tokens, vocab, torch.empty((vocab, d), device=device()), 0.5)


@pytest.mark.parametrize("vocab", [(1 << 21) - 1, (1 << 22) - 2, (1 << 22) - 1, (1 << 22) + 5, 1 << 24])
def test_embed_grad_of_many_rows(vocab):
    """Either side of where a token and its place in a run fit 32 bits."""
    import torch
    n, d = 3000, 1
    grad = _randn((n, d), seed=5)
    t, tokens = _tokens(n, vocab, seed=6, how="uniform")
    t[:3], tokens[:3] = vocab - 1, vocab - 1
    _check_embed_grad(grad, t, tokens, vocab, torch.full((vocab, d), 3.0, device=device()))


def test_embed_grad_of_no_tokens():
    import torch
    grad = torch.empty((0, 6), device=device())
    tokens = torch.empty(0, dtype=torch.int64, device=device())
    out = torch.full((5, 6), 7.0, device=device())
    aspis.embed_grad(grad, tokens, 5, out=out, accumulate=True)
    assert (out == 7.0).all()
    assert (aspis.embed_grad(grad, tokens, 5) == 0).all()


def test_embed_grad_reads_no_row_without_a_token():
    """NaN and infinities where the token is none, and where rows end."""
    n, vocab, d = 300, 50, 70
    grad, _ = _padded(_randn((n, d), "bfloat16", seed=1), 9, fill=math.nan)
    t, tokens = _tokens(n, vocab, seed=2, how="uniform")
    grad[tokens == -1] = math.nan
    grad[n // 2], grad[n // 3] = math.inf, -math.inf
    import torch
    out = torch.empty((vocab, d), device=device())
    aspis.embed_grad(grad, tokens, vocab, out=out)
    assert torch.isfinite(out).all()


def test_embed_grad_has_the_same_bits_every_time():
    import torch
    n, vocab, d = 20_011, 301, 130
    grad = _randn((n, d), seed=1)
    _, tokens = _tokens(n, vocab, seed=2)
    first = _bits(aspis.embed_grad(grad, tokens, vocab))
    for i in range(4):
        moved, _ = _padded(grad, i, i)   # another address and stride
        ws = aspis.embed_workspace(moved, tokens, vocab)
        ws.fill_(255)
        kind = torch.int32 if i % 2 else torch.int64
        limited = tokens.clamp(-1, vocab).to(kind)
        assert (_bits(aspis.embed_grad(moved, limited, vocab, ws=ws)) == first).all()


def test_embed_grad_against_differences():
    """The directional derivative of <w, embed(table)> is what the gradient
    says (the loss is linear: exact up to rounding)."""
    import torch
    n, vocab, d = 40, 11, 7
    _, tokens = _tokens(n, vocab, seed=1)
    w, step = _randn((n, d), seed=2), _randn((vocab, d), seed=3)
    got = aspis.embed_grad(w, tokens, vocab, scale=1.5)
    rise = (w.double() * aspis.embed(step, tokens, scale=1.5).double()).sum()
    assert abs(float((got.double() * step.double()).sum() - rise)) <= 1e-5 * n * d
    assert torch.equal(aspis.embed(step, tokens)[tokens < 0], torch.zeros_like(w)[tokens < 0])


# ---------------------------------------------------------------- dropout

def _dropped(x, p, seed, offset=0, residual=None):
    """The call's operations in f32 on the host; x a tensor [rows, d]."""
    import torch
    limit = round(p * 65536)
    scale = np.float32(65536 / (65536 - limit)) if limit < 65536 else np.float32(0)
    keep = torch.from_numpy(kept(x.numel(), p, seed, offset).reshape(x.shape))
    v = torch.where(keep, x.float().cpu() * float(scale), torch.zeros(x.shape))
    if residual is not None:
        v = v + residual.float().cpu()
    return v.to(x.dtype)


def _same(got, want):
    return (_bits(got) == _bits(want)).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,d,pad", [(1, 1, 0), (1, 7, 0), (1, 8, 0), (3, 5, 2), (40, 1, 1),
                                        (17, 33, 0), (5, 2049, 63), (2, 30_001, 1), (1, 100_003, 0),
                                        (300, 2056, 8)])
@pytest.mark.parametrize("offset", [0, 3, 2 ** 35 + 5, 2 ** 64 - 11])
def test_dropout(rows, d, pad, kind, offset):
    import torch
    x, _ = _padded(_randn((rows, d), kind, seed=d), pad, 1)
    res, _ = _padded(_randn((rows, d), kind, seed=d + 1), 2 * pad)
    out, buf = _padded(torch.zeros((rows, d), dtype=_type(kind), device=device()), 3 * pad, 3)
    seed = 0x9876543210ABCDEF
    assert aspis.dropout(x, 0.3, seed, offset=offset, out=out) is out
    assert _same(out, _dropped(x, 0.3, seed, offset))
    aspis.dropout(x, 0.3, seed, offset=offset, residual=res, out=out)
    assert _same(out, _dropped(x, 0.3, seed, offset, res))
    out.fill_(7.0)
    assert (f64(buf) == 7.0).all()
    want = _dropped(x, 0.3, seed, offset, res)
    kept_res = res.clone()
    aspis.dropout(x, 0.3, seed, offset=offset, residual=res, out=res)   # onto the residual
    assert _same(res, want)
    aspis.dropout(x, 0.3, seed, offset=offset, residual=kept_res, out=x)   # in place
    assert _same(x, want)


@pytest.mark.parametrize("p", [0.0, 2.0 ** -17, 2.0 ** -16, 0.1, 0.5, 1.0 - 2.0 ** -16, 1.0])
def test_dropout_shares(p):
    x = _randn((64, 1000), seed=1)
    got = aspis.dropout(x, p, 5)
    assert _same(got, _dropped(x, p, 5))
    if p <= 2.0 ** -17:   # rounds to none (ties to even)
        assert _same(got, x)
    if p == 1.0:
        assert (got == 0).all()
    share = float((got == 0).float().mean())
    assert abs(share - p) <= 5 * math.sqrt(max(p * (1 - p), 1e-9) / x.numel()) + 2.0 ** -17


def test_dropout_drops_nan_and_infinities():
    import torch
    for bad in (math.nan, math.inf, -math.inf):
        x = torch.full((7, 333), bad, device=device())
        keep = torch.from_numpy(kept(x.numel(), 0.4, 3, 0).reshape(x.shape)).to(device())
        got = aspis.dropout(x, 0.4, 3)
        assert (got[~keep] == 0).all() and not torch.isfinite(got[keep]).any()


def test_dropout_of_shards_is_dropout_of_the_whole():
    import torch
    x = _randn((1, 10_007), "bfloat16", seed=2)
    whole = aspis.dropout(x, 0.25, -5, offset=77)
    cuts = [0, 1, 9, 4096, 4103, 10_007]
    parts = [aspis.dropout(x[:, a:b], 0.25, -5, offset=77 + a) for a, b in zip(cuts, cuts[1:])]
    assert _same(torch.cat(parts, 1), whole)
    # and the gradient is the same mask on what comes back
    ones = torch.ones_like(x)
    mask = aspis.dropout(ones, 0.25, -5, offset=77)
    assert ((mask == 0) == (whole == 0)).all() and set(mask.unique().tolist()) == {0.0, 1.3359375}


def test_dropout_seed_on_the_device():
    import torch
    x = _randn((5, 100), seed=1)
    for seed in (3, -7, 2 ** 63 - 1):
        at = torch.tensor([seed], device=device())
        assert _same(aspis.dropout(x, 0.5, at), aspis.dropout(x, 0.5, seed))


# ---------------------------------------- log-probabilities, policy loss

SIZES = [(1, 1), (3, 2), (5, 8), (4, 9), (64, 255), (9, 1001), (33, 4097), (3, 8192), (5, 8193),
         (7, 32_003), (300, 515), (2, 70_001)]


def _cuda(*arrays):
    import torch
    return [torch.from_numpy(a).to(device()) if isinstance(a, np.ndarray) else a.to(device())
            for a in arrays]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,vocab", SIZES)
def test_token_logps(rows, vocab, kind):
    z, t, *_ = policy_inputs(rows, vocab, seed=vocab, kind=kind)
    for pad, temperature in ((0, 1.0), (3, 0.7)):
        logits, _ = _padded(z.to(device()), pad, pad % 2)
        ref = Policy(f64(z), t, temperature=temperature)
        for index in ("int64", "int32"):
            tokens, = _cuda(t.astype(index))
            ref.check_logps(aspis.token_logps(logits, tokens, temperature=temperature))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,vocab", SIZES)
@pytest.mark.parametrize("kl", [0.0, 0.1])
def test_policy_loss(rows, vocab, kind, kl):
    import torch
    scale = 4096.0 if kind == "float16" else 1.0
    for pad, temperature in ((0, 1.0), (3, 1.3)):
        clip = (0.2, 0.3)
        z, t, old, adv, w, refs = policy_inputs(rows, vocab, seed=rows + pad, kind=kind,
                                                temperature=temperature, clip=clip)
        t[rows // 2] = vocab if pad else -1
        logits, _ = _padded(z.to(device()), pad, pad % 2)
        grad, buf = _padded(torch.zeros_like(logits), 2 * pad, 3)
        plain = Policy(f64(z), t, old, adv, w, refs if kl or pad else None, clip, kl, temperature,
                       scale)
        tokens, old, adv, w, refs = _cuda(t, old, adv, w, refs)
        args = dict(ref=refs if kl or pad else None, clip=clip, kl=kl, temperature=temperature,
                    grad_scale=scale)
        bufs = aspis.policy_loss(logits, tokens, old, adv, w, grad=grad, **args)
        plain.check_logps(bufs.logps)
        plain.check_sums(bufs.sums)
        plain.check_grad(grad, kind)
        first = _bits(grad)
        grad.fill_(7.0)
        assert (f64(buf) == 7.0).all()
        alone = aspis.policy_loss(logits, tokens, old, adv, w, **args)   # no gradient
        assert _same(alone.sums, bufs.sums) and _same(alone.logps, bufs.logps)
        aspis.policy_loss(logits, tokens, old, adv, w, grad=logits, **args)   # in place
        assert (_bits(logits) == first).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("vocab", [40, 300, 4099, 9000, 40_000, 90_001])
def test_rows_wherever_they_begin(vocab, kind):
    """Logits and gradient at every place in a 16-byte block, many rows and
    few: the same bits, and nothing written beside the rows."""
    import torch
    rows = 200
    z, t, old, adv, w, refs = policy_inputs(rows, vocab, seed=2, kind=kind)
    t[::7] = np.arange(len(t[::7])) % min(vocab, 9)            # in the first vectors
    t[1::7] = vocab - 1 - np.arange(len(t[1::7])) % min(vocab, 9)   # and in the last
    tokens, old, adv, w, refs = _cuda(t, old, adv, w, refs)
    plain = None
    places = range(8 if kind != "float32" else 4)
    for at in places:
        logits, _ = _padded(z.to(device()), 16, at)
        for to in ((at + 3) % len(places), at):
            grad, buf = _padded(torch.zeros_like(logits), 8, to)
            bufs = aspis.policy_loss(logits, tokens, old, adv, w, ref=refs, kl=0.1, grad=grad)
            got = _bits(grad), _bits(bufs.logps)
            if plain is None:
                plain = got
            assert (got[0] == plain[0]).all() and (got[1] == plain[1]).all(), (at, to)
            grad.fill_(7.0)
            assert (f64(buf) == 7.0).all()
            few = aspis.policy_loss(logits[:9], tokens[:9], old[:9], adv[:9], w[:9], ref=refs[:9],
                                    kl=0.1, grad=grad[:9])
            assert (_bits(grad[:9]) == plain[0][:9]).all() and (_bits(few.logps) == plain[1][:9]).all()
            grad.fill_(7.0)
            assert (f64(buf) == 7.0).all()


@pytest.mark.parametrize("rows,vocab", [(700, 33), (600, 2500), (520, 9000), (300, 40_003)])
@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
def test_policy_loss_of_many_rows(rows, vocab, kind):
    import torch
    z, t, old, adv, w, refs = policy_inputs(rows, vocab, seed=1, kind=kind)
    plain = Policy(f64(z), t, old, adv, w, refs, kl=0.05)
    logits, tokens, old, adv, w, refs = _cuda(z, t, old, adv, w, refs)
    grad = torch.empty_like(logits)
    bufs = aspis.policy_loss(logits, tokens, old, adv, w, ref=refs, kl=0.05, grad=grad)
    plain.check_logps(bufs.logps)
    plain.check_sums(bufs.sums)
    plain.check_grad(grad, kind)
    plain = Policy(f64(z), t)
    plain.check_logps(aspis.token_logps(logits, tokens))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("vocab", [300, 20_000, 70_000])
def test_masked_logits(vocab, kind):
    """Logits at -inf and at the type's lowest value, whole parts of a row
    and all of it."""
    import torch
    low = torch.finfo(_type(kind)).min
    z = torch.randn((6, vocab), generator=torch.Generator().manual_seed(1)).to(_type(kind))
    z[0, : vocab // 2] = -math.inf
    z[1, vocab // 2:] = low
    z[2] = low                       # uniform
    z[3, : vocab - 1] = -math.inf    # one token left
    z[4, 1:] = low
    z[4, 0] = torch.finfo(_type(kind)).max
    z[5] = -math.inf                 # nothing left
    t = np.array([vocab - 1, 0, vocab // 3, vocab - 1, 0, 0])
    old, adv = np.full(6, -3.0, np.float32), np.ones(6, np.float32)
    logits, tokens, o, a = _cuda(z, t, old, adv)
    w = torch.ones(6, device=device())
    got = aspis.token_logps(logits, tokens)
    plain = Policy(f64(z[:5]), t[:5])
    plain.check_logps(got[:5])
    assert float(got[3]) == 0.0 and math.isnan(float(got[5]))
    assert abs(float(got[2]) + math.log(vocab)) < 1e-4
    w[5] = 0.0                       # left out: no NaN from it
    grad = torch.empty_like(logits)
    bufs = aspis.policy_loss(logits, tokens, o, a, w, clip=(0.2, 1e6), grad=grad)
    plain = Policy(f64(z[:5]), t[:5], old[:5], adv[:5], np.ones(5), clip=(0.2, 1e6))
    assert torch.isfinite(grad).all() and torch.isfinite(bufs.sums).all()
    plain.check_grad(grad[:5], kind)
    plain.check_sums(bufs.sums)
    assert (grad[5] == 0).all()


def test_positions_left_out_are_not_read():
    import torch
    z, t, old, adv, w, refs = policy_inputs(50, 9000, seed=3, kind="bfloat16")
    w[7], t[8] = 0.0, 9000
    out = (w == 0) | (t == 9000)
    z[torch.from_numpy(out)] = math.nan
    for a in (old, adv, refs):
        a[out] = math.nan
    logits, tokens, old, adv, w, refs = _cuda(z, t, old, adv, w, refs)
    grad = torch.empty_like(logits)
    bufs = aspis.policy_loss(logits, tokens, old, adv, w, ref=refs, kl=0.1, grad=grad)
    assert torch.isfinite(bufs.sums).all() and torch.isfinite(grad).all()
    assert (grad[torch.from_numpy(out)] == 0).all() and (bufs.logps[torch.from_numpy(out)] == 0).all()
    w.zero_()   # nothing left at all
    bufs = aspis.policy_loss(logits, tokens, old, adv, w, ref=refs, kl=0.1, grad=grad)
    assert (bufs.sums == 0).all() and (grad == 0).all() and (bufs.logps == 0).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("vocab", [600, 9000, 70_000])
@pytest.mark.parametrize("rise", [20.0, 60.0, 150.0])
def test_a_logit_far_above_the_others(vocab, rise, kind):
    """Wherever it is in a vector: the scale a unit takes is that of other
    elements, or, where a sum says so, of all."""
    import torch
    rows = 24
    z, t, old, adv, w, refs = policy_inputs(rows, vocab, seed=5, kind=kind, masked=0.0)
    at = (np.arange(rows) * 37 + np.arange(rows) * (vocab // rows)) % vocab
    z[np.arange(rows), at] = rise
    t[::2] = at[::2]
    lp = Policy(f64(z), t).logps
    old = (lp - 0.05).astype(np.float32)
    refs = np.maximum(lp + 0.1, -1e4).astype(np.float32)
    plain = Policy(f64(z), t, old, adv, w, refs, kl=0.05)
    logits, tokens, old, adv, w, refs = _cuda(z, t, old, adv, w, refs)
    grad = torch.empty_like(logits)
    bufs = aspis.policy_loss(logits, tokens, old, adv, w, ref=refs, kl=0.05, grad=grad)
    plain.check_logps(bufs.logps)
    plain.check_sums(bufs.sums)
    plain.check_grad(grad, kind)


def test_rows_with_nan_or_infinity_say_so():
    import torch
    z = torch.zeros((4, 12_000), device=device())
    z[0, 11_999], z[1, 0], z[2, 5] = math.nan, math.inf, -math.inf
    tokens = torch.full((4,), 3, device=device())
    got = aspis.token_logps(z, tokens).tolist()
    assert math.isnan(got[0]) and math.isnan(got[1])
    assert all(abs(g + math.log(n)) < 1e-5 for g, n in ((got[2], 11_999), (got[3], 12_000)))


def test_ratios_that_leave_f32():
    """An infinite ratio: clipped for a positive advantage, nothing for none,
    and the loss is infinite for a negative one."""
    import torch
    z = torch.zeros((3, 5), device=device())
    tokens = torch.zeros(3, dtype=torch.int32, device=device())
    old = torch.full((3,), -400.0, device=device())
    for adv, loss in ((1.0, -1.2), (0.0, 0.0), (-1.0, math.inf)):
        a, w = torch.full((3,), adv, device=device()), torch.full((3,), 1 / 3, device=device())
        grad = torch.empty_like(z)
        bufs = aspis.policy_loss(z, tokens, old, a, w, grad=grad)
        got = bufs.sums.tolist()
        assert got[0] == loss or abs(got[0] - loss) < 1e-6
        assert abs(got[2] - (adv > 0)) < 1e-6
        if adv >= 0:
            assert (grad == 0).all()


def test_policy_gradient_against_differences():
    import torch
    rows, vocab, kl, temperature, clip = 6, 11, 0.2, 0.8, (0.2, 0.2)
    z, t, old, adv, w, refs = policy_inputs(rows, vocab, seed=4, masked=0.0, temperature=temperature)
    z = z.double().numpy()
    w = np.linspace(0.1, 1.0, rows).astype(np.float32)
    logits, tokens, o, a, wt, r = _cuda(z.astype(np.float32), t, old, adv, w, refs)
    grad = torch.empty_like(logits)
    bufs = aspis.policy_loss(logits, tokens, o, a, wt, ref=r, clip=clip, kl=kl,
                             temperature=temperature, grad=grad)
    z = f64(logits)
    args = (t, old.astype(float), adv.astype(float), w.astype(float), refs.astype(float), clip, kl,
            temperature)
    assert abs(float(bufs.sums[0]) - softmax_loss(z, *args)) < 1e-5
    h = 1e-5
    for i in range(rows):
        for v in range(vocab):
            up, down = z.copy(), z.copy()
            up[i, v] += h
            down[i, v] -= h
            slope = (softmax_loss(up, *args) - softmax_loss(down, *args)) / (2 * h)
            # h^2 of the third derivative, and f32's roundings
            assert abs(slope - float(grad[i, v])) < 2e-6, (i, v)


# ------------------------------------------------- streams, graphs, refusals

def _step(s, seed):
    """One step of a small model on tokens: its loss and gradients."""
    x = aspis.embed(s["table"], s["tokens"], scale=2.0, out=s["x"])
    y = aspis.dropout(x, 0.2, seed, out=s["y"])
    s["logits"].copy_(y @ s["head"])
    aspis.token_logps(s["logits"], s["targets"], logps=s["old"], ws=s["pw"])
    s["old"].add_(s["shift"])
    aspis.policy_loss(s["logits"], s["targets"], s["old"], s["adv"], s["w"], ref=s["ref"], kl=0.1,
                      grad=s["logits"], bufs=s["bufs"], ws=s["pw"])
    s["dy"].copy_(s["logits"] @ s["head_t"])
    aspis.dropout(s["dy"], 0.2, seed, out=s["dy"])
    aspis.embed_grad(s["dy"], s["tokens"], s["vocab"], scale=2.0, out=s["grad"], ws=s["ew"])


def _model(n=700, vocab=1111, d=72, seed=0):
    import torch
    dev = device()
    s = {"vocab": vocab, "table": _randn((vocab, d), seed=seed + 1), "tokens": _tokens(n, vocab, seed)[1],
         "head": _randn((d, vocab), seed=seed + 2, scale=0.1), "targets": _tokens(n, vocab, seed + 5)[1],
         "adv": _randn((n,), seed=seed + 3), "ref": _randn((n,), seed=seed + 4) * 0.1 - 7.0,
         "w": torch.full((n,), 1.0 / n, device=dev), "shift": _randn((n,), seed=seed + 6, scale=0.2)}
    s["head_t"] = s["head"].t().contiguous()
    for k, shape in (("x", (n, d)), ("y", (n, d)), ("dy", (n, d)), ("logits", (n, vocab)),
                     ("grad", (vocab, d)), ("old", (n,))):
        s[k] = torch.zeros(shape, device=dev)
    s["bufs"] = aspis.PolicyBuffers.empty(n, dev)
    s["pw"], s["ew"] = aspis.policy_workspace(s["logits"]), aspis.embed_workspace(s["x"], s["tokens"], vocab)
    return s


def _results(s):
    return [_bits(s[k]).copy() for k in ("x", "y", "logits", "grad")] + [
        _bits(s["bufs"].sums).copy(), _bits(s["bufs"].logps).copy()]


def _equal(a, b):
    return all((x == y).all() for x, y in zip(a, b))


def test_a_step_against_the_chain_in_64_bits():
    import torch
    s = _model()
    seed = 11
    _step(s, seed)
    table = s["table"].double().cpu().requires_grad_()
    t, targets = s["tokens"].cpu(), s["targets"].cpu()
    vocab, n = s["vocab"], len(t)
    there = ((t >= 0) & (t < vocab)).double()[:, None]
    x = 2.0 * table[t.clamp(0, vocab - 1)] * there
    mask = torch.from_numpy(kept(x.numel(), 0.2, seed, 0).reshape(x.shape)).double()
    y = x * mask * (65536 / (65536 - round(0.2 * 65536)))
    lp = torch.log_softmax(y @ s["head"].double().cpu(), 1)
    used = ((targets >= 0) & (targets < vocab)).double()
    lp = lp.gather(1, targets.clamp(0, vocab - 1)[:, None])[:, 0] * used
    r = torch.exp(lp - lp.detach() - s["shift"].double().cpu())
    adv, ref = s["adv"].double().cpu(), s["ref"].double().cpu()
    d = ref - lp
    loss = (used / n * (0.1 * (d.exp() - 1 - d) - torch.minimum(r * adv, r.clamp(0.8, 1.2) * adv))).sum()
    loss.backward()
    # the products of f32 matrices add d and vocab roundings
    assert abs(float(s["bufs"].sums[0]) - float(loss.detach())) < 1e-4
    want = table.grad
    assert float((s["grad"].double().cpu() - want).abs().max()) <= 2e-5 * float(want.abs().max())


def test_a_step_on_another_stream():
    import torch
    s = _model()
    _step(s, 3)
    want = _results(s)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for k in ("x", "y", "dy", "grad"):
            s[k].fill_(5.0)
        _step(s, 3)
    side.synchronize()
    assert _equal(_results(s), want)


def test_a_step_captured_and_replayed():
    """Two graphs with workspaces of their own, their inputs changed between
    the replays, eager work in between."""
    import torch
    models = [_model(seed=0), _model(n=2500, vocab=400, d=64, seed=50)]
    seeds = [torch.tensor([5], device=device()), torch.tensor([6], device=device())]
    graphs = []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for s, seed in zip(models, seeds):
            _step(s, seed)   # the library of matrix products sets itself up
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for s, seed in zip(models, seeds):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            _step(s, seed)
        graphs.append(g)
    for turn in range(4):
        for i, s in enumerate(models):
            s["tokens"].copy_(_tokens(len(s["tokens"]), s["vocab"], seed=10 * turn + i)[1])
            seeds[i].fill_(100 * turn + i)
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        got = [_results(s) for s in models]
        for i, s in enumerate(models):
            _step(s, 100 * turn + i)
            torch.cuda.synchronize()
            assert _equal(_results(s), got[i]), (turn, i)


def test_refusals():
    import torch
    f, dev = torch.float32, device()
    x, t = torch.zeros((4, 6), device=dev), torch.zeros(4, dtype=torch.int64, device=dev)
    v, long_v = torch.zeros(4, device=dev), torch.zeros(5, device=dev)
    wide = torch.zeros(24, device=dev)
    long, many = torch.zeros((2000, 6), device=dev), torch.zeros(2000, dtype=torch.int64, device=dev)
    bad = [
        lambda: aspis.embed(x, t.to(torch.int16)), lambda: aspis.embed(x, t.cpu()),
        lambda: aspis.embed(x.double(), t), lambda: aspis.embed(x[0], t),
        lambda: aspis.embed(x, t.new_zeros(8)[::2]), lambda: aspis.embed(x, [0, 1]),
        lambda: aspis.embed(x, t, out=x), lambda: aspis.embed(x, t, out=torch.zeros((3, 6), device=dev)),
        lambda: aspis.embed(x, t, scale=math.inf), lambda: aspis.embed(x, t, scale=1e39),
        lambda: aspis.embed(x.t(), t), lambda: aspis.embed(x.cpu(), t),
        lambda: aspis.embed(x, t, out=torch.zeros((4, 6))),
        lambda: aspis.embed_grad(x, t[:3], 9), lambda: aspis.embed_grad(x, t, 9, accumulate=True),
        lambda: aspis.embed_grad(x, t, 4, out=x), lambda: aspis.embed_grad(x, t, 9, out=x),
        lambda: aspis.embed_grad(x, t, 9, scale=math.nan),
        lambda: aspis.embed_grad(long, many, 9, ws=torch.zeros(16, dtype=torch.uint8, device=dev)),
        lambda: aspis.embed_grad(long, many, 9,
                                 ws=torch.zeros(99_999, dtype=torch.uint8, device=dev)[1:]),
        lambda: aspis.embed_grad(x, t, 9, ws=torch.zeros(99_999, dtype=torch.uint8)),
        lambda: aspis.embed_grad(x, t.float(), 9),
        lambda: aspis.dropout(x, -0.1, 1), lambda: aspis.dropout(x, 1.1, 1),
        lambda: aspis.dropout(x, math.nan, 1), lambda: aspis.dropout(x.cpu(), 0.1, 1),
        lambda: aspis.dropout(x, 0.1, 1, out=torch.zeros((4, 5), device=dev)),
        lambda: aspis.dropout(x, 0.1, 1, out=torch.zeros((4, 6), device=dev, dtype=torch.float16)),
        lambda: aspis.dropout(x, 0.1, 1, residual=torch.zeros((4, 6))),
        lambda: aspis.dropout(x[:3], 0.1, 1, out=x[1:]),
        lambda: aspis.dropout(x[:3], 0.1, 1, residual=x[1:], out=x[:3]),
        lambda: aspis.dropout(x.double(), 0.1, 1),
        lambda: aspis.dropout(x, 0.1, torch.zeros(1, device=dev)),
        lambda: aspis.dropout(x, 0.1, torch.zeros(1, dtype=torch.int64)),
        lambda: aspis.token_logps(x, t, temperature=0.0),
        lambda: aspis.token_logps(x, t, temperature=math.inf),
        lambda: aspis.token_logps(x, t, temperature=-1.0),
        lambda: aspis.token_logps(x, t, logps=v[:3]), lambda: aspis.token_logps(x, t[:3]),
        lambda: aspis.token_logps(x, t, ws=torch.zeros(8, dtype=torch.uint8, device=dev)),
        lambda: aspis.policy_loss(x, t, v, v, v.double()), lambda: aspis.policy_loss(x, t, v[:3], v, v),
        lambda: aspis.policy_loss(x, t, long_v, v, v), lambda: aspis.policy_loss(x, t, v, long_v, v),
        lambda: aspis.policy_loss(x, t, v, v, long_v), lambda: aspis.policy_loss(x, t, v, v, v, ref=long_v),
        lambda: aspis.embed(x, wide.view(torch.int64)[:4], out=wide.view(4, 6)),
        lambda: aspis.dropout(x[:1], 0.1, x.view(torch.int64)[0, :1], out=x[:1]),
        lambda: aspis.token_logps(x, t, logps=x[0, :4]),
        lambda: aspis.policy_loss(x, t, v, v, v, kl=0.1), lambda: aspis.policy_loss(x, t, v, v, v, ref=v.cpu()),
        lambda: aspis.policy_loss(x, t, v, v, v, clip=(1.5, 0.2)),
        lambda: aspis.policy_loss(x, t, v, v, v, clip=(0.2, -0.1)),
        lambda: aspis.policy_loss(x, t, v, v, v, ref=v, kl=-1.0),
        lambda: aspis.policy_loss(x, t, v, v, v, grad_scale=math.inf),
        lambda: aspis.policy_loss(x, t, v, v, v, grad=torch.zeros((4, 6), device=dev).half()),
        lambda: aspis.policy_loss(x[:3], t[:3], v[:3], v[:3], v[:3], grad=x[1:]),
        lambda: aspis.policy_loss(x, t, v, v, v, ws=torch.zeros(8, dtype=torch.uint8, device=dev)),
        lambda: aspis.policy_loss(x, t, v, v, v, bufs=aspis.PolicyBuffers.empty(3, dev)),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(aspis.AspisError):
            call()
            raise AssertionError(i)
    assert (x == 0).all() and (v == 0).all()
    assert aspis.token_logps(x, t).dtype == f


@pytest.mark.parametrize("d", [6, 64, 257])
@pytest.mark.parametrize("kind", KINDS)
def test_columns_of_one_tensor(kind, d):
    """Results beside inputs in the same rows, which share no memory."""
    import torch
    rows = 40
    x = _randn((rows, d), kind, seed=d)
    _, t = _tokens(rows, d, seed=d)
    v = _randn((rows,), seed=3)

    def beside():
        both = torch.full((rows, 2 * d + 3), 7.0, dtype=x.dtype, device=x.device)
        both[:, :d] = x
        return both, both[:, :d], both[:, d + 3:]

    def policy(a, out):
        aspis.policy_loss(a, t, v, v, v, ref=v, kl=0.1, grad=out)
        return out

    for call in (lambda a, out: aspis.dropout(a, 0.3, 5, residual=a, out=out),
                 lambda a, out: aspis.embed(a, t % rows, out=out),
                 lambda a, out: aspis.embed_grad(a, t % rows, rows, out=out), policy):
        both, a, out = beside()
        call(a, out)
        want = call(x, torch.empty_like(x))
        assert (_bits(out.contiguous()) == _bits(want)).all()
        assert (_bits(a.contiguous()) == _bits(x)).all() and (both[:, d:d + 3] == 7.0).all()


@pytest.mark.parametrize("rows,d", [(0, 5), (3, 0), (0, 0)])
def test_empty(rows, d):
    import torch
    dev = device()
    x = torch.zeros((rows, d), device=dev)
    t = torch.zeros(rows, dtype=torch.int64, device=dev)
    v = torch.ones(rows, device=dev)
    assert aspis.dropout(x, 0.5, 1).shape == (rows, d)
    assert aspis.embed(torch.zeros((4, d), device=dev), t).shape == (rows, d)
    assert aspis.embed_grad(x, t, 4).shape == (4, d)
    assert (aspis.token_logps(x, t) == 0).all()
    bufs = aspis.policy_loss(x, t, v, v, v, ref=v, kl=0.1, grad=torch.empty_like(x))
    assert (bufs.sums == 0).all() and (bufs.logps == 0).all()
