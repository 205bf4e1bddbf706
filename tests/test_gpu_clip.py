"""Norms, clipping and the model updates on the GPU against plain formulas in
64 bits.

Tolerances, from the formulas (u = 2^-24, half an f32 ulp relative to the
value):
- norm: the fp64 sum is off by far less than u; one rounding to f32.
- clipped values: the coefficient's rounding and the product's, 2 u together,
  plus the rounding to a 16-bit result; half the smallest step of the type
  once per rounding below its normal range.
- updates: every operation adds at most u of the magnitudes it works on;
  the bounds below count operations and rounded constants.
"""
import math

import numpy as np
import pytest

from paper_2108_02416_amd import aspis

from _helpers import device, to_np

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
KINDS = ["float32", "bfloat16", "float16"]
HALF_ULP = {"float32": 0.0, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
TINY = {"float32": 2.0 ** -149, "bfloat16": 2.0 ** -133, "float16": 2.0 ** -24}


def _type(kind):
    import torch
    return getattr(torch, kind)


def _randn(n, kind="float32", seed=0, scale=0.01):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(n, generator=gen, device=device()).mul_(scale).to(_type(kind))


def _views(numels, kind="float32", seed=0, offset=0, scale=0.01):
    """Tensors packed in one buffer, `offset` elements from its start."""
    flat = _randn(offset + sum(numels), kind, seed, scale)
    return list(flat[offset:].split(list(numels)))


def _f64(t):
    return t.detach().double().cpu().numpy().reshape(-1)


def _norm64(tensors):
    return math.sqrt(sum(float(np.dot(x, x)) for x in map(_f64, tensors)))


def _coef64(norm, bound):
    return 1.0 if norm <= bound or math.isinf(bound) else bound / norm


def _assert_norm(got, want):
    got = float(got)
    assert abs(got - want) <= U * want * (1 + 1e-6) + 2.0 ** -150, (got, want)


def _assert_scaled(got, x, c, kind):
    """got = c x in the type `kind`, within the roundings."""
    want = c * _f64(x)
    tol = np.abs(want) * (2 * U * (1 + 1e-6) + HALF_ULP[kind] * (1 + 1e-5)) + 1.5 * TINY[kind]
    bad = ~(np.abs(_f64(got) - want) <= tol)
    assert not bad.any(), (int(bad.sum()), _f64(got)[bad][:4], want[bad][:4])


def _bits(t):
    import torch
    return t.detach().reshape(-1).contiguous().view(
        torch.int32 if t.dtype == torch.float32 else torch.int16).cpu().numpy()


LISTS = {
    "one": [1],
    "softmax": [7840, 10],
    "with_empty": [5, 0, 3],
    "all_empty": [0, 0],
    "chunk": [16384],
    "chunk_less": [16383],
    "chunk_more": [16385, 1],
    "uneven": [3, 70_001, 1, 250_007, 64],
    "many": [(37 * i) % 101 for i in range(400)],
    "over_grid": [40_000_003, 17, 2_000_001],
}


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("name", list(LISTS))
@pytest.mark.parametrize("offset", [0, 1, 3])
def test_grad_norm(name, kind, offset):
    ts = _views(LISTS[name], kind, seed=len(name), offset=offset)
    plain = aspis.grad_norm(ts)
    bufs = aspis.grad_norm(ts, each=True)
    _assert_norm(bufs.norm, _norm64(ts))
    assert float(bufs.norm) == float(plain.norm)
    sumsq = _norm64(ts) ** 2
    assert abs(float(bufs.sumsq) - sumsq) <= 1e-12 * sumsq
    for got, t in zip(bufs.each.tolist(), ts):
        _assert_norm(got, _norm64([t]))


def test_grad_norm_of_no_tensors():
    bufs = aspis.grad_norm(aspis.TensorList([], device=device()))
    assert float(bufs.norm) == 0.0 and float(bufs.sumsq) == 0.0


def test_mixed_types_and_orders_of_dimensions():
    import torch
    ts = [_randn(300, "bfloat16").reshape(10, 30).t(),
          _randn(2 * 3 * 4 * 5).reshape(2, 3, 4, 5).to(memory_format=torch.channels_last),
          _randn(77, "float16"), _randn(1).reshape(()), _randn(20_000).reshape(1, 20_000)]
    bufs = aspis.grad_norm(ts, each=True)
    _assert_norm(bufs.norm, _norm64(ts))
    out = [torch.empty_like(t) for t in ts]   # keeps the strides
    norm = _norm64(ts)
    aspis.clip_grads(ts, norm / 3, out=out)
    for t, o in zip(ts, out):
        assert o.stride() == t.stride()
        _assert_scaled(o, t, _coef64(norm, norm / 3), str(t.dtype).split(".")[1])


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("name", ["softmax", "with_empty", "all_empty", "uneven", "many",
                                  "over_grid"])
@pytest.mark.parametrize("where", ["in_place", "out"])
def test_clip_grads(name, kind, where):
    import torch
    ts = _views(LISTS[name], kind, seed=3, offset=1)
    before = [t.clone() for t in ts]
    norm = _norm64(ts)
    for bound in (norm * 0.4, norm * 1.5 + 1e-3):
        for t, b in zip(ts, before):
            t.copy_(b)
        out = None if where == "in_place" else \
            list(torch.empty(2 + sum(LISTS[name]), dtype=_type(kind),
                             device=device())[2:].split(LISTS[name]))
        bufs = aspis.clip_grads(ts, bound, out=out)
        _assert_norm(bufs.norm, norm)
        got = ts if out is None else out
        for g, b in zip(got, before):
            if bound > norm:
                assert np.array_equal(_bits(g), _bits(b))
            else:
                _assert_scaled(g, b, _coef64(norm, bound), kind)
        if out is not None:
            for t, b in zip(ts, before):
                assert np.array_equal(_bits(t), _bits(b))


def test_in_place_clip_brings_the_norm_to_the_bound():
    ts = _views([30_001, 5, 1_000_003], seed=5)
    aspis.clip_grads(ts, 1.0)
    assert abs(float(aspis.grad_norm(ts).norm) - 1.0) <= 3 * U


@pytest.mark.parametrize("n", [4, 9, 40_000])
def test_special_values(n):
    import torch
    inf, nan = float("inf"), float("nan")
    dev = device()
    x = _randn(n, seed=1)
    # a sum of squares past f32: 3e38 in every place
    big = torch.full((n,), 3e38, device=dev)
    out = torch.empty_like(big)
    bufs = aspis.clip_grads([big], 1.0, out=[out])
    want = 3.0000000054977558e38
    assert abs(float(bufs.sumsq) / (n * float(big[0]) ** 2) - 1) < 1e-12
    assert math.isinf(float(bufs.norm)) == (math.sqrt(n) * want > 3.4028235e38)
    _assert_scaled(out, big, 1.0 / (math.sqrt(n) * float(big[0])), "float32")
    # a coefficient below the smallest f32
    aspis.clip_grads([big], 1e-20, out=[out])
    _assert_scaled(out, big, 1e-20 / (math.sqrt(n) * float(big[0])), "float32")
    # denormals: squares below the smallest f32
    small = torch.full((n,), 1e-41, device=dev)
    bufs = aspis.clip_grads([small], 5e-42, out=[out])
    _assert_norm(bufs.norm, math.sqrt(n) * float(small[0].double()))
    _assert_scaled(out, small, _coef64(math.sqrt(n) * float(small[0].double()), 5e-42), "float32")
    # zeros
    bufs = aspis.clip_grads([torch.zeros(n, device=dev)], 0.0, out=[out])
    assert float(bufs.norm) == 0.0 and not out.any()
    # a bound of nothing
    aspis.clip_grads([x], 0.0, out=[out])
    assert not out.any()
    # no bound
    aspis.clip_grads([x], inf, out=[out])
    assert np.array_equal(_bits(out), _bits(x))
    # an infinity: finite elements go to 0, the infinite one to NaN
    y = x.clone()
    y[2] = -inf
    bufs = aspis.clip_grads([y], 1.0, out=[out])
    assert float(bufs.norm) == inf
    got = to_np(out)
    assert math.isnan(got[2]) and not np.delete(got, 2).any()
    # a NaN is never hidden
    y[2] = nan
    bufs = aspis.clip_grads([y], 1.0, out=[out])
    assert math.isnan(float(bufs.norm)) and np.isnan(to_np(out)).all()
    aspis.clip_grads([y], inf, out=[out])
    assert np.array_equal(np.isnan(to_np(out)), np.isnan(to_np(y)))


def test_same_bits_wherever_the_tensors_lie():
    """Clipping depends on values and sizes alone: other offsets, and one
    buffer or many."""
    sizes = [100_003, 7, 16_384, 1]
    ref = _views(sizes, seed=9, offset=0)
    a = aspis.clip_grads([t.clone() for t in ref], 0.25, out=[t.clone() for t in ref])
    want = None
    for offset in (0, 1, 2, 3, 5):
        ts = _views(sizes, seed=9, offset=offset)
        for t, r in zip(ts, ref):
            t.copy_(r)
        bufs = aspis.clip_grads(ts, 0.25)
        assert float(bufs.sumsq) == float(a.sumsq)
        got = [_bits(t) for t in ts]
        want = want or got
        assert all(np.array_equal(g, w) for g, w in zip(got, want))


def test_sum_of_squares_of_all_ranks():
    """Two shards of one model: each rank's sum, added, clips both."""
    a, b = _views([5_000, 3], seed=1), _views([70_000], seed=2)
    total = aspis.grad_norm(a).sumsq + aspis.grad_norm(b).sumsq
    norm = _norm64(a + b)
    for shard in (a, b):
        before = [t.clone() for t in shard]
        bufs = aspis.clip_grads(shard, 0.5, sumsq=total)
        _assert_norm(bufs.norm, norm)
        for t, x in zip(shard, before):
            _assert_scaled(t, x, 0.5 / norm, "float32")
    # a rank without tensors reports the norm of all
    bufs = aspis.clip_grads(aspis.TensorList([], device=device()), 0.5, sumsq=total)
    _assert_norm(bufs.norm, norm)


def test_a_list_follows_its_tensors():
    import torch
    ts = [_randn(1000, seed=1), _randn(50, seed=2)]
    handle = aspis.TensorList(ts)
    _assert_norm(aspis.grad_norm(handle).norm, _norm64(ts))
    ts[0].data = _randn(40_000, seed=3)
    _assert_norm(aspis.grad_norm(handle).norm, _norm64(ts))
    ts[1].fill_(3.0)
    _assert_norm(aspis.grad_norm(handle).norm, _norm64(ts))
    with pytest.raises(aspis.AspisError):
        aspis.clip_grads(handle, 1.0, out=[torch.empty(1000, device="cuda"),
                                           torch.empty(50, device="cuda")])


# --------------------------------------------------------------------- rows

ROW_LENGTHS = [1, 2, 3, 4, 5, 7, 8, 9, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256,
               257, 511, 512, 513, 1024, 1025, 2047, 2048, 2049, 4096, 4097, 8191, 8192, 8193,
               16384, 16385, 32767, 32768, 32769, 49153, 65536, 65537, 100_003, 1_048_579]


def _check_rows(x, bound, got, norms, kind):
    x64 = x.detach().double()
    want_norms = x64.square().sum(-1).sqrt()
    assert bool(((norms.double() - want_norms).abs() <= U * want_norms * (1 + 1e-6)).all())
    c = torch_where(want_norms, bound)
    want = x64 * c[..., None]
    tol = want.abs() * (2 * U * (1 + 1e-6) + HALF_ULP[kind] * (1 + 1e-5)) + 1.5 * TINY[kind]
    assert bool(((got.double() - want).abs() <= tol).all())
    whole = c == 1.0
    assert bool((got[whole] == x[whole]).all())


def torch_where(norms, bound):
    import torch
    return torch.where(norms <= bound, torch.ones_like(norms), bound / norms)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d", ROW_LENGTHS)
def test_clip_rows(d, kind):
    import torch
    rows = 67 if d <= 4096 else 5
    for pad, where in ((0, "out"), (3, "in_place")):
        x = _randn(rows * (d + pad), kind, seed=d).reshape(rows, d + pad)[:, :d]
        x[::3].mul_(10.0)
        bound = 0.03 * math.sqrt(d)
        before = x.clone()
        norms = aspis.row_norms(x)
        if where == "out":
            wide = torch.full((rows, d + 5), 7.0, dtype=x.dtype, device=x.device)
            got, after = aspis.clip_rows(x, bound, out=wide[:, 5:])
            assert bool((wide[:, :5] == 7.0).all())
            assert bool((x == before).all())
        else:
            got, after = aspis.clip_rows(x, bound)
            assert got is x
        assert bool((norms == after).all())
        _check_rows(before, bound, got, after, kind)


@pytest.mark.parametrize("rows", [1, 2, 3, 255, 256, 257, 70_001])
@pytest.mark.parametrize("d", [1, 6, 40])
def test_clip_rows_counts(rows, d):
    x = _randn(rows * d, seed=rows).reshape(rows, d)
    got, norms = aspis.clip_rows(x, 0.01, out=x.clone())
    _check_rows(x, 0.01, got, norms, "float32")


@pytest.mark.parametrize("kind,rows,d", [("float32", 23, 1_500_001), ("float32", 9, 17_000_003),
                                         ("float32", 5, 25_000_003), ("bfloat16", 70, 800_003),
                                         ("float16", 1, 20_000_001)])
@pytest.mark.parametrize("where", ["out", "in_place"])
def test_clip_long_rows_over_several_launches(kind, rows, d, where):
    x = _randn(rows * d, kind, seed=rows).reshape(rows, d)
    x[::4].mul_(5.0)
    before = x.clone()
    bound = 0.015 * math.sqrt(d)
    got, norms = aspis.clip_rows(x, bound, out=None if where == "in_place" else x.clone())
    for i in range(rows):
        _check_rows(before[i:i + 1], bound, got[i:i + 1], norms[i:i + 1], kind)
    assert bool((aspis.row_norms(before) == norms).all())


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,d", [(1, 40_001), (40, 140_003), (200, 70_007), (9, 1_300_003),
                                    (3, 9_000_001)])
def test_long_rows_have_the_same_bits_by_every_way(rows, d, kind):
    """Alone or among others (few rows take two passes over the cache, more
    stay in registers), with and without workgroups waiting for one another,
    in place or not, at any alignment."""
    import torch
    x = _randn(rows * d, kind, seed=d).reshape(rows, d)
    x[::2].mul_(3.0)
    bound = 0.015 * math.sqrt(d)
    out, norms = aspis.clip_rows(x, bound, out=torch.empty_like(x))
    _check_rows(x, bound, out, norms, kind)
    again, same = aspis.clip_rows(x, bound, out=torch.empty_like(x), flags=aspis.CLIP_NO_WAIT)
    assert np.array_equal(_bits(again), _bits(out)) and bool((norms == same).all())
    assert bool((aspis.row_norms(x) == norms).all())
    for i in {0, rows // 2, rows - 1}:
        one, norm = aspis.clip_rows(x[i], bound, out=torch.empty_like(x[i]))
        assert np.array_equal(_bits(one), _bits(out[i])) and float(norm) == float(norms[i])
    wide = torch.empty((rows, d + 3), dtype=x.dtype, device=x.device)[:, 1:d + 1]
    wide.copy_(x)
    aspis.clip_rows(wide, bound, flags=aspis.CLIP_NO_WAIT)
    assert np.array_equal(_bits(wide), _bits(out))


@pytest.mark.parametrize("d", [3, 300, 5_000, 70_000])
def test_rows_with_special_values(d):
    import torch
    inf, nan = float("inf"), float("nan")
    x = _randn(6 * d, seed=d).reshape(6, d)
    x[0] = 0.0
    x[1, 1] = inf
    x[2, 2] = nan
    x[3] = 3e38
    x[4] = 1e-41
    out, norms = aspis.clip_rows(x, 1e-3, out=torch.empty_like(x))
    n, got = to_np(norms), to_np(out)
    assert n[0] == 0 and not got[0].any()
    assert n[1] == inf and math.isnan(got[1, 1]) and not np.delete(got[1], 1).any()
    assert math.isnan(n[2]) and np.isnan(got[2]).all()
    for i in (3, 4, 5):
        norm = _norm64([x[i]])
        _assert_scaled(out[i], x[i], _coef64(norm, 1e-3), "float32")


def test_rows_shapes():
    import torch
    x = _randn(4 * 3 * 50, seed=1).reshape(4, 3, 50)
    out, norms = aspis.clip_rows(x, 0.05, out=torch.empty_like(x))
    assert norms.shape == (4, 3)
    _check_rows(x, 0.05, out, norms, "float32")
    every = x[::2]                      # rows equally far apart within a file only
    with pytest.raises(aspis.AspisError):
        aspis.row_norms(every)
    one = x[1:2, ::2]                   # one series of rows, two apart
    _check_rows(one, 0.05, *aspis.clip_rows(one, 0.05, out=torch.empty_like(one)), "float32")
    flat, norm = aspis.clip_rows(x[0, 0], 0.01, out=torch.empty(50, device="cuda"))
    assert norm.shape == ()
    _check_rows(x[0, 0][None], 0.01, flat[None], norm[None], "float32")
    for shape in ((0, 5), (5, 0), (0, 0)):
        e = torch.empty(shape, device="cuda")
        out, norms = aspis.clip_rows(e, 1.0)
        assert norms.shape == shape[:1] and not norms.any()


def test_clipped_replicas_still_agree():
    """Replicas with equal bits are equal after clipping, in both layouts, and
    the step selects the same files."""
    import oracle
    import synth
    import torch
    wl = synth.WORKLOADS[1]
    g, _ = synth.generate(wl, oracle.assign(wl.K, wl.r), d=5_001)
    grads = torch.from_numpy(g).to(device())
    ref = aspis.detect_aggregate(grads, wl.K, wl.r, wl.q)
    clipped, norms = aspis.clip_rows(grads, 0.5, out=torch.empty_like(grads))
    got = aspis.detect_aggregate(clipped, wl.K, wl.r, wl.q)
    assert np.array_equal(to_np(got["sel"]), to_np(ref["sel"]))
    assert np.array_equal(to_np(got["bufs"].pair_diff), to_np(ref["bufs"].pair_diff))
    by_worker = torch.empty((wl.K, grads.shape[0] * wl.r // wl.K, 5_001), device=device())
    rows = aspis.worker_rows(wl.K, wl.r).reshape(-1)
    by_worker.view(-1, 5_001)[torch.from_numpy(rows).long().to(device())] = grads.view(-1, 5_001)
    aspis.clip_rows(by_worker, 0.5)
    again = aspis.detect_aggregate(by_worker, wl.K, wl.r, wl.q, layout="worker")
    assert np.array_equal(_bits(again["out"]), _bits(got["out"]))


# ------------------------------------------------------------------ updates

def _sgd64(p, g, m, lr, mu, wd, nesterov):
    g = g + wd * p
    m = mu * m + g
    step = g + mu * m if nesterov else m
    size = (1 + mu) * (np.abs(g) + 2 * wd * np.abs(p) + mu * np.abs(m) * 2)
    return p - lr * step, m, 8 * U * (np.abs(p) + lr * size), 8 * U * size


def _assert_near(got, want, tol):
    bad = ~(np.abs(_f64(got) - want) <= tol + 1e-44)
    assert not bad.any(), (int(bad.sum()), _f64(got)[bad][:4], want[bad][:4], tol[bad][:4])


def _assert_copy(copy, params):
    """The copy is the new parameter rounded to its type, to the bit."""
    assert np.array_equal(_bits(copy), _bits(params.to(copy.dtype)))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("name", ["one", "softmax", "with_empty", "uneven", "many"])
@pytest.mark.parametrize("mu,nesterov,wd,copy", [(0.9, False, 0.0, None), (0.9, True, 5e-4, "bfloat16"),
                                                 (0.0, False, 1e-2, "float16"),
                                                 (0.0, False, 0.0, "float32")])
def test_clipped_sgd(name, kind, mu, nesterov, wd, copy):
    import torch
    sizes = LISTS[name]
    grads = _views(sizes, kind, seed=1, offset=1)
    params = _views(sizes, seed=2, offset=3, scale=0.5)
    mean = _views(sizes, seed=3, offset=2, scale=0.003) if mu else None
    copies = None if copy is None else \
        list(torch.empty(1 + sum(sizes), dtype=_type(copy), device=device())[1:].split(sizes))
    g0 = [g.clone() for g in grads]
    norm = _norm64(grads)
    bound = 0.3 * norm
    want = [_sgd64(_f64(p), 0.3 * _f64(g), _f64(mean[i]) if mu else np.zeros(g.numel()), 0.1, mu, wd,
                   nesterov) for i, (p, g) in enumerate(zip(params, grads))]
    bufs = aspis.clipped_sgd(params, grads, mean, lr=0.1, momentum=mu, nesterov=nesterov,
                             weight_decay=wd, max_norm=bound, copies=copies)
    _assert_norm(bufs.norm, norm)
    for i, (p64, m64, p_tol, m_tol) in enumerate(want):
        assert np.array_equal(_bits(grads[i]), _bits(g0[i]))
        _assert_near(params[i], p64, p_tol)
        if mu:
            _assert_near(mean[i], m64, m_tol)
        if copy:
            _assert_copy(copies[i], params[i])


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("name", ["one", "softmax", "with_empty", "uneven", "many"])
@pytest.mark.parametrize("step,wd,copy", [(1, 0.0, None), (1000, 0.1, "bfloat16"),
                                          (7, 0.01, "float16")])
def test_clipped_adamw(name, kind, step, wd, copy):
    import torch
    sizes = LISTS[name]
    b1, b2, eps, lr = 0.9, 0.95, 1e-8, 3e-3
    grads = _views(sizes, kind, seed=1, offset=1)
    params = _views(sizes, seed=2, offset=3, scale=0.5)
    mean = _views(sizes, seed=3, offset=2, scale=0.003)
    square = [v.square_() for v in _views(sizes, seed=4, offset=0, scale=0.003)]
    copies = None if copy is None else \
        list(torch.empty(1 + sum(sizes), dtype=_type(copy), device=device())[1:].split(sizes))
    norm = _norm64(grads)
    bound = 0.3 * norm
    want = []
    for p, g, m, v in zip(params, grads, mean, square):
        p, g, m, v = _f64(p), 0.3 * _f64(g), _f64(m), _f64(v)
        m_new = b1 * m + (1 - b1) * g
        v_new = b2 * v + (1 - b2) * g * g
        m_tol = 6 * U * (b1 * np.abs(m) + (1 - b1) * np.abs(g))
        v_tol = 8 * U * v_new
        rate = lr / (1 - b1 ** step)
        root = np.sqrt(v_new / (1 - b2 ** step)) + eps
        # the root's relative error is half the square's, plus its own roundings
        p_tol = 4 * U * np.abs(p) + rate * (m_tol + 16 * U * np.abs(m_new)) / root
        want.append((p * (1 - lr * wd) - rate * m_new / root, m_new, v_new, p_tol, m_tol, v_tol))
    bufs = aspis.clipped_adamw(params, grads, mean, square, step=step, lr=lr, betas=(b1, b2),
                               eps=eps, weight_decay=wd, max_norm=bound, copies=copies)
    _assert_norm(bufs.norm, norm)
    for i, (p64, m64, v64, p_tol, m_tol, v_tol) in enumerate(want):
        _assert_near(mean[i], m64, m_tol)
        _assert_near(square[i], v64, v_tol)
        _assert_near(params[i], p64, p_tol)
        if copy:
            _assert_copy(copies[i], params[i])


@pytest.mark.parametrize("sizes", [[900, 7], [300_001, 5], [40_000_003]])
def test_updates_by_the_sum_of_all_ranks(sizes):
    """An update by a given sum of squares is the one by gradients that have
    it: twice the norm gives half the coefficient."""
    import torch
    g, p = _views(sizes, seed=1, offset=1), _views(sizes, seed=2, offset=2, scale=0.5)
    q, m, n = [t.clone() for t in p], [torch.zeros_like(t) for t in p], [torch.zeros_like(t) for t in p]
    own = aspis.grad_norm(g)
    bound = 0.5 * float(own.norm)
    a = aspis.clipped_sgd(p, g, m, lr=0.1, momentum=0.9, max_norm=bound, sumsq=4.0 * own.sumsq)
    b = aspis.clipped_sgd(q, g, n, lr=0.1, momentum=0.9, max_norm=0.5 * bound)
    assert float(a.norm) == 2.0 * float(own.norm) and float(b.norm) == float(own.norm)
    assert all(np.array_equal(_bits(x), _bits(y)) for x, y in zip(p + m, q + n))


@pytest.mark.parametrize("rule,n,kind", [("sgd", 51_000_001, "bfloat16"), ("sgd", 3_000_001, "float32"),
                                         ("adamw", 12_000_003, "float32"),
                                         ("adamw", 34_000_001, "float16")])
def test_updates_of_long_lists(rule, n, kind):
    """The kernels for lists of some thousand chunks and of more than the
    cache keeps, against the formulas in 64 bits on the GPU."""
    import torch
    sizes = [n // 3, 5, n - n // 3 - 5]
    grads = _views(sizes, kind, seed=1, offset=1)
    params, mean = _views(sizes, seed=2, offset=2, scale=0.5), _views(sizes, seed=3, scale=0.003)
    square = [v.square_() for v in _views(sizes, seed=4, offset=1, scale=0.003)]
    copies = [torch.empty(k, dtype=torch.bfloat16, device=device()) for k in sizes]
    norm = math.sqrt(sum(float(g.double().square().sum()) for g in grads))
    bound, lr = 0.3 * norm, 3e-3
    start = [[t.double() for t in x] for x in (params, mean, square)]
    if rule == "sgd":
        bufs = aspis.clipped_sgd(params, grads, mean, lr=lr, momentum=0.9, max_norm=bound,
                                 copies=copies)
    else:
        bufs = aspis.clipped_adamw(params, grads, mean, square, step=3, lr=lr, betas=(0.9, 0.95),
                                   weight_decay=0.1, max_norm=bound, copies=copies)
    _assert_norm(bufs.norm, norm)
    for i in range(3):
        g = 0.3 * grads[i].double()
        p, m, v = (x[i] for x in start)
        if rule == "sgd":
            m_tol = 8 * U * (g.abs() + 0.9 * m.abs() * 2)
            m = 0.9 * m + g
            p_tol, p = 8 * U * p.abs() + lr * m_tol, p - lr * m
        else:
            m_tol = 6 * U * (0.9 * m.abs() + 0.1 * g.abs())
            m, v = 0.9 * m + 0.1 * g, 0.95 * v + 0.05 * g * g
            rate, root = lr / (1 - 0.9 ** 3), (v / (1 - 0.95 ** 3)).sqrt() + 1e-8
            p_tol = 4 * U * p.abs() + rate * (m_tol + 16 * U * m.abs()) / root
            p = p * (1 - lr * 0.1) - rate * m / root
            assert bool(((square[i].double() - v).abs() <= 8 * U * v + 1e-44).all())
        assert bool(((mean[i].double() - m).abs() <= m_tol + 1e-44).all())
        assert bool(((params[i].double() - p).abs() <= p_tol + 1e-44).all())
        assert bool((copies[i] == params[i].bfloat16()).all())


def test_unclipped_updates_use_the_gradients_bits():
    """Without a bound SGD with lr = 1 from zero gives -g to the bit."""
    import torch
    g = _views([1_003, 20_000], seed=1, offset=1)
    p = [torch.zeros_like(t) for t in g]
    aspis.clipped_sgd(p, g, lr=1.0)
    for a, b in zip(p, g):
        assert np.array_equal(_bits(a), _bits(-b))


@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_updates_can_skip_a_norm_that_is_not_finite(value):
    import torch
    for rule in ("sgd", "adamw"):
        g = _views([70_000, 30], seed=1)
        g[1][7] = value
        p, m, v = (_views([70_000, 30], seed=s, offset=1) for s in (2, 3, 4))
        v = [x.square_() for x in v]
        copies = [torch.full((n,), 9.0, dtype=torch.bfloat16, device=device()) for n in (70_000, 30)]
        before = [_bits(t) for t in p + m + v + copies]

        def go(skip):
            if rule == "sgd":
                return aspis.clipped_sgd(p, g, m, lr=0.1, momentum=0.9, max_norm=1.0, copies=copies,
                                         skip_nonfinite=skip)
            return aspis.clipped_adamw(p, g, m, v, step=3, lr=0.1, max_norm=1.0, copies=copies,
                                       skip_nonfinite=skip)
        bufs = go(True)
        assert not math.isfinite(float(bufs.norm))
        assert all(np.array_equal(_bits(t), b) for t, b in zip(p + m + v + copies, before))
        go(False)
        if math.isnan(value):
            assert bool(torch.isnan(p[0]).all())
        else:
            assert math.isnan(float(p[1][7])) and bool(torch.isfinite(p[0]).all())


# ------------------------------------------------- streams, graphs, lengths

def test_lists_and_buffers_on_another_stream():
    import torch
    side = torch.cuda.Stream()
    ts = _views([500_000, 3], seed=1)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        handle = aspis.TensorList(ts)
        a = aspis.grad_norm(handle)
    side.synchronize()
    b = aspis.grad_norm(handle)
    torch.cuda.synchronize()
    assert float(a.norm) == float(b.norm)
    _assert_norm(a.norm, _norm64(ts))


def test_long_rows_on_two_streams_at_once():
    """Two calls whose rows each take most of the device: workgroups that
    wait for others that cannot start give up and their parts are read again.
    Both results are those of a call alone."""
    import torch
    xs = [_randn(6 * 11_000_001, seed=s).reshape(6, 11_000_001) for s in (1, 2)]
    bound = 0.004 * math.sqrt(11_000_001)
    want = [aspis.clip_rows(x, bound, out=torch.empty_like(x)) for x in xs]
    streams = [torch.cuda.Stream() for _ in xs]
    outs = [torch.empty_like(x) for x in xs]
    sizes = [aspis.row_workspace(x) for x in xs]
    norms = [torch.empty(6, device=device()) for _ in xs]
    torch.cuda.synchronize()
    for _ in range(3):
        for x, o, n, w, s in zip(xs, outs, norms, sizes, streams):
            with torch.cuda.stream(s):
                o.zero_()
                aspis.clip_rows(x, bound, out=o, norms=n, ws=w)
        torch.cuda.synchronize()
        for (a, b), o, n in zip(want, outs, norms):
            assert bool((a == o).all()) and bool((b == n).all())


def test_in_a_graph():
    """An update and a clip of rows captured once and replayed on new
    gradients, with other work between the replays."""
    import torch
    sizes = [70_001, 513]
    grads = aspis.TensorList(_views(sizes, "bfloat16", seed=1))
    params, mean = (aspis.TensorList(_views(sizes, seed=s)) for s in (2, 3))
    rows = _randn(3 * 100_003, seed=4).reshape(3, 100_003)
    out, norms = torch.empty_like(rows), torch.empty(3, device=device())
    bufs, ws = aspis.NormBuffers.empty(device()), aspis.norm_workspace(grads)
    row_ws = aspis.row_workspace(rows)

    def go():
        aspis.clip_rows(rows, 1.0, out=out, norms=norms, ws=row_ws)
        aspis.clipped_sgd(params, grads, mean, lr=0.1, momentum=0.9, max_norm=0.5, bufs=bufs, ws=ws)

    start = [[t.clone() for t in x.tensors] for x in (params, mean)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        go()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    for replay in range(4):
        for x, kept in zip((params, mean), start):
            for t, k in zip(x.tensors, kept):
                t.copy_(k)
        for i, t in enumerate(grads.tensors):
            t.copy_(_randn(t.numel(), "bfloat16", seed=50 + 7 * replay + i))
        rows.copy_(_randn(rows.numel(), seed=90 + replay).reshape(rows.shape))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for x in (params, mean) for t in x.tensors] + [out.clone(), norms.clone()]
        for x, kept in zip((params, mean), start):
            for t, k in zip(x.tensors, kept):
                t.copy_(k)
        go()
        torch.cuda.synchronize()
        want = [t for x in (params, mean) for t in x.tensors] + [out, norms]
        assert all(np.array_equal(_bits(a), _bits(b)) for a, b in zip(got, want)), replay


def test_more_than_two_to_the_31_elements():
    """Offsets past 32 bits: in a list's one tensor and in rows."""
    import torch
    n = 2 ** 31 + 12_345
    x = torch.zeros(n, dtype=torch.bfloat16, device=device())
    x[-1], x[2 ** 31], x[5] = 3.0, 4.0, 12.0
    assert float(aspis.grad_norm([x]).norm) == 13.0
    aspis.clip_grads([x], 6.5)
    assert (float(x[-1]), float(x[2 ** 31]), float(x[5])) == (1.5, 2.0, 6.0)
    rows = x[:2 ** 31].view(4, 2 ** 29)
    rows.zero_()
    rows[3, -1], rows[3, 1] = 3.0, 4.0
    out, norms = aspis.clip_rows(rows, 2.5)
    assert norms.tolist() == [0.0, 0.0, 0.0, 5.0]
    assert (float(rows[3, -1]), float(rows[3, 1])) == (1.5, 2.0)
    many = x[:2 ** 31].view(2 ** 17, 2 ** 14)
    many.zero_()
    many[-1, -1] = 8.0
    _, norms = aspis.clip_rows(many, 2.0)
    assert float(norms[-1]) == 8.0 and float(many[-1, -1]) == 2.0 and not norms[:-1].any()


# ----------------------------------------------------------------- refusals

def test_refusals():
    import torch
    dev = device()
    g = [torch.ones(10, device=dev), torch.ones(4, device=dev)]
    p = [torch.ones(10, device=dev), torch.ones(4, device=dev)]

    def refused(status, call):
        with pytest.raises(aspis.AspisError) as e:
            call()
        assert e.value.status == status, e.value

    bad = aspis.ERR_INVALID_ARG
    refused(bad, lambda: aspis.grad_norm([torch.ones(3)]))                          # host
    refused(bad, lambda: aspis.grad_norm([torch.ones(3, dtype=torch.float64, device=dev)]))
    refused(bad, lambda: aspis.grad_norm([torch.ones(3, device=dev).expand(2, 3)]))   # overlap
    refused(bad, lambda: aspis.grad_norm([torch.ones(8, device=dev)[::2]]))         # gaps
    refused(bad, lambda: aspis.grad_norm([1.0]))
    for bound in (-1.0, float("nan")):
        refused(bad, lambda: aspis.clip_grads(g, bound))
        refused(bad, lambda: aspis.clip_rows(g[0], bound))
    twice = torch.ones(10, device=dev)
    refused(bad, lambda: aspis.clip_grads([twice, twice[:4]], 1.0))
    assert float(aspis.grad_norm([twice, twice[:4]]).norm) == np.float32(math.sqrt(14))
    refused(bad, lambda: aspis.clip_grads(g, 1.0, out=[p[0]]))
    refused(bad, lambda: aspis.clip_grads(g, 1.0, out=[p[0], p[1].bfloat16()]))
    refused(bad, lambda: aspis.clip_grads([g[0].view(2, 5).t()], 1.0, out=[p[0].view(5, 2)]))
    refused(bad, lambda: aspis.clip_grads(g, 1.0, sumsq=torch.ones(1, device=dev)))
    refused(bad, lambda: aspis.grad_norm(g, ws=torch.empty(1, dtype=torch.uint8, device=dev)))
    refused(bad, lambda: aspis.grad_norm(g, each=True, bufs=aspis.NormBuffers.empty(dev, each=1)))
    refused(bad, lambda: aspis.clipped_sgd(p, g, lr=0.1, momentum=0.9))             # no mean
    refused(bad, lambda: aspis.clipped_sgd([t.half() for t in p], g, lr=0.1))
    refused(bad, lambda: aspis.clipped_sgd(p[:1], g, lr=0.1))
    refused(bad, lambda: aspis.clipped_sgd(p, g, lr=float("nan")))
    refused(bad, lambda: aspis.clipped_sgd(p, g, p, lr=0.1, momentum=1.0))
    refused(bad, lambda: aspis.clipped_sgd(p, g, lr=0.1, weight_decay=-1.0))
    refused(bad, lambda: aspis.clipped_adamw(p, g, g, g, step=0, lr=0.1))
    refused(bad, lambda: aspis.clipped_adamw(p, g, g, g, step=1, lr=0.1, betas=(1.0, 0.9)))
    refused(bad, lambda: aspis.clipped_adamw(p, g, g, g, step=1, lr=0.1, eps=-1.0))
    assert all(bool((t == 1).all()) for t in g + p)
    x = torch.ones(6, 8, device=dev)
    refused(bad, lambda: aspis.clip_rows(x.t(), 1.0))
    refused(bad, lambda: aspis.clip_rows(torch.ones(3, 4), 1.0))
    refused(bad, lambda: aspis.clip_rows(x[:5], 1.0, out=x[1:]))                    # overlap
    refused(bad, lambda: aspis.clip_rows(x, 1.0, out=torch.ones(6, 9, device=dev)))
    refused(bad, lambda: aspis.clip_rows(x, 1.0, out=x.half()))
    refused(bad, lambda: aspis.row_norms(x, norms=torch.ones(5, device=dev)))
    refused(bad, lambda: aspis.clip_rows(x, 1.0, flags=8))
    assert bool((x == 1).all())


def test_a_list_sees_a_type_or_layout_that_changes_in_place():
    """Same address, same number of elements: another type, another order."""
    import torch
    memory = _randn(600, "bfloat16", seed=4)
    t = memory.reshape(20, 30)
    handle, out = aspis.TensorList([t]), aspis.TensorList([torch.empty_like(t)])
    _assert_norm(aspis.grad_norm(handle).norm, _norm64([t]))
    t.data = memory.view(torch.float16).reshape(20, 30)
    assert t.data_ptr() == memory.data_ptr()
    _assert_norm(aspis.grad_norm(handle).norm, _norm64([t]))
    with pytest.raises(aspis.AspisError):   # out is still bfloat16
        aspis.clip_grads(handle, 1.0, out=out)
    t.data = memory.reshape(30, 20).t()
    with pytest.raises(aspis.AspisError):   # out has another order of elements
        aspis.clip_grads(handle, 1.0, out=out)
    same = [torch.empty_like(t)]
    norm = _norm64([t])
    aspis.clip_grads(handle, norm / 2, out=same)
    _assert_scaled(same[0], t, 0.5, "bfloat16")


def test_lists_that_overlap_are_refused():
    import torch
    flat = _randn(4000, seed=6)
    before = flat.clone()
    g, shifted = flat[:2000], flat[1000:3000]
    p, m, v = (_randn(2000, seed=7 + i).abs_() for i in range(3))
    for call in (lambda: aspis.clip_grads([g], 1.0, out=[shifted]),
                 lambda: aspis.clipped_sgd([p], [g], [p], lr=0.1, momentum=0.9),
                 lambda: aspis.clipped_sgd([shifted], [g], [m], lr=0.1, momentum=0.9),
                 lambda: aspis.clipped_adamw([p], [g], [m], [m], step=1, lr=0.1),
                 lambda: aspis.clipped_adamw([p], [g], [m], [v], step=1, lr=0.1, copies=[p]),
                 lambda: aspis.clipped_adamw([p], [g], [m], [v], step=1, lr=0.1,
                                             copies=[shifted])):
        with pytest.raises(aspis.AspisError, match="overlap"):
            call()
    assert bool((flat == before).all())
    # onto itself, and next to each other
    norm = _norm64([g])
    aspis.clip_grads([g], norm / 2, out=[flat[:2000]])
    _assert_scaled(g, before[:2000], 0.5, "float32")
    aspis.clip_grads([flat[:1000]], 1e9, out=[flat[1000:2000]])
    assert bool((flat[:1000] == flat[1000:2000]).all())


@pytest.mark.parametrize("sizes", [[], [900, 7], [300_001, 5]])
@pytest.mark.parametrize("call", ["clip", "sgd", "adamw"])
def test_the_sum_a_call_went_by_is_in_its_buffers(call, sizes):
    """With new buffers, kept ones and the sum already there."""
    import torch
    dev = device()
    as_list = lambda ts: aspis.TensorList(ts, device=dev)
    g, p, m, v = (as_list(_views(sizes, seed=s)) if sizes else as_list([]) for s in range(4))
    for t in v.tensors:
        t.square_()
    total = torch.tensor([6.25], dtype=torch.float64, device=dev)
    kept = aspis.NormBuffers.empty(dev)
    kept.sumsq.fill_(1e30)
    there = aspis.NormBuffers(kept.norm.clone(), total.clone())
    for bufs, given in ((None, total), (kept, total), (there, there.sumsq)):
        keep = {"sumsq": given, "bufs": bufs}
        if call == "clip":
            got = aspis.clip_grads(g, 0.5, **keep)
        elif call == "sgd":
            got = aspis.clipped_sgd(p, g, m, lr=0.1, momentum=0.9, max_norm=0.5, **keep)
        else:
            got = aspis.clipped_adamw(p, g, m, v, step=1, lr=0.1, max_norm=0.5, **keep)
        assert bufs is None or got is bufs
        assert got.norm.tolist() == [2.5] and got.sumsq.tolist() == [6.25]
        assert total.tolist() == [6.25]


@pytest.mark.parametrize("rule,n", [("sgd", 4), ("sgd", 70_000), ("sgd", 34_000_001), ("adamw", 4),
                                    ("adamw", 70_000), ("adamw", 12_000_003)])
def test_an_update_is_skipped_where_the_norm_returned_is_not_finite(rule, n):
    """Finite gradients whose norm passes the largest float32 are skipped,
    the largest float32 itself as a norm is not: what is returned decides."""
    import torch
    dev = device()
    top = float(np.finfo(np.float32).max)
    g = torch.zeros(n, device=dev)
    p, m, v = (torch.full((n,), x, device=dev) for x in (1.0, 0.5, 0.25))

    def go():
        if rule == "sgd":
            return aspis.clipped_sgd([p], [g], [m], lr=1.0, momentum=0.5, max_norm=1.0,
                                     skip_nonfinite=True)
        return aspis.clipped_adamw([p], [g], [m], [v], step=1, lr=1.0, betas=(0.5, 0.5),
                                   max_norm=1.0, skip_nonfinite=True)
    g[0] = g[-1] = top
    bufs = go()
    assert float(bufs.norm) == math.inf and math.isfinite(float(bufs.sumsq))
    assert bool((p == 1.0).all() and (m == 0.5).all() and (v == 0.25).all())
    g[-1] = 0.0
    bufs = go()
    assert float(bufs.norm) == top
    assert float(m[0]) == (1.25 if rule == "sgd" else 0.75)   # the clipped gradient is 1
    assert bool((m[1:] == 0.25).all()) and not bool((p == 1.0).any())


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
@pytest.mark.parametrize("chunks", [1, 2, 4, 5, 6, 8, 9, 12, 15, 16, 17, 40, 1025, 2768, 9001])
def test_every_call_sums_a_list_alike(chunks, kind):
    """The sum of squares has the same bits from the norm, with and without
    the tensors' own norms, the clip and the updates, whether one workgroup
    or many form it."""
    n = chunks * 4096 - 7
    part = 4096 * (chunks // 3)
    sizes = [n] if chunks < 3 else [part, n - part - 4096, 4096]
    ts = _views(sizes, kind, seed=chunks, offset=1)
    for t, scale in zip(ts, (1.0, 3.0, 0.1)):
        t.mul_(scale)
    p, m, v = (_views(sizes, seed=s) for s in (1, 2, 3))
    for t in v:
        t.square_()
    want = aspis.grad_norm(ts)
    exact = sum(float(t.double().square().sum()) for t in ts)
    assert abs(float(want.sumsq) - exact) <= 1e-12 * exact
    for got in (aspis.grad_norm(ts, each=True),
                aspis.clip_grads(ts, 1.0, out=[t.clone() for t in ts]),
                aspis.clipped_sgd(p, ts, m, lr=0.1, momentum=0.9, max_norm=1.0),
                aspis.clipped_adamw(p, ts, m, v, step=1, lr=0.1, max_norm=1.0),
                aspis.clip_grads(ts, 1.0)):
        assert float(got.sumsq) == float(want.sumsq) and float(got.norm) == float(want.norm)


# ------------------------- lists on both sides of every switch, and past the
# length from which they are walked from their end (16,384 chunks of 4,096)

EDGE_CHUNKS = [3, 4, 5, 8, 9, 16, 17]
PAST_THE_CACHE = 68_000_003


def _uneven(n):
    """Four tensors of n elements together, of very different sizes."""
    return [n // 3, 5, n // 7, n - n // 3 - 5 - n // 7]


def _of_chunks(chunks):
    """Tensors that take so many chunks, none a whole number of them."""
    return [4096 * (chunks - 2) - 7, 5, 4095] if chunks < 4 else \
        [4096 * (chunks - 3) - 7, 5, 4095, 100]


def _within(got, want, tol):
    return bool(((got.double() - want).abs() <= tol + 1e-44).all())


def _check_update_on_gpu(rule, sizes, kind, copy):
    import torch
    n, lr, wd = sum(sizes), 0.1, 0.01
    grads = _views(sizes, kind, seed=1, offset=1)
    params, mean = _views(sizes, seed=2, offset=2, scale=0.5), _views(sizes, seed=3, offset=3,
                                                                      scale=0.003)
    square = [v.square_() for v in _views(sizes, seed=4, offset=1, scale=0.003)]
    copies = list(torch.full((n + 1,), 9.0, dtype=_type(copy), device=device())[1:].split(sizes))
    norm = math.sqrt(sum(float(g.double().square().sum()) for g in grads))
    start = [[t.clone() for t in x] for x in (params, mean, square)]
    keep = {"lr": lr, "weight_decay": wd, "max_norm": 0.3 * norm, "copies": copies}
    if rule == "sgd":
        bufs = aspis.clipped_sgd(params, grads, mean, momentum=0.9, **keep)
    elif rule == "plain":
        bufs = aspis.clipped_sgd(params, grads, **keep)
    else:
        bufs = aspis.clipped_adamw(params, grads, mean, square, step=3, betas=(0.9, 0.95), **keep)
    _assert_norm(bufs.norm, norm)
    for i in range(len(sizes)):
        g = 0.3 * grads[i].double()
        p, m, v = (x[i].double() for x in start)
        if rule == "adamw":
            m_tol = 6 * U * (0.9 * m.abs() + 0.1 * g.abs())
            m, v = 0.9 * m + 0.1 * g, 0.95 * v + 0.05 * g * g
            rate, root = lr / (1 - 0.9 ** 3), (v / (1 - 0.95 ** 3)).sqrt() + 1e-8
            p_tol = 4 * U * p.abs() + rate * (m_tol + 16 * U * m.abs()) / root
            p = p * (1 - lr * wd) - rate * m / root
            assert _within(square[i], v, 8 * U * v)
            assert _within(mean[i], m, m_tol)
        else:   # the roundings that _sgd64 counts
            mu = 0.9 if rule == "sgd" else 0.0
            g = g + wd * p
            step = mu * m + g
            size = (1 + mu) * (g.abs() + 2 * wd * p.abs() + 2 * mu * step.abs())
            p_tol, p = 8 * U * (p.abs() + lr * size), p - lr * step
            if mu:
                assert _within(mean[i], step, 8 * U * size)
        assert _within(params[i], p, p_tol)
        assert bool((copies[i] == params[i].to(copies[i].dtype)).all())


@pytest.mark.parametrize("chunks", EDGE_CHUNKS)
@pytest.mark.parametrize("rule", ["sgd", "plain", "adamw"])
@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
def test_updates_at_the_switches(rule, chunks, kind):
    sizes = _of_chunks(chunks)
    assert sum(-(-n // 4096) for n in sizes) == chunks
    _check_update_on_gpu(rule, sizes, kind, "float16")


@pytest.mark.parametrize("rule,n,kind", [("plain", 34_000_001, "float32"),
                                         ("plain", 34_000_001, "float16"),
                                         ("adamw", 11_000_003, "bfloat16"),
                                         ("sgd", PAST_THE_CACHE, "float32"),
                                         ("plain", PAST_THE_CACHE, "bfloat16"),
                                         ("adamw", PAST_THE_CACHE, "float32"),
                                         ("adamw", PAST_THE_CACHE, "float16")])
def test_updates_of_lists_past_the_cache(rule, n, kind):
    _check_update_on_gpu(rule, _uneven(n), kind, "bfloat16")


def _check_clip_on_gpu(sizes, kind, where):
    import torch
    ts = _views(sizes, kind, seed=5, offset=1)
    for t, scale in zip(ts, (1.0, 40.0, 3.0, 0.2)):
        t.mul_(scale)
    before = [t.clone() for t in ts]
    squares = [float(t.double().square().sum()) for t in ts]
    norm = math.sqrt(sum(squares))
    each = aspis.grad_norm(ts, each=True).each.tolist()
    for got, s in zip(each, squares):
        _assert_norm(got, math.sqrt(s))
    out = None if where == "in_place" else \
        list(torch.full((sum(sizes) + 3,), 7.0, dtype=_type(kind),
                        device=device())[3:].split(sizes))
    _assert_norm(aspis.clip_grads(ts, 0.4 * norm, out=out).norm, norm)
    for got, x in zip(ts if out is None else out, before):
        want = 0.4 * x.double()
        assert _within(got, want, want.abs() * (2 * U * (1 + 1e-6) + HALF_ULP[kind] * (1 + 1e-5))
                       + 1.5 * TINY[kind])
    if out is not None:
        assert all(bool((t == b).all()) for t, b in zip(ts, before))


@pytest.mark.parametrize("chunks", EDGE_CHUNKS)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("where", ["in_place", "out"])
def test_clips_at_the_switches(chunks, kind, where):
    _check_clip_on_gpu(_of_chunks(chunks), kind, where)


@pytest.mark.parametrize("n,kind", [(11_000_003, "float32"), (PAST_THE_CACHE, "float32"),
                                    (PAST_THE_CACHE, "bfloat16"), (150_000_001, "float16")])
@pytest.mark.parametrize("where", ["in_place", "out"])
def test_clips_of_lists_past_the_cache(n, kind, where):
    _check_clip_on_gpu(_uneven(n), kind, where)


def test_calls_on_plain_sequences_do_not_wait():
    """The host is back while the stream still works on what came before, and
    the results are those of kept lists."""
    import torch
    dev = device()
    sizes = [70_001, 5, 300]
    a = torch.randn(8192, 8192, device=dev).bfloat16()
    b = torch.empty_like(a)

    def lists():
        g, p, m, v = (_views(sizes, seed=s) for s in (1, 2, 3, 4))
        for t in v:
            t.square_()
        return g, p, m, v

    def go(wrap, g, p, m, v):
        norm = aspis.grad_norm(wrap(g), each=True)
        aspis.clipped_sgd(wrap(p), wrap(g), wrap(m), lr=0.1, momentum=0.9, max_norm=0.5)
        aspis.clipped_adamw(wrap(p), wrap(g), wrap(m), wrap(v), step=2, lr=0.1, max_norm=0.5)
        aspis.clip_grads(wrap(g), 0.25, out=wrap([t.clone() for t in g]))
        aspis.clip_grads(wrap(g), 0.25)
        return [norm.norm, norm.each, *g, *p, *m, *v]
    want = go(aspis.TensorList, *lists())
    go(list, *lists())   # memory for all of it is there
    tensors = lists()
    torch.cuda.synchronize()
    for _ in range(300):   # some hundred milliseconds
        torch.mm(a, a, out=b)
    done = torch.cuda.Event()
    done.record()
    got = go(list, *tensors)
    assert not done.query()
    torch.cuda.synchronize()
    assert all(np.array_equal(_bits(x), _bits(y)) for x, y in zip(got, want))


def test_plain_sequences_are_refused_in_a_capture():
    """... by a message, and the capture goes on; kept lists capture."""
    import torch
    dev = device()
    x, y = _randn(5_000, seed=1), torch.empty(5_000, device=dev)
    handle, out = aspis.TensorList([x]), aspis.TensorList([y])
    bufs, ws = aspis.NormBuffers.empty(dev), aspis.norm_workspace(handle)
    norm = _norm64([x])
    aspis.clip_grads(handle, norm / 2, out=out, bufs=bufs, ws=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for call in (lambda: aspis.grad_norm([x]), lambda: aspis.TensorList([x]),
                     lambda: aspis.clip_grads(handle, 1.0, out=[y])):
            with pytest.raises(aspis.AspisError, match="captured"):
                call()
        aspis.clip_grads(handle, norm / 2, out=out, bufs=bufs, ws=ws)
    for replay in range(3):
        x.copy_(_randn(5_000, seed=7 + replay))
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        _assert_norm(bufs.norm, _norm64([x]))
        _assert_scaled(y, x, _coef64(_norm64([x]), norm / 2), "float32")


SIGNALLING = {"float32": 0x7F800001, "bfloat16": 0x7F81, "float16": 0x7C01}


def _with_signalling_nans(x, kind):
    """x with signalling NaNs in places of a 16-byte load and of a tail."""
    import torch
    ints = x.view(torch.int32 if kind == "float32" else torch.int16)
    for row in ints.reshape(-1, x.shape[-1]):
        for i in {0, row.numel() // 2, row.numel() - 1}:
            row[i] = SIGNALLING[kind]
    return x


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n", [1, 7, 4_095, 70_001, 40_000_003])
@pytest.mark.parametrize("offset", [0, 1])
def test_no_bound_returns_a_lists_own_bits(n, kind, offset):
    import torch
    x = _with_signalling_nans(_randn(n + offset, kind, seed=n)[offset:], kind)
    out = torch.zeros_like(x)
    aspis.clip_grads([x], math.inf, out=[out])
    assert np.array_equal(_bits(out), _bits(x))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,d", [(70, 3), (70, 50), (9, 300), (5, 1_001), (5, 10_007), (3, 32_767),
                                    (3, 50_001), (2, 100_003), (40, 300_001), (3, 7_000_001),
                                    (1, 25_000_003)])
def test_no_bound_returns_the_rows_own_bits(rows, d, kind):
    import torch
    x = _with_signalling_nans(_randn(rows * d + 1, kind, seed=d)[1:].reshape(rows, d), kind)
    for flags in (0, aspis.CLIP_NO_WAIT):
        out, _ = aspis.clip_rows(x, math.inf, out=torch.zeros_like(x), flags=flags)
        assert np.array_equal(_bits(out), _bits(x))


def test_the_norms_of_no_tensors_are_an_empty_tensor():
    import torch
    none = aspis.TensorList([], device=device())
    for bufs in (None, aspis.NormBuffers.empty(device(), each=len(none))):
        got = aspis.grad_norm(none, each=True, bufs=bufs)
        assert got.each.dtype == torch.float32 and got.each.shape == (0,)
        assert float(got.norm) == 0.0
    assert aspis.grad_norm(none).each is None


def test_adamw_by_a_given_sum_in_a_graph():
    """What a call took by value is what every replay goes by (the step, and
    so the bias correction); what it took on the device is read anew (the
    gradients, the sum of squares)."""
    import torch
    dev, sizes, step = device(), [70_001, 513], 5
    grads = aspis.TensorList(_views(sizes, "bfloat16", seed=1))
    params, mean, square = (aspis.TensorList(_views(sizes, seed=s)) for s in (2, 3, 4))
    for t in square.tensors:
        t.square_()
    copies = aspis.TensorList([torch.empty(n, dtype=torch.bfloat16, device=dev) for n in sizes])
    bufs, ws = aspis.NormBuffers.empty(dev), aspis.norm_workspace(grads)
    total = torch.ones(1, dtype=torch.float64, device=dev)

    def go():
        aspis.clipped_adamw(params, grads, mean, square, step=step, lr=0.1, max_norm=0.5,
                            copies=copies, sumsq=total, bufs=bufs, ws=ws)
    state = [t for x in (params, mean, square, copies) for t in x.tensors]
    start = [t.clone() for t in state]

    def reset():
        for t, k in zip(state, start):
            t.copy_(k)
    go()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    for replay in range(4):
        reset()
        for i, t in enumerate(grads.tensors):
            t.copy_(_randn(t.numel(), "bfloat16", seed=50 + 7 * replay + i))
        total.fill_(2.0 + replay)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in state] + [bufs.norm.clone(), bufs.sumsq.clone().float()]
        reset()
        go()
        torch.cuda.synchronize()
        want = state + [bufs.norm, bufs.sumsq.float()]
        assert all(np.array_equal(_bits(a), _bits(b)) for a, b in zip(got, want)), replay
        assert bufs.sumsq.tolist() == [2.0 + replay]


def test_negated_views_are_refused():
    """The imaginary parts of conjugates: memory that holds the opposite."""
    import torch
    dev = device()
    z = torch.complex(torch.full((5, 1), 3.0, device=dev), torch.full((5, 1), 4.0, device=dev))
    rows, one = z.conj().imag, z.conj().imag[:1, 0]
    assert rows.is_neg() and one.is_neg() and one.is_contiguous()
    x = torch.ones(1, device=dev)
    total = torch.ones(1, dtype=torch.complex128, device=dev).conj().imag
    for call in (lambda: aspis.clip_rows(rows, 1.0, out=torch.empty(5, 1, device=dev)),
                 lambda: aspis.clip_rows(one, 1.0), lambda: aspis.row_norms(rows),
                 lambda: aspis.clip_rows(x, 1.0, out=one), lambda: aspis.grad_norm([one]),
                 lambda: aspis.clip_grads([x], 1.0, out=[one]),
                 lambda: aspis.row_norms(x, norms=one.view(())),
                 lambda: aspis.clip_grads([x], 1.0, sumsq=total)):
        with pytest.raises(aspis.AspisError, match="negated"):
            call()
    assert bool((z.imag == 4.0).all()) and float(x) == 1.0
    out, norms = aspis.clip_rows(rows.resolve_neg(), 1.0)
    assert bool((out == -1.0).all() and (norms == 4.0).all())
