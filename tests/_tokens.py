"""Plain forms of the token operators, in 64 bits and on the host (shared by
the GPU tests; not collected by pytest)."""
import math

import numpy as np

U = 2.0 ** -24                      # half an f32 ulp, relative to the value
HALF_ULP = {"float32": 0.0, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
TINY = {"float32": 2.0 ** -149, "bfloat16": 2.0 ** -133, "float16": 2.0 ** -24}


def f64(t):
    return t.detach().double().cpu().numpy()


def philox(key: int, counters: np.ndarray) -> np.ndarray:
    """Philox4x32-10 blocks [n, 4] (uint32) of counters [n] (uint64)."""
    low, up = np.uint64(0xFFFFFFFF), np.uint64(32)
    c = [counters & low, counters >> up, np.zeros_like(counters), np.zeros_like(counters)]
    for i in range(10):
        k = [np.uint64(((key & 0xFFFFFFFF) + i * 0x9E3779B9) & 0xFFFFFFFF),
             np.uint64(((key >> 32) + i * 0xBB67AE85) & 0xFFFFFFFF)]
        p, q = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(q >> up) ^ c[1] ^ k[0], q & low, (p >> up) ^ c[3] ^ k[1], p & low]
    return np.stack(c, axis=1).astype(np.uint32)


def kept(n: int, p: float, seed: int, offset: int) -> np.ndarray:
    """Which of n elements dropout keeps."""
    q = np.array([offset & (2 ** 64 - 1)], dtype=np.uint64) + np.arange(n, dtype=np.uint64)
    first = int(q[0]) >> 3 if n else 0
    blocks = np.array([first], dtype=np.uint64) + np.arange((n + 14) // 8, dtype=np.uint64)
    blocks &= np.uint64(2 ** 61 - 1)
    words = philox(seed & (2 ** 64 - 1), blocks)
    halves = words.astype("<u4").view("<u2").reshape(-1)
    at = (int(q[0]) & 7) if n else 0
    return halves[at:at + n] >= round(p * 65536)


def embedded(table, tokens, scale):
    """scale * table[token], zeros outside the table."""
    t = np.asarray(tokens).reshape(-1)
    there = (t >= 0) & (t < len(table))
    out = np.zeros((len(t), table.shape[1]))
    out[there] = scale * table[t[there]]
    return out


def embed_sums(grad, tokens, vocab):
    """Sums of grad by token, of their magnitudes, and how many there are."""
    t = np.asarray(tokens).reshape(-1)
    there = (t >= 0) & (t < vocab)
    sums, sizes = np.zeros((vocab, grad.shape[1])), np.zeros((vocab, grad.shape[1]))
    np.add.at(sums, t[there], grad[there])
    np.add.at(sizes, t[there], np.abs(grad[there]))
    return sums, sizes, np.bincount(t[there], minlength=vocab)


class Policy:
    """The policy loss and its gradient in 64 bits, with bounds on what f32
    arithmetic may add.

    With x_v = (z_v - M) / T: a power's exponent carries three roundings (the
    difference, the constant, the product) and the power itself one f32 ulp, so
    each power is off by (3 |x| + 2) U of itself.  Sums of at most 200 terms
    one after the other (128 of a thread, then lanes, waves and parts) add 200 U of
    S.  log p adds the logarithm's ulp and the roundings of its two terms and
    of the result."""

    def __init__(self, z, tokens, old=None, adv=None, weight=None, ref=None, clip=(0.2, 0.2),
                 kl=0.0, temperature=1.0, grad_scale=1.0):
        rows, vocab = z.shape
        t = np.asarray(tokens).reshape(-1)
        w = np.ones(rows) if weight is None else weight.astype(float)
        self.used = (t >= 0) & (t < vocab) & (w != 0)
        at = np.where(self.used, t, 0)
        r = np.arange(rows)
        with np.errstate(all="ignore"):
            top = z.max(1, keepdims=True)
            x = (z - top) / temperature
            e = np.exp(x)
            s = e.sum(1, keepdims=True)
            p = e / s
            lp = x[r, at] - np.log(s[:, 0])
            spread = np.where(p > 0, p * np.abs(x), 0.0).sum(1)
            self.rel_s = U * (3 * spread + 202)
            self.logps = np.where(self.used, lp, 0.0)
            self.logps_tol = 1.01 * np.where(
                self.used, self.rel_s + U * (3 * np.abs(np.log(s[:, 0])) + 3 * np.abs(x[r, at])
                                             + np.abs(lp)), 0.0) + 1e-30
            if old is None:
                return
            d_lp = self.logps_tol
            ratio = np.exp(lp - old)
            lo, hi = 1 - clip[0], 1 + clip[1]
            cut = np.where(adv > 0, ratio > hi, (adv < 0) & (ratio < lo))
            gain = np.where(adv == 0, 0.0, np.where(cut, np.where(adv > 0, hi, lo), ratio) * adv)
            slope = np.where(cut, 0.0, -gain)
            # the ratio: log p's error, the difference's rounding, the power's ulp
            gain_tol = np.abs(gain) * (d_lp + U * (np.abs(lp - old) + 6))
            k, k_tol, rise, rise_tol = (np.zeros(rows) for _ in range(4))
            if ref is not None:
                d = ref - lp
                rise = -np.expm1(d)
                k = np.expm1(d) - d
                d_err = d_lp + U * np.abs(d)
                # the rest's slope is e^d - 1; its evaluation adds 8 U of it, and
                # off the series 6 U of what it subtracts
                far = np.where(np.abs(d) > 0.49, np.exp(d) + 1 + np.abs(d), 0.0)
                k_tol = np.abs(rise) * d_err + np.exp(d) * d_err ** 2 + U * (8 * k + 6 * far)
                rise_tol = np.exp(d) * d_err + k_tol + 4 * U * (np.abs(d) + np.abs(k))
            self.loss = kl * k - gain
            slope = slope + kl * rise
            slope_tol = np.where(cut, 0.0, gain_tol) + kl * rise_tol + 4 * U * (
                np.abs(gain) + kl * (np.abs(rise) + np.abs(k)))
            self.ratio, self.cut = ratio, cut
            zero = np.zeros(rows)
            terms = [np.where(self.used, w * v, zero) for v in (self.loss, k, cut)]
            self.sums = np.array([v.sum() for v in terms])
            loss_tol = gain_tol + kl * k_tol + 4 * U * (np.abs(gain) + kl * np.abs(k))
            self.sums_tol = np.array([
                np.where(self.used, np.abs(w) * tol, zero).sum() for tol in
                (loss_tol, k_tol, zero)]) + 2 * U * np.array(
                    [np.abs(v).sum() for v in terms]) + 1e-30
            coef = grad_scale * w * slope / temperature
            coef_tol = np.abs(grad_scale * w / temperature) * slope_tol + 4 * U * np.abs(coef)
            g = -coef[:, None] * p
            # a power's error and the sum's, then two products
            p_tol = p * (U * (3 * np.abs(np.where(p > 0, x, 0.0)) + 6) + self.rel_s[:, None])
            g_tol = np.abs(coef)[:, None] * p_tol + coef_tol[:, None] * p
            own = p[r, at]
            g[r, at] = coef * (1 - own)
            g_tol[r, at] = np.abs(coef) * (p_tol[r, at] + 2 * U) + coef_tol * (1 - own)
            self.grad = np.where(self.used[:, None], g, 0.0)
            # powers below the smallest normal f32 may be taken as 0
            small = 2.0 ** -125 * np.abs(coef)[:, None]
            self.grad_tol = np.where(self.used[:, None], 1.01 * g_tol + small, 0.0)

    def check_logps(self, got):
        got = f64(got).reshape(-1)
        bad = ~(np.abs(got - self.logps) <= self.logps_tol)
        assert not bad.any(), (np.flatnonzero(bad)[:4], got[bad][:4], self.logps[bad][:4],
                               self.logps_tol[bad][:4])

    def check_grad(self, got, kind):
        got = f64(got).reshape(self.grad.shape)
        tol = self.grad_tol + np.abs(self.grad) * HALF_ULP[kind] * 1.01 + TINY[kind]
        bad = ~(np.abs(got - self.grad) <= tol)
        assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist(), got[bad][:4],
                               self.grad[bad][:4], tol[bad][:4])

    def check_sums(self, got):
        got = f64(got)
        assert (np.abs(got - self.sums) <= self.sums_tol).all(), (got, self.sums, self.sums_tol)


def policy_inputs(rows, vocab, seed=0, kind="float32", masked=0.3, spread=2.0, temperature=1.0,
                  clip=(0.2, 0.2)):
    """Logits and what goes with them, as numpy arrays; ratios lie off the
    clip's borders, where the loss has two slopes."""
    import torch
    rng = np.random.default_rng(seed)
    z = torch.from_numpy(spread * rng.standard_normal((rows, vocab))).to(getattr(torch, kind))
    tokens = rng.integers(0, vocab, rows)
    ref = Policy(f64(z), tokens, temperature=temperature)
    lp = ref.logps
    ratio = np.exp(rng.normal(0, 0.2, rows))
    for border in (1 - clip[0], 1 + clip[1]):
        ratio = np.where(np.abs(ratio / border - 1) < 1e-2, ratio * 1.03, ratio)
    old = (lp - np.log(ratio)).astype(np.float32)
    refs = (lp + rng.normal(0, 0.3, rows)).astype(np.float32)
    adv = rng.standard_normal(rows).astype(np.float32)
    weight = np.full(rows, 1.0 / rows, dtype=np.float32)
    weight[rng.random(rows) < masked] = 0.0
    return z, tokens, old, adv, weight, refs


def softmax_loss(z, tokens, old, adv, weight, ref, clip, kl, temperature):
    """The loss alone, straight from its formula (for differences)."""
    x = z / temperature
    top = x.max(1, keepdims=True)
    lp = (x - top - np.log(np.exp(x - top).sum(1, keepdims=True)))[np.arange(len(z)), tokens]
    r = np.exp(lp - old)
    gain = np.minimum(r * adv, np.clip(r, 1 - clip[0], 1 + clip[1]) * adv)
    k = np.exp(ref - lp) - 1 - (ref - lp)
    return math.fsum(weight * (kl * k - gain))
