"""Plain 64-bit forms of the 8-bit projections and of the scores of tokens, and
the bounds on a float32 kernel's distance from them.

U = 2^-24 is half a float32 step relative to the value.  Each bound counts
roundings: one for an addition, product, division or square root, four for an
exponential or logarithm (two units in the last place), n for a chain of n
additions.
"""
import math

import torch

U = 2.0 ** -24
TINY = 2.0 ** -100
HALF_STEP = {torch.float32: U, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
# below the normal range a float16 is off by half of its smallest step
SMALLEST = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25}


def gemm(a, sa, w, sw):
    # float64 holds sums of products below 2^53 exactly
    return (a.double() @ w.double().t()) * (sa.double()[:, None] * sw.double())


def check_gemm(out, a, sa, w, sw):
    """The exact sum is rounded to float32, and so are the product of the scales
    and the product of both: 3 U, then once to the output's type."""
    ref = gemm(a, sa, w, sw)
    tol = ref.abs() * (4 * U + HALF_STEP[out.dtype]) + SMALLEST[out.dtype]
    bad = ~((out.double() - ref).abs() <= tol)
    assert not bool(bad.any()), (int(bad.sum()), float(((out.double() - ref).abs() - tol).max()))


def swiglu(x, d):
    g, u = x[:, :d].double(), x[:, d:].double()
    return g * torch.sigmoid(g) * u


def check_codes(q, scale, y, rel):
    """Codes and scales of rows whose float32 values are within rel of y (64 bits)."""
    assert q.dtype == torch.int8 and scale.dtype == torch.float32
    amax = y.abs().amax(1)
    tiny = amax < TINY
    s = torch.where(tiny, 0.0, amax / 127)
    # the largest magnitude is within rel, and the division rounds once
    assert bool(((scale.double() - s).abs() <= s * (rel + 2 * U)).all())
    assert not bool(q[tiny].any())
    # y * (127 / amax): rel twice and two roundings, of a value up to 127; then half a step
    off = (q.double() - torch.where(tiny[:, None], 0.0, y / torch.where(tiny, 1.0, s)[:, None])).abs()
    assert float(off.max()) <= 0.5 + 127 * (2 * rel + 4 * U), float(off.max())
    # the largest value of a row has the largest code
    assert bool((q.abs().amax(1)[~tiny] == 127).all())


def norm(r, gain, eps):
    r = r.double()
    return r / torch.sqrt((r * r).mean(1, keepdim=True) + eps) * gain.double()


def norm_rel(d):
    """Squares summed in chains of at most max(16, d / 256), and 16 more additions
    to join them; halved by the square root; mean, eps, root, inverse and two
    products after it."""
    return ((max(16, d / 256) + 16) / 2 + 6) * U


SWIGLU_REL = 12 * U      # an exponential, an addition, a division, a product; the sum's own size


def scores(logits, mask_id):
    x = logits.double().clone()
    if mask_id >= 0:
        x[:, mask_id] = -math.inf
    m = x.amax(1, keepdim=True)
    logp = (x - m) - (x - m).exp().sum(1, keepdim=True).log()
    p = logp.exp()
    return x, logp, -torch.where(p == 0, 0.0, p * logp).sum(1)


SCORES_REL = 3 * U       # two roundings of the value itself, and one to spare


def scores_tol(vocab):
    """z = sum exp(x - m): a term e^y is off by |y| U (the difference's rounding),
    1.3 |y| U (y log2(e), of a constant that is itself off by a quarter of U) and
    4 U; weighted by e^y / z, |y| averages to at most ln vocab + 1.  The sum is at
    most max(32, vocab / 256) additions in a chain, each with a move to another
    maximum at most every 16th (6 U), and 16 joins of 6 U.  t = sum y e^y is at
    most z (ln vocab + 1) in size and off by the same relative amount and one
    product.  The logarithm and the quotient round values of up to 40 (4 U each).
    To be added for a log probability: x - m and the last difference each round a
    value of about its own size, which can be thousands: SCORES_REL."""
    chain = max(32, vocab / 256)
    return (math.log(vocab) + 2) * (1.4 * chain + 102 + 3 * (math.log(vocab) + 1)) * U + 40 * 8 * U


def top(x, k):
    """Ids of the k largest finite logits, lower id first on ties, -1 past them."""
    x = torch.where(torch.isnan(x), -math.inf, x)
    v, i = torch.sort(x, dim=1, descending=True, stable=True)
    pad = max(0, k - x.shape[1])
    v = torch.nn.functional.pad(v[:, :k], (0, pad), value=-math.inf)
    i = torch.nn.functional.pad(i[:, :k], (0, pad), value=-1)
    return torch.where(v > -math.inf, i, -1).int()
