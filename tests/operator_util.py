"""Plain implementations in 64 bits of the operators around the AllReduce, and the bounds their kernels
are held to.

The bounds follow from the arithmetic, with u = 2^-24 the unit roundoff of fp32. A sum of a row's
values passes at most SUM = 80 roundings: 16 values a lane (64 in the balance kernels), 6 exchanges
within a wave, 16 waves' sums; rows of more than 16384 values add one for every further round of
1024 lanes' vectors, which the tests' rows have at most five of. Outputs in 16 bits add half a unit
of their own last place."""

import math

import torch

U = 2.0 ** -24
SUM = 80
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def rounding(want, dtype):
    """Half a unit in the last place of `dtype` at the values `want`."""
    if dtype == torch.float32:
        return U * want.abs()
    if dtype == torch.bfloat16:
        return 2.0 ** -8 * want.abs()
    return 2.0 ** -11 * want.abs() + 2.0 ** -25


def assert_within(got, want, bound, what):
    got = got.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what + ": NaN in other places"
    err = (got - want).abs()
    bad = err > bound
    assert not bool(bad.any()), "%s: %d of %d values off, the worst by %.3g times the bound" % (
        what, int(bad.sum()), bad.numel(), float((err / bound.clamp(min=1e-300))[bad].max()))


def layernorm_forward(x, gamma, beta, eps):
    """y, mean, rstd of double rows and the bounds of fp32 arithmetic on them."""
    mean = x.mean(-1)
    d = x - mean[..., None]
    rstd = 1 / torch.sqrt((d * d).mean(-1) + eps)
    h = d * rstd[..., None]
    y = h * gamma + beta
    size = x.abs().mean(-1)
    off = SUM * U * size  # of the mean
    # the variance: roundings of the sum, and the square of the mean's error
    rel = SUM * U + (off * rstd) ** 2
    bound = gamma.abs() * (rstd * off)[..., None] \
        + gamma.abs() * h.abs() * (rel + 8 * U)[..., None] + 4 * U * (y.abs() + beta.abs())
    return (y, bound), (mean, off + U * mean.abs() + 1e-45), (rstd, rstd * (rel + 8 * U))


def layernorm_backward(dy, x, gamma, mean, rstd):
    """dx, dgamma, dbeta [ranks, width] of double [ranks, tokens, width] rows, with bounds; mean and
    rstd are the fp32 values that the kernel reads."""
    r = rstd[..., None]
    h = (x - mean[..., None]) * r
    g = dy * gamma
    s1, s2 = g.mean(-1, keepdim=True), (g * h).mean(-1, keepdim=True)
    dx = r * (g - s1 - h * s2)
    a1, a2 = g.abs().mean(-1, keepdim=True), (g * h).abs().mean(-1, keepdim=True)
    bound = r * U * (8 * g.abs() + (SUM + 8) * a1 + (SUM + 16) * h.abs() * a2)
    # a lane adds its rows one by one, and a workgroup its at most 32 groups
    n = (x.shape[1] + 40) * U
    return (dx, bound), ((dy * h).sum(1), n * (dy * h).abs().sum(1)), (dy.sum(1), n * dy.abs().sum(1))


def softmax(logits):
    """Probabilities of double logits, zero where all are -inf, and the relative bound of fp32 ones: an
    exponent rounds by u times its size, and the sum by its roundings."""
    top = logits.amax(-1, keepdim=True)
    none = torch.isneginf(top)
    z = logits - torch.where(none, torch.zeros_like(top), top)
    e = torch.exp(z)
    s = e.sum(-1, keepdim=True)
    p = torch.where(none, torch.zeros_like(e), e / torch.where(none, torch.ones_like(s), s))
    far = torch.where(torch.isinf(z), torch.zeros_like(z), z.abs()).amax(-1, keepdim=True)
    return p, (2 * far + SUM + 16) * U


def balance_counts(logits, chosen, mask):
    """counts [ranks, experts + 1], and (probs, bound), of double logits."""
    ranks, tokens, experts = logits.shape
    live = torch.ones((ranks, tokens), dtype=torch.bool, device=logits.device) if mask is None else mask.bool()
    counts = torch.zeros((ranks, experts + 1), dtype=torch.int64)
    for r in range(ranks):
        ids = chosen[r][live[r]].long().flatten().cpu()
        ids = ids[(ids >= 0) & (ids < experts)]
        counts[r, :experts] = torch.bincount(ids, minlength=experts)
        counts[r, experts] = int(live[r].sum())
    p, rel = softmax(torch.where(live[..., None], logits, torch.zeros_like(logits)))
    p = torch.where(live[..., None], p, torch.zeros_like(p))
    return counts, (p.sum(1), (p * (rel + (tokens + 40) * U)).sum(1) + 1e-45)


def balance_loss(counts, probs, top_k, scale):
    c, n = counts[:, :-1].double(), counts[:, -1].double()
    loss = scale * c.shape[1] * (c * probs.double()).sum(1) / (top_k * n * n)
    return torch.where(n > 0, loss, torch.zeros_like(loss))


def balance_backward(logits, counts, top_k, mask, scale, dloss):
    """(dlogits, bound) of double logits."""
    ranks, tokens, experts = logits.shape
    live = torch.ones((ranks, tokens), dtype=torch.bool, device=logits.device) if mask is None else mask.bool()
    c, n = counts[:, :-1].double(), counts[:, -1:].double()
    w = torch.where(n > 0, scale * experts * c / (top_k * n * n), torch.zeros_like(c))
    if dloss is not None:
        w = w * dloss.double()[:, None]
    w = w[:, None, :]
    p, rel = softmax(torch.where(live[..., None], logits, torch.zeros_like(logits)))
    d = p * (w - (p * w).sum(-1, keepdim=True))
    bound = p * (rel + (SUM + 16) * U) * 2 * (w.abs() + (p * w).abs().sum(-1, keepdim=True)) + 1e-45
    return (torch.where(live[..., None], d, torch.zeros_like(d)),
            torch.where(live[..., None], bound, torch.zeros_like(bound)))


def orthogonalize(x, coefficients, scale, eps):
    """(out, bound of the Frobenius norm of its error) for each double matrix. A step's error: stored
    numbers have 22 bits and a half unit in the last place, sums of K products round about sqrt(K) times,
    each weighted with the terms a, b A, c A A that it enters; later steps stretch it by the largest
    slope of their polynomials or the largest factor of a singular value, 4 at most for the steps
    used here."""
    outs, bounds = [], []
    for g in x:
        tall = g.shape[0] > g.shape[1]
        v = g.T if tall else g
        v = v / (torch.linalg.matrix_norm(v) + eps)
        depth = max(v.shape)
        unit = 2.0 ** -22 + math.sqrt(depth) * U
        bound = 0.0
        for a, b, c in coefficients:
            # before the step: what earlier steps left, and this one's own, by its inputs' norm
            bound = 4 * bound + (abs(a) + 2 * abs(b) + 3 * abs(c)) * unit * float(torch.linalg.matrix_norm(v))
            q = v @ v.T
            v = a * v + (b * q + c * (q @ q)) @ v
        outs.append(scale * (v.T if tall else v))
        bounds.append(abs(scale) * bound)
    return torch.stack(outs), bounds
