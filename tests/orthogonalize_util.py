"""Newton-Schulz steps in 64 bits and as plain fp32 products, and how far a result may be from the
former, measured by the latter.

The kernels hold matrices in two fp16 numbers: a half unit in the last place of 2^-23 of a value where
fp32 has 2^-24. A step rounds three such matrices (A, P and X); the plain form rounds five (b A, c A A,
their sum, its product with X, and the sum with a X) at half the size, and its products sum in fp32
as the kernels' do. So the kernels' error is at most about twice the plain form's where rounding a matrix
outweighs rounding the sums, and about the same otherwise. NEAR leaves room for both sides' chance."""

import torch

QUINTIC = ((3.4445, -4.7750, 2.0315),) * 5
NEAR = 3.0  # times the plain form's error
FAR_SUMS = 2.0  # the same from 512 rows on, where the sums' roundings weigh as much in both

# A size for every way that a call can run (what tests/c/orthogonalize_plan.cpp prints), none of which fills its
# tiles; some taller than wide.
FORMS = {
    "small": (2, 61, 250),
    "strips": (1, 8100, 50),
    "gram-64few polynomial-64few update-64few": (1, 65, 66),
    "gram-64few polynomial-64few update-64": (64, 129, 66),
    "gram-64few polynomial-64few update-128": (64, 67, 322),
    "gram-64few-shared polynomial-64few update-64few": (1, 8193, 3),
    "gram-64few-shared polynomial-64few update-64": (1, 33, 20003),
    "gram-64few-shared polynomial-64few update-128": (3, 5452, 68),
    "gram-64few-shared polynomial-64few update-256": (1, 193, 49365),
    "gram-64 polynomial-64 update-64": (64, 130, 132),
    "gram-64 polynomial-64 update-128": (16, 344, 332),
    "gram-64-shared polynomial-64 update-64": (4, 673, 1290),
    "gram-64-shared polynomial-64-shared update-64": (1, 1547, 2486),
    "gram-128 polynomial-128 update-64": (8, 740, 656),
    "gram-128 polynomial-128 update-128": (64, 193, 203),
    "gram-128 polynomial-128 update-256": (64, 780, 197),
    "gram-128-shared polynomial-128 update-64": (8, 509, 1054),
    "gram-128-shared polynomial-128 update-128": (8, 917, 457),
    "gram-128-shared polynomial-128 update-256": (8, 728, 1307),
    "gram-128-shared polynomial-128-shared update-64": (1, 833, 1552),
    "gram-128-shared polynomial-128-shared update-128": (1, 2413, 838),
    "gram-128-shared polynomial-128-shared update-256": (3, 643, 5415),
}


def spectrum(kind, size, generator, device):
    b, m, n = size
    dev = {"device": device, "generator": generator}
    x = torch.randn(size, **dev)
    if kind == "steep":  # strong directions that fall off, and little else
        r = max(1, min(m, n) // 4)
        x = (torch.randn((b, m, r), **dev) / torch.arange(1, r + 1, device=device)) @ torch.randn((b, r, n), **dev) + 0.1 * x
    elif kind == "falling":  # a gradient: many directions whose strengths fall off slowly, and noise
        r = max(1, min(m, n) // 8)
        x = (torch.randn((b, m, r), **dev) / torch.arange(1, r + 1, device=device).sqrt()) @ torch.randn((b, r, n), **dev) \
            + 0.3 * x
    elif kind == "strong":  # one direction above all others
        x = x + 2 * torch.randn((b, m, 1), **dev) @ torch.randn((b, 1, n), **dev)
    elif kind == "thin":  # two directions only
        x = torch.randn((b, m, 2), **dev) @ torch.randn((b, 2, n), **dev)
    return x


def steps(g, coefficients, scale, eps, dtype):
    """The steps of one matrix in elementary operations of `dtype`."""
    x = g.to(dtype)
    tall = x.shape[0] > x.shape[1]
    if tall:
        x = x.T.contiguous()
    # the norm is a 64-bit sum in both
    x = x / (torch.linalg.matrix_norm(g.double()) + eps).to(dtype)
    for a, b, c in coefficients:
        q = x @ x.T
        x = a * x + (b * q + c * (q @ q)) @ x
    return scale * (x.T if tall else x)


def spacing(v, dtype):
    """A unit in the last place of the 16-bit type at the double values v."""
    bits, low = (7, -133) if dtype == torch.bfloat16 else (10, -24)
    e = torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -200)))
    return torch.exp2((e - bits).clamp(min=low))


def excess(out, want, plain, near):
    """The error of `out` beyond the rounding of its type, as a part of what `near` times the plain form's
    error allows: at most 1 for a result that is near enough.

    fp32: the error's norm. 16 bits: an error d before the rounding changes the rounded value, by a unit
    u in the last place, with probability |d| / u. So the squared distance from the rounded exact
    values is about the sum of |d| u; four standard deviations and four single units on top."""
    if out.dtype == torch.float32:
        limit = near * float((plain.double() - want).norm()) + 2.0 ** -24 * float(want.norm())
        return float((out.double() - want).norm()) / limit
    u = spacing(want, out.dtype)
    got = float(((out.double() - want.to(out.dtype).double()) ** 2).sum())
    d = near * (plain.double() - want).abs()
    limit = float((d * u).sum()) + 4 * float((d * u ** 3).sum()) ** 0.5 + 4 * float(u.max()) ** 2
    return got / limit


# The kernels' arithmetic with exact sums, to show that the limits tell it from less.

HELD = 2.0 ** 13


def planes(v, upper=False):
    """Two fp16 numbers, or the upper one alone."""
    v = v.float() * HELD
    hi = v.half().float()
    lo = torch.zeros_like(hi) if upper else (v - hi).half().float()
    return hi.double() / HELD, lo.double() / HELD


def product(l, r, drop=""):
    """hi hi + hi lo + lo hi; `drop` leaves out the lower plane of "l" or "r"."""
    s = l[0] @ r[0]
    if drop != "r":
        s = s + l[0] @ r[1]
    if drop != "l":
        s = s + l[1] @ r[0]
    return s


def simulated(g, coefficients, dtype, drop=None):
    """The steps in two planes; `drop` = (step, "gram" | "square" | "update", "l" | "r") plants a mistake."""
    x = g.double()
    x = planes(x / torch.linalg.matrix_norm(x))
    t = lambda p: (p[0].T, p[1].T)
    for i, (a, b, c) in enumerate(coefficients):
        lost = {kind: side for step, kind, side in [drop or (-1, "", "")] if step == i}
        q = planes(product(x, t(x), lost.get("gram", "")))
        s = product(q, t(q), lost.get("square", ""))
        p = planes(b * (q[0] + q[1]) + c * s)
        v = a * (x[0] + x[1]) + product(p, x, lost.get("update", ""))
        x = planes(v)
    return v.to(dtype)
