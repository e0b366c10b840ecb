"""GPU: the operators around the AllReduce through the C ABI against plain 64-bit implementations, at
the sizes, strides, types and masks where they can go wrong. Bounds: operator_util."""

import math

import pytest

import operator_util as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TYPES = ["f32", "bf16", "f16"]


def _say(*a):
    print("[operators]", *a, flush=True)


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return {"device": "cuda", "generator": g}


# The ways that [ranks, tokens, width] rows lie in memory. Values between rows are a pattern that no
# kernel may change.
LAYOUTS = ["dense", "padded", "tokens first", "apart"]
PATTERN = 77.0


def _place(values, layout, dtype):
    """`values` in a tensor of that layout, and the whole memory that it lies in."""
    r, t, w = values.shape
    if layout == "dense":
        base = torch.full((r, t, w), PATTERN, dtype=dtype, device="cuda")
        view = base
    elif layout == "padded":  # rows that start at odd elements
        base = torch.full((r, t, w + 3), PATTERN, dtype=dtype, device="cuda")
        view = base[:, :, 1:w + 1]
    elif layout == "tokens first":
        base = torch.full((t, r, w + 1), PATTERN, dtype=dtype, device="cuda")
        view = base.transpose(0, 1)[:, :, :w]
    else:  # ranks with a gap between them
        base = torch.full((r, t * w + 5), PATTERN, dtype=dtype, device="cuda")
        view = base[:, :t * w].unflatten(1, (t, w)) if t else base[:, :0].reshape(r, 0, w)
    view.copy_(values)
    return view, base


def _gaps_kept(view, base):
    view.fill_(PATTERN)
    assert bool((base == PATTERN).all()), "values between the rows were written"


def _norm_case(ranks, tokens, width, dtype, seed, layout="dense"):
    dev = _gen(seed)
    x = torch.randn((ranks, tokens, width), **dev) * torch.exp(torch.randn(width, **dev)) \
        + torch.randn(width, **dev)
    return _place(x, layout, ref.DTYPES[dtype])


NORM_SIZES = [(1, 1, 1), (2, 3, 2), (1, 5, 7), (3, 33, 63), (2, 70, 64), (1, 9, 65), (3, 40, 129),
              (2, 17, 255), (1, 66, 256), (2, 5, 513), (1, 130, 1000), (2, 9, 1025), (1, 21, 2051),
              (3, 3, 4096), (1, 7, 5000), (1, 5, 8192), (1, 3, 9001), (2, 2, 16384), (1, 3, 16385),
              (1, 2, 40001), (300, 1, 40), (1, 700, 24), (2, 0, 16)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", NORM_SIZES, ids=lambda s: "x".join(map(str, s)))
def test_layernorm(size, dtype):
    import paper_2602_17254_amd as T

    ranks, tokens, width = size
    k = sum(size)
    layout, wtype = LAYOUTS[k % 4], [ref.DTYPES["f32"], ref.DTYPES[dtype], torch.bfloat16][k % 3]
    _say("layernorm", size, dtype, layout, wtype)
    dt, eps = ref.DTYPES[dtype], 1e-5
    x, _ = _norm_case(ranks, tokens, width, dtype, k, layout)
    dev = _gen(k + 1)
    gamma = (1 + 0.3 * torch.randn(width, **dev)).to(wtype)
    beta = (0.3 * torch.randn(width, **dev)).to(wtype)
    y, ybase = _place(torch.zeros_like(x), LAYOUTS[(k + 1) % 4], dt)
    mean = torch.full((ranks, tokens), math.nan, device="cuda")
    rstd = torch.full((ranks, tokens), math.nan, device="cuda")
    T.trivance_layernorm_forward(x, gamma, beta, y, mean, rstd, eps)
    torch.cuda.synchronize()
    wants = ref.layernorm_forward(x.double(), gamma.double(), beta.double(), eps)
    (want, bound), (wm, bm), (ws, bs) = wants
    ref.assert_within(y, want, bound + ref.rounding(want, dt) * 1.01, "y")
    ref.assert_within(mean, wm, bm, "mean")
    ref.assert_within(rstd, ws, bs, "rstd")
    _gaps_kept(y, ybase)

    dy, _ = _place(torch.randn(size, **dev), LAYOUTS[(k + 2) % 4], dt)
    dx, dbase = _place(torch.zeros_like(x), LAYOUTS[(k + 3) % 4], dt)
    # each rank's row of a vector to sum: other gradients, dgamma, dbeta, a gap
    rows = torch.full((ranks, 2 * width + 7), PATTERN, device="cuda")
    dgamma, dbeta = rows[:, 5:5 + width], rows[:, 5 + width:5 + 2 * width]
    need = T.trivance_layernorm_workspace_bytes(ranks, tokens, width)
    ws_ = torch.full((need // 4,), math.nan, device="cuda")
    T.trivance_layernorm_backward(dy, x, gamma, mean, rstd, dx, dgamma, dbeta, ws_)
    torch.cuda.synchronize()
    (want, bound), (wg, bg), (wb, bb) = ref.layernorm_backward(
        dy.double(), x.double(), gamma.double(), mean.double(), rstd.double())
    ref.assert_within(dx, want, bound + ref.rounding(want, dt) * 1.01, "dx")
    ref.assert_within(dgamma, wg, bg, "dgamma")
    ref.assert_within(dbeta, wb, bb, "dbeta")
    _gaps_kept(dx, dbase)
    dgamma.fill_(PATTERN)
    dbeta.fill_(PATTERN)
    assert bool((rows == PATTERN).all())


def test_layernorm_without_weights_and_in_place():
    import paper_2602_17254_amd as T

    for width in (48, 3000, 20000):
        x, _ = _norm_case(2, 6, width, "f32", width, "padded")
        eps = 1e-6
        mean, rstd = torch.empty((2, 6), device="cuda"), torch.empty((2, 6), device="cuda")
        y = torch.empty((2, 6, width), device="cuda")
        ones, zeros = torch.ones(width, device="cuda"), torch.zeros(width, device="cuda")
        T.trivance_layernorm_forward(x, ones, zeros, y, mean, rstd, eps)
        for gamma, beta in ((None, None), (ones, None), (None, zeros)):
            z = torch.empty_like(y)
            T.trivance_layernorm_forward(x, gamma, beta, z, None, None, eps)
            assert torch.equal(y, z)
        dy = torch.randn((2, 6, width), **_gen(1))
        ws = torch.empty(T.trivance_layernorm_workspace_bytes(2, 6, width), dtype=torch.uint8, device="cuda")
        dx, dg, db = torch.empty_like(dy), torch.empty((2, width), device="cuda"), torch.empty((2, width), device="cuda")
        T.trivance_layernorm_backward(dy, x, ones, mean, rstd, dx, dg, db, ws)
        for one in (dict(dgamma=None, dbeta=db), dict(dgamma=dg, dbeta=None), dict(dgamma=None, dbeta=None)):
            for g in (dg, db):
                g2 = g.clone()
                kw = {k: (torch.empty_like(v) if v is not None else None) for k, v in one.items()}
                dx2 = torch.empty_like(dx)
                T.trivance_layernorm_backward(dy, x, None, mean, rstd, dx2, kw["dgamma"], kw["dbeta"],
                                              ws if kw["dgamma"] is not None or kw["dbeta"] is not None else None)
                assert torch.equal(dx, dx2) and torch.equal(g, g2)
                assert kw["dgamma"] is None or torch.equal(kw["dgamma"], dg)
                assert kw["dbeta"] is None or torch.equal(kw["dbeta"], db)
        # the same bits where the output takes the input's place
        d1, x1 = dy.clone(), x.clone()
        T.trivance_layernorm_backward(d1, x, ones, mean, rstd, d1, dg, db, ws)
        assert torch.equal(d1, dx)
        T.trivance_layernorm_forward(x1, ones, zeros, x1, None, None, eps)
        assert torch.equal(x1, y)


def test_layernorm_rows_that_are_no_numbers_stay_apart():
    import paper_2602_17254_amd as T

    for width in (40, 700, 5000):
        x, _ = _norm_case(1, 8, width, "bf16", 3)
        x[0, 2, width // 2] = math.nan
        x[0, 5, 0] = math.inf
        x[0, 6] = 4.0  # no spread: h is zero
        y, mean, rstd = torch.empty_like(x), torch.empty((1, 8), device="cuda"), torch.empty((1, 8), device="cuda")
        T.trivance_layernorm_forward(x, None, torch.full((width,), 0.5, device="cuda"), y, mean, rstd)
        torch.cuda.synchronize()
        for t in range(8):
            assert bool(torch.isnan(rstd[0, t])) == (t in (2, 5))
            assert bool(torch.isnan(y[0, t]).all()) == (t in (2, 5))
            assert bool(torch.isfinite(y[0, t]).all()) == (t not in (2, 5))
        assert bool((y[0, 6] == 0.5).all())


def test_layernorm_mean_of_rows_that_nearly_cancel():
    """The sum of a row's values is exact but for 2^-53 a step: the mean is within its rounding to fp32, and
    2^-40 of the values' mean size."""
    import paper_2602_17254_amd as T

    for width in (5, 60, 1024, 4096, 12000, 20000):
        x = torch.randn((1, 5, width), **_gen(width))
        x -= x.mean(2, keepdim=True) * (1 - 1e-3)
        y, mean, rstd = torch.empty_like(x), torch.empty((1, 5), device="cuda"), torch.empty((1, 5), device="cuda")
        T.trivance_layernorm_forward(x, None, None, y, mean, rstd)
        want = x.double().mean(2)
        ref.assert_within(mean, want, ref.U * want.abs() * 1.01 + 2.0 ** -40 * x.double().abs().mean(2), "mean")


def test_layernorm_statistics_of_rows_far_from_zero():
    """Rows whose mean is 1000 times their spread: the variance is taken about the mean."""
    import paper_2602_17254_amd as T

    for width in (64, 1000, 9000, 18000):
        x = torch.randn((1, 4, width), **_gen(width)) + 1000.0
        y = torch.empty_like(x)
        T.trivance_layernorm_forward(x, None, None, y, eps=0.0)
        one = torch.ones(1, dtype=torch.float64, device="cuda")
        (want, bound), _, _ = ref.layernorm_forward(x.double(), one, 0 * one, 0.0)
        ref.assert_within(y, want, bound + ref.rounding(want, x.dtype), "y")


@pytest.mark.parametrize("width", [96, 1536, 6000])
def test_layernorm_gradient_against_differences(width):
    """dx, dgamma and dbeta along random directions against central differences of the forward pass,
    summed in 64 bits."""
    import paper_2602_17254_amd as T

    dev = _gen(width)
    x = torch.randn((2, 5, width), **dev)
    gamma, beta = 1 + 0.2 * torch.randn(width, **dev), torch.randn(width, **dev)
    dy = torch.randn((2, 5, width), **dev)
    mean, rstd = torch.empty((2, 5), device="cuda"), torch.empty((2, 5), device="cuda")
    y = torch.empty_like(x)
    T.trivance_layernorm_forward(x, gamma, beta, y, mean, rstd, 1e-5)
    dx = torch.empty_like(x)
    dg, db = torch.empty((2, width), device="cuda"), torch.empty((2, width), device="cuda")
    ws = torch.empty(T.trivance_layernorm_workspace_bytes(2, 5, width), dtype=torch.uint8, device="cuda")
    T.trivance_layernorm_backward(dy, x, gamma, mean, rstd, dx, dg, db, ws)

    def loss(x, gamma, beta, forward):
        return float((forward(x, gamma, beta) * dy.double()).sum())

    def kernel(x, gamma, beta):
        T.trivance_layernorm_forward(x.float().contiguous(), gamma.float(), beta.float(), y, None, None, 1e-5)
        return y.double()

    def plain(x, gamma, beta):
        return ref.layernorm_forward(x, gamma, beta, 1e-5)[0][0]

    e = 2.0 ** -6
    for name in ("x", "gamma", "beta"):
        args = {"x": x.double(), "gamma": gamma.double(), "beta": beta.double()}
        v = torch.sign(torch.randn(args[name].shape, **dev)).double()  # e v is exact in fp32
        lo, hi = dict(args), dict(args)
        lo[name] = (args[name].float() - e * v.float()).double()
        hi[name] = (args[name].float() + e * v.float()).double()
        got = (loss(**hi, forward=kernel) - loss(**lo, forward=kernel)) / (2 * e)
        ideal = (loss(**hi, forward=plain) - loss(**lo, forward=plain)) / (2 * e)
        along = float({"x": (dx.double() * v).sum(), "gamma": (dg.double().sum(0) * v).sum(),
                       "beta": (db.double().sum(0) * v).sum()}[name])
        # the kernel's own rounding over the step's width
        (_, bound), _, _ = ref.layernorm_forward(x.double(), gamma.double(), beta.double(), 1e-5)
        noise = float(((bound + ref.U * y.double().abs()) * dy.double().abs()).sum()) / e
        exact = torch.autograd.grad((plain(*(t := [a.clone().requires_grad_() for a in args.values()]))
                                     * dy.double()).sum(), t)
        truth = float((exact[list(args).index(name)] * v).sum())
        _say(name, "difference", got, "gradient", along, "noise", noise)
        # the difference's own error is what it is in 64 bits
        assert abs(got - along) <= 1.5 * noise + abs(ideal - truth) + 1e-4 * abs(truth)


BALANCE_SIZES = [(1, 1, 1, 1), (1, 1, 8, 2), (2, 5, 3, 3), (3, 40, 4, 1), (1, 300, 5, 2), (2, 65, 16, 4),
                 (3, 129, 31, 2), (1, 77, 64, 8), (2, 33, 65, 6), (4, 9, 128, 2), (1, 50, 200, 8),
                 (2, 41, 256, 8), (1, 19, 257, 4), (1, 30, 511, 8), (2, 11, 700, 3), (1, 9, 1500, 2),
                 (1, 5, 4096, 8), (200, 3, 6, 2), (1, 5000, 8, 2), (2, 0, 8, 2)]


def _balance_case(size, dtype, seed, masked, layout="dense", wide=True):
    ranks, tokens, experts, k = size
    dev = _gen(seed)
    values = 2 * torch.randn((ranks, tokens, experts), **dev)
    chosen = torch.randint(-1, experts, (ranks, tokens, k), **dev).to(torch.int64 if wide else torch.int32)
    mask = None
    if masked:
        mask = torch.rand((ranks, tokens), **dev) < 0.7
        if ranks > 1:
            mask[ranks // 2] = False
        values[~mask] = math.nan  # what lies there is never used
        chosen.masked_fill_((~mask).unsqueeze(2), 2 ** 31 - 1)
    if experts > 1:  # excluded experts, by infinity and by the lowest value of the type
        values[:, ::3, experts // 2] = -math.inf
        values[:, 1::3, 0] = torch.finfo(ref.DTYPES[dtype]).min
    if tokens > 4:
        values[:, 4] = -math.inf  # a token with no expert left
    if masked:
        values[~mask] = math.nan
    logits, _ = _place(values, layout, ref.DTYPES[dtype])
    return logits, chosen, mask


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("masked", [False, True], ids=["all", "masked"])
@pytest.mark.parametrize("size", BALANCE_SIZES, ids=lambda s: "x".join(map(str, s)))
def test_balance(size, masked, dtype):
    import paper_2602_17254_amd as T

    ranks, tokens, experts, k = size
    seed = sum(size) + masked
    _say("balance", size, dtype, "masked" if masked else "all")
    logits, chosen, mask = _balance_case(size, dtype, seed, masked, LAYOUTS[seed % 4], seed % 2 == 0)
    if masked and seed % 3 == 0:
        mask = mask.to(torch.uint8) * 255
    crows = torch.full((ranks, experts + 5), 123, dtype=torch.int32, device="cuda")
    prows = torch.full((ranks, experts + 3), PATTERN, device="cuda")
    counts, probs = crows[:, 2:experts + 3], prows[:, 1:experts + 1]
    need = T.trivance_balance_workspace_bytes(ranks, tokens, experts)
    ws = torch.full((need // 4,), math.nan, device="cuda")
    T.trivance_balance_counts(logits, chosen, counts, probs, ws, mask)
    torch.cuda.synchronize()
    want, (wp, bp) = ref.balance_counts(logits.double(), chosen, mask)
    assert torch.equal(counts.cpu().long(), want)
    ref.assert_within(probs, wp, bp, "probs")

    loss = torch.full((ranks,), math.nan, device="cuda")
    T.trivance_balance_loss(counts, probs, k, loss, 0.25)
    wl = ref.balance_loss(counts, probs, k, 0.25)
    ref.assert_within(loss, wl, 2 * ref.U * wl.abs() + 1e-45, "loss")

    dt = ref.DTYPES[dtype]
    dloss = torch.randn(ranks, **_gen(seed)) if seed % 2 else None
    # a scale that keeps the gradients of a mean in fp16's range
    scale = 64.0 * max(1, tokens)
    d, dbase = _place(torch.zeros((ranks, tokens, experts), device="cuda"), LAYOUTS[(seed + 1) % 4], dt)
    T.trivance_balance_backward(logits, counts, k, d, mask, scale, dloss)
    torch.cuda.synchronize()
    wd, bd = ref.balance_backward(logits.double(), counts, k, mask, scale, dloss)
    ref.assert_within(d, wd, bd + ref.rounding(wd, dt) * 1.01, "dlogits")
    _gaps_kept(d, dbase)
    counts.fill_(123)
    probs.fill_(PATTERN)
    assert bool((crows == 123).all()) and bool((prows == PATTERN).all())


def test_balance_numbers_that_are_none_show():
    import paper_2602_17254_amd as T

    for experts in (6, 100, 600):
        for bad in (math.nan, math.inf):
            logits = torch.randn((1, 20, experts), **_gen(experts))
            logits[0, 7, 3] = bad
            logits[0, 9] = math.nan
            chosen = torch.zeros((1, 20, 1), dtype=torch.int64, device="cuda")
            counts = torch.empty((1, experts + 1), dtype=torch.int32, device="cuda")
            probs = torch.empty((1, experts), device="cuda")
            ws = torch.empty(T.trivance_balance_workspace_bytes(1, 20, experts), dtype=torch.uint8, device="cuda")
            T.trivance_balance_counts(logits, chosen, counts, probs, ws)
            assert bool(torch.isnan(probs).all()) and counts[0].tolist() == [20] + [0] * (experts - 1) + [20]
            d = torch.empty_like(logits)
            T.trivance_balance_backward(logits, counts, 1, d)
            for t in range(20):
                assert bool(torch.isnan(d[0, t]).all()) == (t in (7, 9))
                assert bool(torch.isfinite(d[0, t]).all()) == (t not in (7, 9))


@pytest.mark.parametrize("experts", [3, 5, 7, 11, 100])
def test_balance_sums_of_equal_probabilities(experts):
    """Equal terms round the same way in a long sum. A lane adds four tokens here: four roundings, two of the
    probability and one of the result; the lanes' sums are joined in 64 bits."""
    import paper_2602_17254_amd as T

    lanes = 1
    while lanes * 4 < experts and lanes < 64:
        lanes *= 2
    tokens = 4 * 256 // lanes
    logits = torch.zeros((1, tokens, experts), device="cuda")
    chosen = torch.zeros((1, tokens, 1), dtype=torch.int32, device="cuda")
    counts = torch.empty((1, experts + 1), dtype=torch.int32, device="cuda")
    probs = torch.empty((1, experts), device="cuda")
    ws = torch.empty(T.trivance_balance_workspace_bytes(1, tokens, experts), dtype=torch.uint8, device="cuda")
    T.trivance_balance_counts(logits, chosen, counts, probs, ws)
    want = torch.full((1, experts), tokens / experts, dtype=torch.float64, device="cuda")
    ref.assert_within(probs, want, 7 * ref.U * want, "probs")


@pytest.mark.parametrize("experts", [5, 64, 300])
def test_balance_probabilities_far_below_the_largest(experts):
    """Logits in steps of 2^-10, whose distance from the maximum fp32 holds exactly and which is 25 or more: the
    sum is 1 but for a rounding or two, and a probability's relative error that of its exponential (4
    units at most), of the sum, of a division and of a product, at any distance."""
    import paper_2602_17254_amd as T

    tokens, near = 400, 16 * ref.U
    logits = torch.randint(-80 * 1024, -25 * 1024, (tokens, 1, experts), **_gen(experts)) / 1024
    logits[:, :, experts // 2] = 0.0
    chosen = torch.zeros((tokens, 1, 1), dtype=torch.int32, device="cuda")
    counts = torch.empty((tokens, experts + 1), dtype=torch.int32, device="cuda")
    probs = torch.empty((tokens, experts), device="cuda")
    T.trivance_balance_counts(logits, chosen, counts, probs)
    want = torch.softmax(logits.double(), 2)[:, 0]
    ref.assert_within(probs, want, near * want, "probs")
    d = torch.empty_like(logits)
    T.trivance_balance_backward(logits, counts, 1, d, scale=1e6)
    w = 1e6 * experts * counts[:, None, :experts].double() / counts[:, None, experts:].double() ** 2
    p = want[:, None]
    mean = (p * w).sum(2, keepdim=True)
    ref.assert_within(d, p * (w - mean), 2 * near * p * (w + mean) + 1e-45, "dlogits")


@pytest.mark.parametrize("experts", [8, 72, 300])
def test_balance_gradient_of_the_sum_over_ranks_against_differences(experts):
    """Counts and sums through the framework's AllReduce; every rank's gradient is that of the loss over
    all ranks' tokens, by autograd in 64 bits and by differences of the kernels' own loss."""
    import paper_2602_17254_amd as T

    ranks, tokens, k = 9, 14, 2
    plan = T.trivance_plan((9,), "L")
    dev = _gen(experts)
    x = torch.randn((ranks, tokens, experts), **dev)
    chosen = torch.topk(x, k, dim=2).indices
    mask = torch.rand((ranks, tokens), **dev) < 0.8
    mask[4] = False
    ws = torch.empty(T.trivance_balance_workspace_bytes(ranks, tokens, experts), dtype=torch.uint8, device="cuda")

    def loss(logits):
        counts = torch.empty((ranks, experts + 1), dtype=torch.int32, device="cuda")
        probs = torch.empty((ranks, experts), device="cuda")
        out = torch.empty(ranks, device="cuda")
        T.trivance_balance_counts(logits, chosen, counts, probs, ws, mask)
        T.trivance_allreduce_emulated(counts, plan)
        T.trivance_allreduce_emulated(probs, plan)
        T.trivance_balance_loss(counts, probs, k, out)
        return out, counts

    value, counts = loss(x)
    d = torch.empty_like(x)
    T.trivance_balance_backward(x, counts, k, d, mask)

    t = x.double().requires_grad_()
    p = torch.softmax(t[mask], 1)
    f = torch.bincount(chosen[mask].flatten(), minlength=experts).double()
    n = int(mask.sum())
    truth = experts * (f / (k * n) * p.sum(0) / n).sum()
    truth.backward()
    assert counts[0, :experts].tolist() == f.long().tolist() and counts[0, experts] == n
    # nine ranks' sums and the loss's sum: some tens of roundings of positive terms
    assert bool(((value.double() - truth.item()).abs() <= 120 * ref.U * truth.item()).all())
    _, bound = ref.balance_backward(x.double(), counts, k, mask, 1.0, None)
    ref.assert_within(d, t.grad, bound + ref.rounding(t.grad, torch.float32), "dlogits")

    v = torch.sign(torch.randn(x.shape, **dev))
    e = 2.0 ** -5

    def plain(z):
        q = torch.softmax(z.double()[mask], 1)
        return float(experts * (f / (k * n) * q.sum(0) / n).sum())

    got = float(loss(x + e * v)[0].double().mean() - loss(x - e * v)[0].double().mean()) / (2 * e)
    ideal = (plain(x + e * v) - plain(x - e * v)) / (2 * e)
    along = float((d.double() * v.double()).sum())
    noise = 120 * ref.U * truth.item() / e + 2 * ref.U * float(d.double().abs().sum()) * experts
    _say("difference", got, "gradient", along)
    assert abs(got - along) <= noise + abs(ideal - float((t.grad * v.double()).sum()))


ORTHO_SIZES = [(1, 1, 1), (1, 1, 40), (2, 7, 3), (1, 16, 16), (3, 33, 65), (1, 64, 256), (2, 100, 64),
               (1, 257, 130), (1, 128, 515), (2, 300, 300), (1, 20, 2000), (1, 640, 200), (1, 515, 1030),
              (2, 64, 515), (3, 700, 33), (1, 64, 8192), (1, 50, 9000), (2, 1100, 520), (1, 520, 2600),
              (1, 1280, 1280), (1, 600, 5000)]
QUINTIC = [(3.4445, -4.7750, 2.0315)] * 5


def _spectrum(kind, size, seed):
    b, m, n = size
    dev = _gen(seed)
    x = torch.randn(size, **dev)
    if kind == "steep":  # strong directions that fall off, and little else
        r = max(1, min(m, n) // 4)
        x = (torch.randn((b, m, r), **dev) / torch.arange(1, r + 1, device="cuda")) @ torch.randn((b, r, n), **dev) + 0.1 * x
    elif kind == "thin":  # two directions only
        x = torch.randn((b, m, 2), **dev) @ torch.randn((b, 2, n), **dev)
    return x


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["even", "steep", "thin"])
@pytest.mark.parametrize("size", ORTHO_SIZES, ids=lambda s: "x".join(map(str, s)))
def test_orthogonalize(size, kind, dtype):
    import paper_2602_17254_amd as T

    seed = sum(size)
    dt = ref.DTYPES[dtype]
    _say("orthogonalize", size, kind, dtype)
    size_of = {0: 1.0, 1: 1e-3, 2: 30.0}[seed % 3]
    x, _ = _place(_spectrum(kind, size, seed) * size_of, LAYOUTS[seed % 4], dt)
    out, base = _place(torch.zeros(size, device="cuda"), LAYOUTS[(seed + 1) % 4], dt)
    ws = torch.full((T.trivance_orthogonalize_workspace_bytes(*size),), 255, dtype=torch.uint8, device="cuda")
    scale = [1.0, 0.2 * math.sqrt(max(size[1:]))][seed % 2]
    T.trivance_orthogonalize(x, out, ws, QUINTIC, scale, 1e-7)
    torch.cuda.synchronize()
    want, bounds = ref.orthogonalize(x.double(), QUINTIC, scale, 1e-7)
    for b in range(size[0]):
        err = float((out[b].double() - want[b]).norm())
        limit = bounds[b] + float(ref.rounding(want[b], dt).norm())
        _say("  error", err, "bound", limit, "norm", float(want[b].norm()))
        assert err <= limit
    _gaps_kept(out, base)


def test_orthogonalize_steps_in_place_and_zero():
    import paper_2602_17254_amd as T

    size = (3, 90, 70)
    x = torch.randn(size, **_gen(5))
    x[1] = 0.0
    ws = torch.empty(T.trivance_orthogonalize_workspace_bytes(*size), dtype=torch.uint8, device="cuda")
    for steps in (QUINTIC[:1], QUINTIC[:2], tuple(QUINTIC), [(1.5, -0.5, 0.0)] * 12,
                  [(4.0, -8.0, 4.5)] + QUINTIC[:3]):
        out = torch.empty_like(x)
        T.trivance_orthogonalize(x, out, ws, steps)
        again = x.clone()
        T.trivance_orthogonalize(again, again, ws, steps)
        assert torch.equal(out, again)
        assert bool((out[1] == 0).all())
        want, bounds = ref.orthogonalize(x.double()[[0, 2]], steps, 1.0, 1e-7)
        for i, b in ((0, 0), (1, 2)):
            err = float((out[b].double() - want[i]).norm())
            assert err <= bounds[i] + float(ref.rounding(want[i], x.dtype).norm())


def test_orthogonalize_extreme_sizes_of_entries():
    """Norms near the ends of fp32, which squares in fp32 would not hold."""
    import paper_2602_17254_amd as T

    x = torch.randn((1, 48, 80), **_gen(9))
    ws = torch.empty(T.trivance_orthogonalize_workspace_bytes(1, 48, 80), dtype=torch.uint8, device="cuda")
    want, bounds = ref.orthogonalize(x.double(), QUINTIC, 1.0, 0.0)
    for factor in (2.0 ** 120, 2.0 ** -100):
        out = torch.empty_like(x)
        T.trivance_orthogonalize(x * factor, out, ws, QUINTIC, 1.0, 0.0)
        assert float((out.double() - want).norm()) <= bounds[0] + float(ref.rounding(want, x.dtype).norm())


def test_orthogonalize_numbers_that_are_none_stay_in_their_matrix():
    import paper_2602_17254_amd as T

    for bad in (math.nan, math.inf):
        x = torch.randn((3, 70, 90), **_gen(6))
        clean = torch.empty_like(x)
        ws = torch.empty(T.trivance_orthogonalize_workspace_bytes(3, 70, 90), dtype=torch.uint8, device="cuda")
        T.trivance_orthogonalize(x, clean, ws)
        x[1, 3, 4] = bad
        out = torch.empty_like(x)
        T.trivance_orthogonalize(x, out, ws)
        assert torch.equal(out[0], clean[0]) and torch.equal(out[2], clean[2])
        assert bool(torch.isnan(out[1]).all())


def test_operators_repeat_on_streams_and_in_graphs():
    """The same bits on another stream and from the replays of a captured graph."""
    import paper_2602_17254_amd as T

    dev = _gen(11)
    x = torch.randn((4, 200, 300), **dev).bfloat16()
    dy = torch.randn((4, 200, 300), **dev).bfloat16()
    gamma, beta = torch.randn(300, **dev), torch.randn(300, **dev)
    logits = torch.randn((4, 600, 48), **dev)
    chosen = torch.topk(logits, 2, dim=2).indices.to(torch.int32)
    g = torch.randn((1, 130, 300), **dev)

    def buffers():
        return {"y": torch.zeros_like(x), "mean": torch.zeros((4, 200), device="cuda"),
                "rstd": torch.zeros((4, 200), device="cuda"), "dx": torch.zeros_like(x),
                "rows": torch.zeros((4, 600), device="cuda"),
                "counts": torch.zeros((4, 49), dtype=torch.int32, device="cuda"),
                "probs": torch.zeros((4, 48), device="cuda"), "loss": torch.zeros(4, device="cuda"),
                "dlogits": torch.zeros_like(logits), "out": torch.zeros_like(g)}

    w1 = torch.empty(T.trivance_layernorm_workspace_bytes(4, 200, 300), dtype=torch.uint8, device="cuda")
    w2 = torch.empty(T.trivance_balance_workspace_bytes(4, 600, 48), dtype=torch.uint8, device="cuda")
    w3 = torch.empty(T.trivance_orthogonalize_workspace_bytes(1, 130, 300), dtype=torch.uint8, device="cuda")

    def run(b, stream=None):
        T.trivance_layernorm_forward(x, gamma, beta, b["y"], b["mean"], b["rstd"], stream=stream)
        T.trivance_layernorm_backward(dy, x, gamma, b["mean"], b["rstd"], b["dx"], b["rows"][:, :300],
                                      b["rows"][:, 300:], w1, stream)
        T.trivance_balance_counts(logits, chosen, b["counts"], b["probs"], w2, None, stream)
        T.trivance_balance_loss(b["counts"], b["probs"], 2, b["loss"], 1.0, stream)
        T.trivance_balance_backward(logits, b["counts"], 2, b["dlogits"], stream=stream)
        T.trivance_orthogonalize(g, b["out"], w3, stream=stream)

    want, other, replayed = buffers(), buffers(), buffers()
    run(want)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    run(other, stream)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(replayed)
    for turn in range(3):
        for t in replayed.values():
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for name in want:
            assert torch.equal(want[name], other[name]), name
            assert torch.equal(want[name], replayed[name]), (name, turn)
        # the program's own work between replays
        float((x.float() ** 2).sum())


def test_offsets_beyond_32_bits():
    """Rows, ranks and matrices further than 2^31 elements apart."""
    import paper_2602_17254_amd as T

    far = 2 ** 31 + 72
    base = torch.zeros(far + 70000, dtype=torch.bfloat16, device="cuda")
    out = torch.zeros_like(base)
    dev = _gen(2)
    for shape, strides in (((1, 2, 300), (0, far, 1)), ((2, 1, 300), (far, 300, 1)), ((2, 3, 77), (far, 80, 1))):
        x, y = base.as_strided(shape, strides), out.as_strided(shape, strides)
        x.copy_(torch.randn(shape, **dev))
        near = x.contiguous()
        want, mean, rstd = torch.empty_like(near), torch.empty(shape[:2], device="cuda"), torch.empty(shape[:2], device="cuda")
        T.trivance_layernorm_forward(near, None, None, want, mean, rstd)
        T.trivance_layernorm_forward(x, None, None, y)
        assert torch.equal(y, want)
        width = shape[2]
        ws = torch.empty(T.trivance_layernorm_workspace_bytes(*shape), dtype=torch.uint8, device="cuda")
        dg = [torch.empty((shape[0], width), device="cuda") for _ in range(4)]
        T.trivance_layernorm_backward(near, near, None, mean, rstd, want, dg[0], dg[1], ws)
        T.trivance_layernorm_backward(x, x, None, mean, rstd, y, dg[2], dg[3], ws)
        assert torch.equal(y, want) and torch.equal(dg[0], dg[2]) and torch.equal(dg[1], dg[3])

        chosen = torch.zeros((shape[0], shape[1], 1), dtype=torch.int32, device="cuda")
        ws = torch.empty(T.trivance_balance_workspace_bytes(*shape), dtype=torch.uint8, device="cuda")
        got = []
        for logits, d in ((near, want), (x, y)):
            counts = torch.empty((shape[0], width + 1), dtype=torch.int32, device="cuda")
            probs = torch.empty((shape[0], width), device="cuda")
            T.trivance_balance_counts(logits, chosen, counts, probs, ws)
            T.trivance_balance_backward(logits, counts, 1, d)
            got.append((counts, probs))
        assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1]) and torch.equal(y, want)
    for shape, strides in (((2, 70, 90), (far, 96, 1)), ((2, 300, 130), (far, 130, 1)), ((2, 40, 600), (far, 600, 1))):
        x, y = base.as_strided(shape, strides), out.as_strided(shape, strides)
        x.copy_(torch.randn(shape, **dev))
        near = x.contiguous()
        want = torch.empty_like(near)
        ws = torch.empty(T.trivance_orthogonalize_workspace_bytes(*shape), dtype=torch.uint8, device="cuda")
        T.trivance_orthogonalize(near, want, ws)
        T.trivance_orthogonalize(x, y, ws)
        assert torch.equal(y, want)


def _large(shape, seed):
    """bf16 values drawn one rank at a time."""
    t = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    dev = _gen(seed)
    for part in t:
        part.copy_(torch.randn(part.shape, **dev))
    return t


def test_layernorm_of_more_than_2_31_values():
    import paper_2602_17254_amd as T

    ranks, tokens, width = 8, 65537, 4100
    x, dy = _large((ranks, tokens, width), 1), _large((ranks, tokens, width), 2)
    assert x.numel() > 2 ** 31
    gamma = 1 + 0.3 * torch.randn(width, **_gen(3))
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = torch.empty((ranks, tokens), device="cuda"), torch.empty((ranks, tokens), device="cuda")
    sums = torch.full((2, ranks, width), math.nan, device="cuda")
    ws = torch.empty(T.trivance_layernorm_workspace_bytes(ranks, tokens, width), dtype=torch.uint8, device="cuda")
    T.trivance_layernorm_forward(x, gamma, None, y, mean, rstd)
    T.trivance_layernorm_backward(dy, x, gamma, mean, rstd, dx, sums[0], sums[1], ws)
    for r in (0, ranks - 1):
        for part in (slice(0, 50), slice(tokens - 50, tokens)):
            x1, dy1 = x[r:r + 1, part].contiguous(), dy[r:r + 1, part].contiguous()
            y1, dx1 = torch.empty_like(x1), torch.empty_like(x1)
            m1, r1 = torch.empty((1, 50), device="cuda"), torch.empty((1, 50), device="cuda")
            T.trivance_layernorm_forward(x1, gamma, None, y1, m1, r1)
            T.trivance_layernorm_backward(dy1, x1, gamma, m1, r1, dx1, None, None)
            assert torch.equal(y[r:r + 1, part], y1) and torch.equal(mean[r:r + 1, part], m1)
            assert torch.equal(dx[r:r + 1, part], dx1) and torch.equal(rstd[r:r + 1, part], r1)
        d, h = dy[r].double(), (x[r].double() - mean[r, :, None].double()) * rstd[r, :, None].double()
        n = (tokens + 40) * ref.U
        ref.assert_within(sums[1, r], d.sum(0), n * d.abs().sum(0), "dbeta")
        d *= h
        ref.assert_within(sums[0, r], d.sum(0), n * d.abs().sum(0), "dgamma")


def test_balance_of_more_than_2_31_values():
    import paper_2602_17254_amd as T

    ranks, tokens, experts, k = 8, 1048577, 257, 2
    logits = _large((ranks, tokens, experts), 4)
    assert logits.numel() > 2 ** 31
    chosen = torch.randint(-1, experts, (ranks, tokens, k), **_gen(5))
    counts = torch.empty((ranks, experts + 1), dtype=torch.int32, device="cuda")
    probs = torch.full((ranks, experts), math.nan, device="cuda")
    ws = torch.empty(T.trivance_balance_workspace_bytes(ranks, tokens, experts), dtype=torch.uint8, device="cuda")
    T.trivance_balance_counts(logits, chosen, counts, probs, ws)
    d = torch.empty_like(logits)
    T.trivance_balance_backward(logits, counts, k, d, scale=1e6)
    for r in (0, ranks - 1):
        want, (wp, bp) = ref.balance_counts(logits[r:r + 1].double(), chosen[r:r + 1], None)
        assert torch.equal(counts[r:r + 1].cpu().long(), want)
        ref.assert_within(probs[r:r + 1], wp, bp, "probs")
        near = logits[r:r + 1, -300:].contiguous()
        d1 = torch.empty_like(near)
        T.trivance_balance_backward(near, counts[r:r + 1], k, d1, scale=1e6)
        assert torch.equal(d[r:r + 1, -300:], d1)


@pytest.mark.parametrize("tokens,width", [(1, 1030), (3, 1030), (1, 2500), (1, 16400)])
def test_layernorm_of_more_ranks_than_a_grid_has_rows(tokens, width):
    """Workgroups that go on to another rank: the rows, and the gradients of every rank, have the bits that they
    have in calls of fewer ranks."""
    import paper_2602_17254_amd as T

    ranks, dev = 65535 + 70, _gen(width + tokens)
    # the rows of the workgroups' first and second ranks, and some between
    some = list(range(70)) + [30000] + list(range(65535, ranks))
    x = torch.empty((ranks, tokens, width), dtype=torch.bfloat16, device="cuda")
    dy = torch.empty_like(x)
    for t in (x, dy):
        for part in t.split(8192):
            part.copy_(torch.randn(part.shape, **dev))
    dx = torch.empty_like(x)
    gamma = 1 + 0.3 * torch.randn(width, **dev)
    y = torch.empty_like(x)
    mean, rstd = torch.empty((ranks, tokens), device="cuda"), torch.empty((ranks, tokens), device="cuda")
    T.trivance_layernorm_forward(x, gamma, None, y, mean, rstd)
    sums = torch.full((2, ranks, width), math.nan, device="cuda")
    ws = torch.empty(T.trivance_layernorm_workspace_bytes(ranks, tokens, width), dtype=torch.uint8, device="cuda")
    T.trivance_layernorm_backward(dy, x, gamma, mean, rstd, dx, sums[0], sums[1], ws)
    x1, dy1, n = x[some].contiguous(), dy[some].contiguous(), len(some)
    y1, dx1 = torch.empty_like(x1), torch.empty_like(x1)
    m1, r1 = torch.empty((n, tokens), device="cuda"), torch.empty((n, tokens), device="cuda")
    s1 = torch.full((2, n, width), math.nan, device="cuda")
    T.trivance_layernorm_forward(x1, gamma, None, y1, m1, r1)
    T.trivance_layernorm_backward(dy1, x1, gamma, m1, r1, dx1, s1[0], s1[1], ws)
    assert torch.equal(mean[some], m1) and torch.equal(rstd[some], r1) and torch.equal(y[some], y1)
    assert torch.equal(dx[some], dx1) and torch.equal(sums[:, some], s1)


@pytest.mark.parametrize("dtype", TYPES)
def test_tensors_beyond_the_caches(dtype):
    """Large tensors take other loads and stores: every row has the bits that it has in a call of its rank alone,
    which is small."""
    import paper_2602_17254_amd as T

    dt, dev = ref.DTYPES[dtype], _gen(8)
    size = torch.finfo(dt).bits // 8
    tokens, width = 701, 12007 // size
    x, _ = _place(torch.randn((6, tokens, width), **dev), "padded", dt)
    dy, _ = _place(torch.randn((6, tokens, width), **dev), "padded", dt)
    assert x.numel() * size > 2 ** 25 > x[:1].numel() * size
    gamma = 1 + 0.3 * torch.randn(width, **dev)

    def norm(x, dy):
        y, y_base = _place(torch.zeros_like(x), "padded", dt)
        dx, dx_base = _place(torch.zeros_like(x), "padded", dt)
        mean, rstd = (torch.full(x.shape[:2], math.nan, device="cuda") for _ in range(2))
        sums = torch.full((2, x.shape[0], width), math.nan, device="cuda")
        ws = torch.full((T.trivance_layernorm_workspace_bytes(*x.shape) // 4,), math.nan, device="cuda")
        T.trivance_layernorm_forward(x, gamma, None, y, mean, rstd)
        T.trivance_layernorm_backward(dy, x, gamma, mean, rstd, dx, sums[0], sums[1], ws)
        out = y.clone(), mean, rstd, dx.clone(), sums
        _gaps_kept(y, y_base)
        _gaps_kept(dx, dx_base)
        return out

    y, mean, rstd, dx, sums = norm(x, dy)
    for r in range(6):
        one = norm(x[r:r + 1], dy[r:r + 1])
        for got, want in zip((y, mean, rstd, dx), one):
            assert torch.equal(got[r:r + 1], want)
        _, (dgamma, bg), (dbeta, bb) = ref.layernorm_backward(
            dy[r:r + 1].double(), x[r:r + 1].double(), gamma.double(), mean[r:r + 1].double(), rstd[r:r + 1].double())
        ref.assert_within(sums[0][r:r + 1], dgamma, bg, "dgamma")
        ref.assert_within(sums[1][r:r + 1], dbeta, bb, "dbeta")

    experts = 251
    logits, _ = _place(2 * torch.randn((5, 40000 // size, experts), **dev), "padded", dt)
    assert logits.numel() * size > 2 ** 25 > logits[:1].numel() * size
    mask = torch.rand(logits.shape[:2], **dev) < 0.7
    counts = torch.randint(0, 300, (5, experts + 1), **dev).to(torch.int32)
    d, d_base = _place(torch.zeros_like(logits), "padded", dt)
    T.trivance_balance_backward(logits, counts, 2, d, mask)
    got = d.clone()
    _gaps_kept(d, d_base)
    for r in range(5):
        want, _ = _place(torch.zeros_like(logits[r:r + 1]), "padded", dt)
        T.trivance_balance_backward(logits[r:r + 1], counts[r:r + 1], 2, want, mask[r:r + 1])
        assert torch.equal(got[r:r + 1], want)
