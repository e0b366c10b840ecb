"""GPU: the RMS norm, the experts' calls, the embedding and dropout through the C ABI against plain 64-bit
implementations, at the sizes, strides, types and masks where they can go wrong. Bounds: more_operator_util."""

import math

import pytest

import more_operator_util as more
import operator_util as ref
from test_gpu_operators import LAYOUTS, NORM_SIZES, PATTERN, TYPES, _gaps_kept, _gen, _place

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _say(*a):
    print("[more operators]", *a, flush=True)


def _id(size):
    return "x".join(map(str, size))


def _bytes(n):
    """A workspace whose contents are no numbers."""
    return torch.full((n,), 255, dtype=torch.uint8, device="cuda")


# RMS norm.


def _norm(size, dtype, seed, residual, out8, layout):
    """Inputs and outputs of a forward call, all in layouts of their own."""
    ranks, tokens, width = size
    dt, dev = ref.DTYPES[dtype], _gen(seed)
    spread = torch.exp(torch.randn(width, **dev))
    s = {"x": _place(torch.randn(size, **dev) * spread, LAYOUTS[layout % 4], dt)[0], "residual": None}
    if residual:
        s["residual"] = _place(torch.randn(size, **dev) * spread, LAYOUTS[(layout + 1) % 4], dt)[0]
    s["gamma"] = (1 + 0.3 * torch.randn(width, **dev)).to([ref.DTYPES["f32"], dt, torch.bfloat16][layout % 3])
    zero = torch.zeros(size, device="cuda")
    s["total"], s["total_base"] = _place(zero, LAYOUTS[(layout + 2) % 4], dt)
    s["rstd"] = torch.full((ranks, tokens), math.nan, device="cuda")
    s["scales"] = torch.full((ranks, tokens), math.nan, device="cuda") if out8 else None
    if out8:  # a pattern that 8 bits hold
        s["y"], s["y_base"] = _place(zero, LAYOUTS[(layout + 3) % 4], torch.uint8)
        s["y"] = s["y"].view(torch.float8_e4m3fn)
    else:
        s["y"], s["y_base"] = _place(zero, LAYOUTS[(layout + 3) % 4], dt)
    return s


@pytest.mark.parametrize("out8", [False, True], ids=["same", "eight"])
@pytest.mark.parametrize("residual", [False, True], ids=["alone", "residual"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", NORM_SIZES, ids=_id)
def test_rmsnorm(size, dtype, residual, out8):
    import paper_2602_17254_amd as T

    ranks, tokens, width = size
    k, dt, eps = sum(size) + residual, ref.DTYPES[dtype], 1e-5
    _say("rmsnorm", size, dtype, residual, out8)
    s = _norm(size, dtype, k, residual, out8, k)
    T.trivance_rmsnorm_forward(s["x"], s["gamma"], s["y"], s["rstd"], s["residual"], s["total"], s["scales"], eps)
    torch.cuda.synchronize()
    total = s["x"].double() + (s["residual"].double() if residual else 0.0)
    ref.assert_within(s["total"], total, ref.U * total.abs() + ref.rounding(total, dt) * 1.01, "total")
    (y, by), (rstd, bs) = more.rmsnorm_forward(total, s["gamma"].double(), eps)
    ref.assert_within(s["rstd"], rstd, bs, "rstd")
    if out8:
        (q, bq), (scales, bc) = more.eight_bits(y)
        ref.assert_within(s["scales"], scales, bc, "scales")
        ref.assert_within(s["y"].float(), q, bq, "y")
        s["y"] = s["y"].view(torch.uint8)
    else:
        ref.assert_within(s["y"], y, by + ref.rounding(y, dt) * 1.01, "y")
    _gaps_kept(s["y"], s["y_base"])
    if out8:
        _gaps_kept(s["total"], s["total_base"])
        return

    dev = _gen(k + 1)
    dy, _ = _place(torch.randn(size, **dev), LAYOUTS[(k + 1) % 4], dt)
    dtotal = _place(torch.randn(size, **dev), LAYOUTS[k % 4], dt)[0] if residual else None
    dx, dbase = _place(torch.zeros(size, device="cuda"), LAYOUTS[(k + 3) % 4], dt)
    # each rank's row of a vector to sum: other gradients, dgamma, a gap
    rows = torch.full((ranks, width + 12), PATTERN, device="cuda")
    dgamma = rows[:, 5:5 + width]
    ws = torch.full((T.trivance_rmsnorm_workspace_bytes(*size) // 4,), math.nan, device="cuda")
    T.trivance_rmsnorm_backward(dy, s["total"], s["gamma"], s["rstd"], dx, dgamma, ws, dtotal)
    torch.cuda.synchronize()
    (want, bound), (wg, bg) = more.rmsnorm_backward(dy.double(), s["total"].double(), s["gamma"].double(), s["rstd"].double(),
                                                    None if dtotal is None else dtotal.double())
    ref.assert_within(dx, want, bound + ref.rounding(want, dt) * 1.01, "dx")
    ref.assert_within(dgamma, wg, bg, "dgamma")
    _gaps_kept(dx, dbase)
    _gaps_kept(s["total"], s["total_base"])
    dgamma.fill_(PATTERN)
    assert bool((rows == PATTERN).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", [5, 48, 771, 3000, 20001])
def test_rmsnorm_in_place_and_without_weights(width, dtype):
    """The same bits where outputs take inputs' places, where gamma is ones or none, and without the outputs
    that may be left out."""
    import paper_2602_17254_amd as T

    size, dt, dev = (2, 6, width), ref.DTYPES[dtype], _gen(width)
    x, r = (_place(torch.randn(size, **dev), "padded", dt)[0] for _ in range(2))
    ones = torch.ones(width, device="cuda")
    y, total, rstd = torch.empty(size, dtype=dt, device="cuda"), torch.empty(size, dtype=dt, device="cuda"), torch.empty((2, 6), device="cuda")
    T.trivance_rmsnorm_forward(x, ones, y, rstd, r, total)

    def copies():
        return x.clone(memory_format=torch.contiguous_format), r.clone(memory_format=torch.contiguous_format)

    z = torch.empty_like(y)
    T.trivance_rmsnorm_forward(x, None, z, residual=r)
    assert torch.equal(z, y)
    for total_at, y_at in ((0, 1), (1, 0), (0, None), (1, None), (None, 0), (None, 1)):
        ins = copies()
        got_total = torch.empty_like(y) if total_at is None else ins[total_at]
        got_y = torch.empty_like(y) if y_at is None else ins[y_at]
        T.trivance_rmsnorm_forward(ins[0], None, got_y, None, ins[1], got_total)
        assert torch.equal(got_y, y) and torch.equal(got_total, total), (total_at, y_at)
    # the total of an earlier call is the next one's residual, or stands alone
    alone, rstd1 = torch.empty_like(y), torch.empty_like(rstd)
    T.trivance_rmsnorm_forward(total, None, alone, rstd1)
    own = total.clone()
    T.trivance_rmsnorm_forward(own, None, own, None)
    assert torch.equal(own, alone)
    q, scales = torch.empty(size, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty((2, 6), device="cuda")
    T.trivance_rmsnorm_forward(x, None, q, None, r, total, scales)
    ins = copies()
    q1, scales1 = torch.empty_like(q), torch.empty_like(scales)
    T.trivance_rmsnorm_forward(ins[0], ones, q1, None, ins[1], ins[1], scales1)
    assert torch.equal(q1.view(torch.uint8), q.view(torch.uint8)) and torch.equal(scales1, scales) and torch.equal(ins[1], total)

    dy, dtotal = torch.randn(size, **dev).to(dt), torch.randn(size, **dev).to(dt)
    ws = _bytes(T.trivance_rmsnorm_workspace_bytes(*size))
    dx, dg = torch.empty_like(y), torch.empty((2, width), device="cuda")
    T.trivance_rmsnorm_backward(dy, total, ones, rstd, dx, dg, ws, dtotal)
    for at in range(3):
        ins = [dy.clone(), total.clone(), dtotal.clone()]
        dg1 = torch.empty_like(dg)
        T.trivance_rmsnorm_backward(ins[0], ins[1], None, rstd, ins[at], dg1, ws, ins[2])
        assert torch.equal(ins[at], dx) and torch.equal(dg1, dg)
    dx1 = torch.empty_like(dx)
    T.trivance_rmsnorm_backward(dy, total, None, rstd, dx1, None, None, dtotal)
    assert torch.equal(dx1, dx)
    T.trivance_rmsnorm_backward(dy, total, None, rstd, dx1, dg, ws)
    T.trivance_rmsnorm_backward(dy, total, None, rstd, dx, dg, ws, torch.zeros_like(dy))
    assert torch.equal(dx1, dx)


def test_rmsnorm_rows_that_are_no_numbers_stay_apart():
    import paper_2602_17254_amd as T

    for width in (40, 700, 5000, 20000):
        x = torch.randn((1, 8, width), **_gen(3)).bfloat16()
        x[0, 2, width // 2] = math.nan
        x[0, 5, 0] = -math.inf
        x[0, 6] = 0.0
        y, rstd, scales = torch.empty_like(x), torch.empty((1, 8), device="cuda"), torch.empty((1, 8), device="cuda")
        q = torch.empty(x.shape, dtype=torch.float8_e4m3fn, device="cuda")
        T.trivance_rmsnorm_forward(x, None, y, rstd)
        T.trivance_rmsnorm_forward(x, None, q, rstd, scales=scales)
        torch.cuda.synchronize()
        assert bool(torch.isnan(y[0, 2]).all()) and bool((y[0, 6] == 0).all())
        assert bool(torch.isnan(y[0, 5, 0])) and bool((y[0, 5, 1:] == 0).all())
        assert scales[0, 6] == 2.0 ** -126 and bool((q[0, 6].float() == 0).all())
        for t in range(8):
            bad = t in (2, 5)
            assert bool(torch.isnan(q[0, t].float()).all()) == bad and bool(torch.isnan(scales[0, t])) == bad
            assert bool(torch.isfinite(y[0, t]).all()) != bad and bool(torch.isfinite(q[0, t].float()).all()) != bad


@pytest.mark.parametrize("dtype", TYPES)
def test_rmsnorm_eight_bits_reach_the_largest_number(dtype):
    """A row's largest value becomes 448 exactly, whatever rounds on the way, and powers of two of it are exact."""
    import paper_2602_17254_amd as T

    for width in (7, 100, 1000, 9000, 18000):
        x = torch.randn((1, 50, width), **_gen(width)).to(ref.DTYPES[dtype])
        x[0, :, -1] = -8.0 * (1 + torch.arange(50, device="cuda") / 64).to(x.dtype)
        x[0, :, 0] = -x[0, :, -1] / 4
        q, scales = torch.empty(x.shape, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty((1, 50), device="cuda")
        T.trivance_rmsnorm_forward(x, None, q, scales=scales)
        assert bool((q[0, :, -1].float() == -448).all()) and bool((q[0, :, 0].float() == 112).all())


@pytest.mark.parametrize("width", [96, 1536, 6000])
def test_rmsnorm_gradient_against_differences(width):
    """dx, dgamma and the residual's way along random directions against central differences of the forward pass,
    summed in 64 bits: L = sum(c y) + sum(d total)."""
    import paper_2602_17254_amd as T

    size, dev = (2, 5, width), _gen(width)
    x, r, c, d = (torch.randn(size, **dev) for _ in range(4))
    gamma = 1 + 0.3 * torch.randn(width, **dev)
    eps = 1e-5

    def forward(x, r, gamma):
        y, total, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(size[:2], device="cuda")
        T.trivance_rmsnorm_forward(x, gamma, y, rstd, r, total, None, eps)
        return float((y.double() * c.double()).sum() + (total.double() * d.double()).sum()), total, rstd

    def plain(x, r, gamma):
        t = x.double() + r.double()
        y = t / torch.sqrt((t * t).mean(-1, keepdim=True) + eps) * gamma.double()
        return float((y * c.double()).sum() + (t * d.double()).sum())

    _, total, rstd = forward(x, r, gamma)
    dx, dg = torch.empty_like(x), torch.empty((2, width), device="cuda")
    ws = _bytes(T.trivance_rmsnorm_workspace_bytes(*size))
    T.trivance_rmsnorm_backward(c, total, gamma, rstd, dx, dg, ws, d)
    h = 2.0 ** -6
    for which in range(3):
        v = torch.sign(torch.randn(gamma.shape if which == 2 else size, **dev))
        plus, minus = [[x, r, gamma] for _ in range(2)]
        plus, minus = list(plus), list(minus)
        plus[which], minus[which] = plus[which] + h * v, minus[which] - h * v
        got = (forward(*plus)[0] - forward(*minus)[0]) / (2 * h)
        ideal = (plain(*plus) - plain(*minus)) / (2 * h)
        along = float(((dg.sum(0) if which == 2 else dx).double() * v.double()).sum())
        # the gradient in 64 bits along the same direction: what differences leave out is in `ideal` too
        t = [a.double().requires_grad_() for a in (x, r, gamma)]
        s = t[0] + t[1]
        ((s / torch.sqrt((s * s).mean(-1, keepdim=True) + eps) * t[2] * c.double()).sum() + (s * d.double()).sum()).backward()
        truth = float((t[which].grad * v.double()).sum())
        # every y and total is off by up to 60 units, on both sides of the difference
        size_of = float((c.double().abs() * 6).sum() + (total.double().abs() * d.double().abs()).sum())
        noise = 60 * ref.U * size_of / h
        _say("difference", got, "gradient", along, "truth", truth, "ideal", ideal, "noise", noise)
        assert abs(got - ideal) <= 2 * noise
        assert abs(along - truth) <= 200 * ref.U * (float(t[which].grad.abs().sum()) + size_of)


# Experts.


SORT_SIZES = [(1, 1, 1, 1), (2, 0, 2, 8), (1, 1, 8, 64), (3, 5, 2, 4), (2, 64, 1, 3), (1, 65, 3, 7), (4, 300, 2, 64), (9, 128, 2, 60),
              (2, 1000, 8, 256), (1, 4096, 2, 512), (3, 1025, 8, 513), (1, 700, 6, 2048), (2, 900, 3, 4096),
              (1, 30000, 8, 256), (2, 9000, 4, 3000), (5, 2049, 4, 17), (300, 3, 2, 8), (1, 100000, 1, 2), (2, 40000, 9, 31)]


def _choices(size, seed, id_type, holes):
    """Chosen experts, distinct within a token where there are enough, and a mask; `holes`: empty slots,
    numbers beyond the experts and masked tokens, one rank's all."""
    ranks, tokens, k, experts = size
    dev = _gen(seed)
    chosen = torch.randint(0, experts, (ranks, tokens, k), **dev)
    chosen = torch.where(torch.rand((ranks, tokens, k), **dev) < 0.3, chosen[:, :, :1] // 3, chosen)  # some more often
    mask = None
    if holes:
        chosen[torch.rand(chosen.shape, **dev) < 0.1] = -1
        chosen[torch.rand(chosen.shape, **dev) < 0.05] = experts
        chosen[torch.rand(chosen.shape, **dev) < 0.02] = -(2 ** 31)
        if id_type == torch.int64:
            chosen[torch.rand(chosen.shape, **dev) < 0.05] += 2 ** 32
        mask = torch.rand((ranks, tokens), **dev) < 0.7
        mask[ranks // 2] = False
    return chosen.to(id_type), mask


@pytest.mark.parametrize("holes", [False, True], ids=["full", "holes"])
@pytest.mark.parametrize("id_type", [torch.int32, torch.int64], ids=["i32", "i64"])
@pytest.mark.parametrize("size", SORT_SIZES, ids=_id)
def test_experts_sort(size, id_type, holes):
    import paper_2602_17254_amd as T

    ranks, tokens, k, experts = size
    _say("experts_sort", size, id_type, holes)
    chosen, mask = _choices(size, sum(size), id_type, holes)
    i32 = {"dtype": torch.int32, "device": "cuda"}
    offsets, places, slots = (torch.full(s, 77, **i32) for s in ((ranks, experts + 1), (ranks, tokens, k), (ranks, tokens * k)))
    ws = _bytes(T.trivance_experts_workspace_bytes(*size))
    T.trivance_experts_sort(chosen, offsets, places, ws, mask, slots)
    torch.cuda.synchronize()
    for name, got, want in zip(("offsets", "places", "slots"), (offsets, places, slots), more.experts_sort(chosen, mask, experts)):
        assert torch.equal(got.cpu().long(), torch.from_numpy(want)), name
    # without the slots, the mask as bytes
    again = torch.full_like(places, 5)
    T.trivance_experts_sort(chosen, offsets, again, ws, None if mask is None else mask.to(torch.uint8) * 3)
    assert torch.equal(again, places)


ROW_SIZES = [(1, 1, 1, 1), (1, 1, 8, 4096), (2, 3, 2, 5), (3, 33, 1, 64), (2, 70, 3, 65), (1, 9, 4, 255), (2, 40, 8, 129), (1, 130, 9, 513),
             (9, 17, 2, 1030), (1, 21, 5, 2051), (1, 5, 2, 20000), (300, 2, 2, 24), (1, 700, 17, 7), (2, 0, 2, 16),
             (2, 600, 8, 520)]


def _sorted_rows(size, seed, holes=True):
    """places of random choices, some of them beyond the sorted rows' capacity, and the capacity."""
    ranks, tokens, k, _ = size
    chosen, mask = _choices((ranks, tokens, k, 6), seed, torch.int32, holes)
    _, places, _ = more.experts_sort(chosen, mask, 6)
    places = torch.from_numpy(places).to("cuda", torch.int32)
    capacity = tokens * k + seed % 4 - 1 if tokens else 3
    return places, max(1, capacity)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", ROW_SIZES, ids=_id)
def test_experts_rows(size, dtype):
    """Out, back and the gradients, rows of no slot and between rows untouched."""
    import paper_2602_17254_amd as T

    ranks, tokens, k, width = size
    n, dt = sum(size), ref.DTYPES[dtype]
    _say("experts rows", size, dtype)
    places, capacity = _sorted_rows(size, n, n % 2 == 0)
    live = (places >= 0) & (places < capacity)
    dev = _gen(n)
    x, _ = _place(torch.randn((ranks, tokens, width), **dev), LAYOUTS[n % 4], dt)
    shape = (ranks, capacity, width)
    before = torch.randn(shape, **dev).to(dt)
    rows, base = _place(before, LAYOUTS[(n + 1) % 4], dt)
    T.trivance_experts_dispatch(x, places, rows)
    torch.cuda.synchronize()
    want = before.clone()
    rank = torch.arange(ranks, device="cuda").view(-1, 1, 1).expand(places.shape)[live]
    token = torch.arange(tokens, device="cuda").view(1, -1, 1).expand(places.shape)[live]
    want[rank, places[live].long()] = x[rank, token]
    assert torch.equal(rows, want)

    values, _ = _place(torch.randn(shape, **dev), LAYOUTS[(n + 2) % 4], dt)
    for wtype in (torch.float32, dt, None):
        weights = None if wtype is None else torch.randn(places.shape, **dev).to(wtype)
        w = torch.ones(places.shape, dtype=torch.float64, device="cuda") if weights is None else weights.double()
        y, ybase = _place(torch.zeros_like(x), LAYOUTS[(n + 3) % 4], dt)
        T.trivance_experts_combine(values, places, y, weights)
        torch.cuda.synchronize()
        wy, by = more.combine(values.double(), places, w)
        ref.assert_within(y, wy, by + ref.rounding(wy, dt) * 1.01, "y")
        _gaps_kept(y, ybase)

        dy, _ = _place(torch.randn(x.shape, **dev), LAYOUTS[n % 4], dt)
        drows, dbase = _place(before, LAYOUTS[(n + 1) % 4], dt)
        dweights = torch.full(places.shape, math.nan, device="cuda")
        T.trivance_experts_combine_backward(dy, values, places, weights, drows, dweights)
        torch.cuda.synchronize()
        (wd, bd), (ww, bw) = more.combine_backward(dy.double(), values.double(), places, w, before.double())
        untouched = bd == 0
        ref.assert_within(drows, wd, bd + torch.where(untouched, 0.0, ref.rounding(wd, dt) * 1.01), "drows")
        ref.assert_within(dweights, ww, bw, "dweights")
        # in place: the same bits, and rows of no slot as they were
        own = values.clone(memory_format=torch.contiguous_format)
        dw2 = torch.empty_like(dweights)
        T.trivance_experts_combine_backward(dy, own, places, weights, own, dw2)
        assert torch.equal(dw2, dweights)
        assert torch.equal(own, torch.where(untouched, values, drows))
        _gaps_kept(drows, dbase)
    _gaps_kept(rows, base)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vectors,more_values", [(128, 1), (192, 2), (256, 3), (320, 1)])
def test_experts_gradients_in_place_of_rows_that_end_inside_a_vector(vectors, more_values, dtype):
    """drows in rows' place, where a row's last vector and the one before it are of different waves: the bits of a
    call with rows of its own."""
    import paper_2602_17254_amd as T

    dt = ref.DTYPES[dtype]
    width = vectors * (4 if dt == torch.float32 else 8) + more_values
    dev = _gen(width)
    for k in (1, 2, 4, 8):
        ranks, tokens = 2, 1500
        places, capacity = _sorted_rows((ranks, tokens, k, width), 64)
        rows = torch.randn((ranks, capacity, width), **dev).to(dt)
        dy, weights = torch.randn((ranks, tokens, width), **dev).to(dt), torch.randn((ranks, tokens, k), **dev)
        drows, dweights, own = rows.clone(), torch.empty_like(weights), rows.clone()
        T.trivance_experts_combine_backward(dy, rows, places, weights, drows, dweights)
        again = torch.empty_like(dweights)
        T.trivance_experts_combine_backward(dy, own, places, weights, own, again)
        assert torch.equal(again, dweights) and torch.equal(own, drows), (width, k)


def test_experts_empty_slots_are_neither_read_nor_added():
    """Rows of no slot, weights of empty slots and dy of tokens without one may hold anything."""
    import paper_2602_17254_amd as T

    ranks, tokens, k, width = 2, 40, 3, 300
    places, capacity = _sorted_rows((ranks, tokens, k, width), 8)
    live = places >= 0
    assert bool((~live).any()) and bool((~live).all(2).any())
    dev = _gen(1)
    rows = torch.full((ranks, capacity, width), math.nan, device="cuda")
    rank = torch.arange(ranks, device="cuda").view(-1, 1, 1).expand(places.shape)[live]
    rows[rank, places[live].long()] = torch.randn((int(live.sum()), width), **dev)
    weights = torch.where(live, torch.randn(places.shape, **dev), math.inf)
    y = torch.empty((ranks, tokens, width), device="cuda")
    T.trivance_experts_combine(rows, places, y, weights)
    assert bool(torch.isfinite(y).all()) and bool((y[(~live).all(2)] == 0).all())
    dy = torch.where(live.any(2, keepdim=True), torch.randn(y.shape, **dev), math.nan)
    drows, dweights = torch.full_like(rows, 5.0), torch.empty_like(weights)
    T.trivance_experts_combine_backward(dy, rows, places, weights, drows, dweights)
    assert bool(torch.isfinite(drows).all()) and bool(torch.isfinite(dweights).all())
    assert bool((dweights[~live] == 0).all())


@pytest.mark.parametrize("width", [40, 770])
def test_experts_gradients_against_autograd(width):
    """Dispatch and combine with something in between, and the gradients of both, against autograd in 64 bits
    and against differences (the sums are bilinear, so differences are exact but for rounding)."""
    import paper_2602_17254_amd as T

    ranks, tokens, k, experts = 3, 50, 2, 5
    dev = _gen(width)
    chosen, mask = _choices((ranks, tokens, k, experts), 3, torch.int64, True)
    i32 = {"dtype": torch.int32, "device": "cuda"}
    offsets, places = torch.empty((ranks, experts + 1), **i32), torch.empty((ranks, tokens, k), **i32)
    T.trivance_experts_sort(chosen, offsets, places, _bytes(T.trivance_experts_workspace_bytes(ranks, tokens, k, experts)), mask)
    x, c = torch.randn((ranks, tokens, width), **dev), torch.randn((ranks, tokens, width), **dev)
    weights, factor = torch.rand((ranks, tokens, k), **dev), torch.randn((experts, width), **dev)

    def expert_of_row():
        row = torch.arange(tokens * k, device="cuda").expand(ranks, -1).contiguous()
        return torch.searchsorted(offsets[:, 1:].contiguous().long(), row, right=True).clamp(max=experts - 1)

    f = factor[expert_of_row()]

    def forward(x, weights):
        rows, y = torch.zeros((ranks, tokens * k, width), device="cuda"), torch.empty_like(x)
        T.trivance_experts_dispatch(x, places, rows)
        rows *= f
        T.trivance_experts_combine(rows, places, y, weights)
        return rows, y

    rows, y = forward(x, weights)
    drows, dweights, dx = torch.zeros_like(rows), torch.empty_like(weights), torch.empty_like(x)
    T.trivance_experts_combine_backward(c, rows, places, weights, drows, dweights)
    drows *= f
    T.trivance_experts_combine(drows, places, dx)

    tx, tw = x.double().requires_grad_(), weights.double().requires_grad_()
    live = (chosen >= 0) & (chosen < experts) & mask[..., None]
    of = factor.double()[torch.where(live, chosen, 0)]
    want = (torch.where(live, tw, 0.0)[..., None] * of * tx[:, :, None]).sum(2)
    (want * c.double()).sum().backward()
    size = (weights.double()[..., None] * of.abs() * live[..., None]).sum(2)
    ref.assert_within(y, want.detach(), 8 * ref.U * size * x.double().abs() + 1e-45, "y")
    ref.assert_within(dx, tx.grad, 8 * ref.U * size * c.double().abs() + 1e-45, "dx")
    terms = (of * x.double()[:, :, None] * c.double()[:, :, None] * live[..., None]).abs().sum(3)
    ref.assert_within(dweights, tw.grad, (width / 64 + 30) * ref.U * terms + 1e-45, "dweights")
    h = 0.5
    vx, vw = torch.sign(torch.randn(x.shape, **dev)), torch.sign(torch.randn(weights.shape, **dev))
    for got, (plus, minus) in (((dx.double() * vx.double()).sum(), ((x + h * vx, weights), (x - h * vx, weights))),
                               ((dweights.double() * vw.double()).sum(), ((x, weights + h * vw), (x, weights - h * vw)))):
        across = float(((forward(*plus)[1].double() - forward(*minus)[1].double()) * c.double()).sum()) / (2 * h)
        most = float(((size + k * of.abs().amax(2)) * (x.double().abs() + 1) * c.double().abs()).sum())
        _say("difference", across, "gradient", float(got))
        assert abs(across - float(got)) <= 40 * ref.U * most


# Embedding.


TABLE_SIZES = [(1, 1, 1, 1), (5, 128, 40, 50), (5, 129, 40, 50), (2, 64, 900, 520), (2, 127, 3, 4097), (2, 3, 5, 7), (1, 1, 50000, 64), (3, 100, 10, 33), (2, 0, 20, 16), (1, 65, 1, 130), (2, 700, 1024, 40), (2, 700, 1025, 40), (2, 700, 4096, 40),
               (2, 700, 4097, 40), (1, 5000, 300, 257), (9, 333, 1000, 100), (1, 20000, 70000, 24), (3, 3000, 9, 515),
               (1, 300, 7, 9000), (2, 17000, 131, 64), (70, 40, 60, 8), (1, 40000, 2, 65)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", TABLE_SIZES, ids=_id)
def test_embedding(size, dtype):
    import paper_2602_17254_amd as T

    ranks, tokens, vocab, width = size
    n, dt = sum(size), ref.DTYPES[dtype]
    scale = [1.0, math.sqrt(width), -0.3][n % 3]
    id_type = [torch.int32, torch.int64][n % 2]
    _say("embedding", size, dtype, scale)
    dev = _gen(n)
    # few numbers often, the rest rarely
    ids = (vocab ** torch.rand((ranks, tokens), dtype=torch.float64, **dev)).long() - 1
    ids = ids.clamp(max=vocab - 1)
    if n % 3:
        ids[torch.rand(ids.shape, **dev) < 0.1] = -1
        ids[torch.rand(ids.shape, **dev) < 0.05] = vocab
        if id_type == torch.int64:
            ids[torch.rand(ids.shape, **dev) < 0.02] += 2 ** 32
    live = (ids >= 0) & (ids < vocab)
    ids = ids.to(id_type)
    ttype = [torch.float32, dt, torch.bfloat16][n % 3]
    table = torch.randn((vocab, width + 3), **dev).to(ttype)[:, 1:width + 1]
    y, base = _place(torch.zeros((ranks, tokens, width), device="cuda"), LAYOUTS[n % 4], dt)
    T.trivance_embedding_forward(ids, table, y, scale)
    torch.cuda.synchronize()
    want = torch.where(live[..., None], table.double()[torch.where(live, ids, 0).long()] * scale, 0.0)
    ref.assert_within(y, want, 2 * ref.U * want.abs() + ref.rounding(want, dt) * 1.01 * live[..., None] + 1e-45, "y")
    _gaps_kept(y, base)

    dy, _ = _place(torch.randn((ranks, tokens, width), **dev), LAYOUTS[(n + 1) % 4], dt)
    dy[~live] = math.nan  # what padding has is not read
    # each rank's row of a vector to sum: other gradients, the table's, a gap
    rows = torch.full((ranks, vocab * width + 9), PATTERN, device="cuda")
    dtable = rows[:, 4:4 + vocab * width].unflatten(1, (vocab, width))
    ws = _bytes(T.trivance_embedding_workspace_bytes(ranks, tokens, width, vocab))
    T.trivance_embedding_backward(dy, ids, dtable, ws, scale)
    torch.cuda.synchronize()
    want, bound = more.table_gradient(dy.double(), ids, vocab, scale, more.piece_of(tokens))
    ref.assert_within(dtable, want, bound, "dtable")
    dtable.fill_(PATTERN)
    assert bool((rows == PATTERN).all())


@pytest.mark.parametrize("tokens", [64, 65, 128, 129, 192, 4096, 4097, 9000])
@pytest.mark.parametrize("dtype", TYPES)
def test_embedding_runs_that_start_and_end_at_pieces(tokens, dtype):
    """Long runs of one number beside others, whose ends fall on, before and behind the ends of pieces."""
    import paper_2602_17254_amd as T

    width, vocab, piece = 70, 12, more.piece_of(tokens)
    for lengths in ((tokens,), (piece, tokens - piece), (piece + 1, 0, 3, tokens - piece - 4), (1, piece, tokens - piece - 1),
                    (piece - 1, piece + 1, tokens - 2 * piece), (0, 0, tokens // 2, tokens - tokens // 2)):
        if min(lengths) < 0:
            continue
        ids = torch.repeat_interleave(torch.arange(len(lengths)), torch.tensor(lengths)).view(1, -1)
        ids = torch.cat((ids, ids.flip(1)))[:, torch.randperm(tokens, generator=torch.Generator().manual_seed(tokens))].to("cuda")
        dy = torch.randn((2, tokens, width), **_gen(tokens)).to(ref.DTYPES[dtype])
        d = torch.full((2, vocab, width), math.nan, device="cuda")
        T.trivance_embedding_backward(dy, ids, d, _bytes(T.trivance_embedding_workspace_bytes(2, tokens, width, vocab)))
        want, bound = more.table_gradient(dy.double(), ids, vocab, 1.0, piece)
        ref.assert_within(d, want, bound, "dtable of %s" % (lengths,))


def test_embedding_gradient_against_differences():
    """The sum of the ranks' gradients, through the framework's AllReduce, along a direction: lookups are linear in
    the table."""
    import paper_2602_17254_amd as T

    ranks, tokens, vocab, width, scale = 9, 60, 40, 64, 8.0
    dev = _gen(4)
    ids = torch.randint(-1, vocab, (ranks, tokens), **dev)
    table, c, v = torch.randn((vocab, width), **dev), torch.randn((ranks, tokens, width), **dev), torch.randn((vocab, width), **dev)
    rows = torch.empty((ranks, vocab * width), device="cuda")
    T.trivance_embedding_backward(c, ids, rows.unflatten(1, (vocab, width)),
                                  _bytes(T.trivance_embedding_workspace_bytes(ranks, tokens, width, vocab)), scale)
    T.trivance_allreduce_emulated(rows, T.trivance_plan((ranks,), "B"))
    y = [torch.empty_like(c) for _ in range(2)]
    T.trivance_embedding_forward(ids, table + v, y[0], scale)
    T.trivance_embedding_forward(ids, table - v, y[1], scale)
    across = float(((y[0].double() - y[1].double()) * c.double()).sum()) / 2
    size = float(((y[0].double().abs() + y[1].double().abs()) * c.double().abs()).sum())
    for r in (0, 4, 8):
        along = float((rows[r].double() * v.double().flatten()).sum())
        assert abs(across - along) <= 40 * ref.U * (size + float((rows[r].double() * v.double().flatten()).abs().sum()))


# Dropout.


DROP_SIZES = [(1, 1, 1), (2, 3, 7), (1, 5, 8), (3, 33, 63), (2, 70, 64), (1, 9, 65), (2, 17, 255), (3, 5, 513), (1, 13, 2051), (1, 3, 20001),
              (300, 2, 40), (2, 0, 16), (1, 700, 24)]


def _state(seed, call):
    return torch.tensor([seed, call], dtype=torch.int64, device="cuda")


@pytest.mark.parametrize("rate", [0.0, 0.1, 0.5, 0.999])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", DROP_SIZES, ids=_id)
def test_dropout(size, dtype, rate):
    import paper_2602_17254_amd as T

    n, dt = sum(size), ref.DTYPES[dtype]
    seed, call = [n * 0x9E3779B97F4A7C1 % (1 << 62), -n, n][n % 3], [n, (1 << 32) - 1, (1 << 32) + 5][n % 3]
    _say("dropout", size, dtype, rate)
    kept = torch.from_numpy(more.kept(size, seed, call, rate)).to("cuda")
    state, dev = _state(seed, call), _gen(n)
    x, _ = _place(torch.randn(size, **dev), LAYOUTS[n % 4], dt)
    res, _ = _place(torch.randn(size, **dev), LAYOUTS[(n + 1) % 4], dt)
    x[~kept] = math.nan  # a dropped value counts as zero, whatever it is
    limit = round(rate * 65536)
    for residual in (None, res):
        y, base = _place(torch.full(size, math.nan, device="cuda"), LAYOUTS[(n + 2) % 4], dt)
        T.trivance_dropout(x, y, state, rate, residual)
        torch.cuda.synchronize()
        part = torch.where(kept, x.double() / (1 - limit / 65536), 0.0)
        want = part if residual is None else part + residual.double()
        bound = 2 * ref.U * part.abs() + ref.U * want.abs() + 1e-45
        ref.assert_within(y, want, torch.where(kept | (residual is not None), bound + ref.rounding(want, dt) * 1.01, 0.0), "y")
        for at in (x, residual):
            if at is not None:
                ins = [x.clone(), None if residual is None else residual.clone()]
                to = ins[0] if at is x else ins[1]
                T.trivance_dropout(ins[0], to, state, rate, ins[1])
                assert torch.equal(to, y)
        _gaps_kept(y, base)


def test_dropout_of_a_rank_does_not_depend_on_the_others():
    import paper_2602_17254_amd as T

    x, state = torch.randn((9, 50, 130), **_gen(1)), _state(77, 3)
    y, more_ranks, wide = torch.empty_like(x), torch.empty((3, 50, 130), device="cuda"), torch.empty((9, 60, 200), device="cuda")
    T.trivance_dropout(x, y, state, 0.3)
    T.trivance_dropout(x[:3].contiguous(), more_ranks, state, 0.3)
    assert torch.equal(y[:3], more_ranks)
    big = torch.ones((9, 60, 200), device="cuda")
    big[:, :50, :130] = x
    T.trivance_dropout(big, wide, state, 0.3)
    assert torch.equal(wide[:, :50, :130], y)


# All of them.


def _step(T, seed):
    """Inputs and buffers of every call, and a function that makes them all."""
    dev = _gen(seed)
    ranks, tokens, width, experts, k, vocab = 4, 200, 300, 24, 2, 500
    f32, i32 = {"device": "cuda"}, {"dtype": torch.int32, "device": "cuda"}
    x, dy = (torch.randn((ranks, tokens, width), **dev).bfloat16() for _ in range(2))
    gamma, table = torch.randn(width, **dev), torch.randn((vocab, width), **dev)
    ids = torch.randint(-1, vocab, (ranks, tokens), **dev)
    ids[:, :90] = 3
    chosen = torch.topk(torch.randn((ranks, tokens, experts), **dev), k, dim=2).indices
    weights = torch.rand((ranks, tokens, k), **dev)
    state = _state(9, 4)
    work = [_bytes(n) for n in (T.trivance_rmsnorm_workspace_bytes(ranks, tokens, width),
                                T.trivance_experts_workspace_bytes(ranks, tokens, k, experts),
                                T.trivance_embedding_workspace_bytes(ranks, tokens, width, vocab))]

    def buffers():
        rows = (ranks, tokens * k, width)
        b = {n: torch.zeros_like(x) for n in ("drop", "total", "y", "back", "dx", "lookup")}
        b |= {n: torch.zeros(rows, dtype=x.dtype, device="cuda") for n in ("rows", "drows")}
        b |= {"rstd": torch.zeros((ranks, tokens), **f32), "scales": torch.zeros((ranks, tokens), **f32),
              "q": torch.zeros(x.shape, dtype=torch.uint8, device="cuda"), "dgamma": torch.zeros((ranks, width), **f32),
              "offsets": torch.zeros((ranks, experts + 1), **i32), "places": torch.zeros((ranks, tokens, k), **i32),
              "slots": torch.zeros((ranks, tokens * k), **i32), "dweights": torch.zeros((ranks, tokens, k), **f32),
              "dtable": torch.zeros((ranks, vocab, width), **f32)}
        return b

    def run(b, stream=None):
        T.trivance_embedding_forward(ids, table, b["lookup"], 2.0, stream)
        T.trivance_dropout(x, b["drop"], state, 0.2, b["lookup"], stream)
        T.trivance_rmsnorm_forward(b["drop"], gamma, b["y"], b["rstd"], x, b["total"], stream=stream)
        T.trivance_rmsnorm_forward(b["drop"], gamma, b["q"].view(torch.float8_e4m3fn), None, x, None, b["scales"], stream=stream)
        T.trivance_experts_sort(chosen, b["offsets"], b["places"], work[1], None, b["slots"], stream)
        T.trivance_experts_dispatch(b["y"], b["places"], b["rows"], stream)
        T.trivance_experts_combine(b["rows"], b["places"], b["back"], weights, stream)
        T.trivance_experts_combine_backward(dy, b["rows"], b["places"], weights, b["drows"], b["dweights"], stream)
        T.trivance_rmsnorm_backward(dy, b["total"], gamma, b["rstd"], b["dx"], b["dgamma"], work[0], b["back"], stream)
        T.trivance_embedding_backward(dy, ids, b["dtable"], work[2], 2.0, stream)

    return buffers, run, state


def test_more_operators_repeat_on_streams_and_in_graphs():
    """The same bits on another stream and from the replays of a captured graph; a graph's dropout follows the
    call number that the program counts up between the replays."""
    import paper_2602_17254_amd as T

    buffers, run, state = _step(T, 12)
    want, other, replayed = buffers(), buffers(), buffers()
    run(want)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    run(other, stream)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(replayed)
    drops = []
    for turn in range(4):
        for t in replayed.values():
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for name in want:
            assert torch.equal(want[name], replayed[name]), (name, turn)
            if turn == 0:
                assert torch.equal(want[name], other[name]), name
        drops.append(want["drop"].clone())
        # the program's own work between replays: the next call's number, and what it gives eagerly
        state[1] += 1
        run(want)
    assert not torch.equal(drops[0], drops[1]) and not torch.equal(drops[1], drops[2])


def test_two_graphs_and_eager_calls_with_workspaces_of_their_own():
    """Two captured graphs, replayed in turn on two streams at once, each with its own buffers and workspaces."""
    import paper_2602_17254_amd as T

    sides = []
    for seed in (1, 2):
        buffers, run, _ = _step(T, seed)
        want, got = buffers(), buffers()
        run(want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run(got)
        sides.append((want, got, graph, torch.cuda.Stream(), run))  # run keeps the inputs that the graph reads
    torch.cuda.synchronize()
    for _ in range(3):
        for _, _, graph, stream, _ in sides:
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for want, got, _, _, _ in sides:
            for name in want:
                assert torch.equal(want[name], got[name]), name


def test_offsets_beyond_32_bits():
    """Rows and ranks further than 2^31 elements apart."""
    import paper_2602_17254_amd as T

    far = 2 ** 31 + 72
    base, out, third = (torch.zeros(far + 4000, dtype=torch.bfloat16, device="cuda") for _ in range(3))
    dev = _gen(2)
    for shape, strides in (((1, 2, 300), (0, far, 1)), ((2, 1, 300), (far, 300, 1)), ((2, 3, 77), (far, 80, 1))):
        ranks, tokens, width = shape
        x, y, z = (t.as_strided(shape, strides) for t in (base, out, third))
        near = torch.randn(shape, **dev).bfloat16()
        x.copy_(near)
        want, total = torch.empty_like(near), torch.empty_like(near)
        rstd = torch.empty(shape[:2], device="cuda")
        T.trivance_rmsnorm_forward(near, None, want, rstd, near, total)
        T.trivance_rmsnorm_forward(x, None, y, rstd, x, z)
        assert torch.equal(y, want) and torch.equal(z, total)
        ws = _bytes(T.trivance_rmsnorm_workspace_bytes(*shape))
        dg = [torch.empty((ranks, width), device="cuda") for _ in range(2)]
        T.trivance_rmsnorm_backward(near, near, None, rstd, want, dg[0], ws, near)
        T.trivance_rmsnorm_backward(x, x, None, rstd, y, dg[1], ws, x)
        assert torch.equal(y, want) and torch.equal(dg[0], dg[1])

        places = torch.arange(tokens, dtype=torch.int32, device="cuda").flip(0).expand(ranks, -1)[..., None].contiguous()
        w = torch.rand(places.shape, **dev)
        T.trivance_experts_dispatch(near, places, want)
        T.trivance_experts_dispatch(x, places, y)
        assert torch.equal(y, want)
        T.trivance_experts_combine(near, places, want, w)
        T.trivance_experts_combine(x, places, y, w)
        assert torch.equal(y, want)
        dw = [torch.empty_like(w) for _ in range(2)]
        T.trivance_experts_combine_backward(near, near, places, w, want, dw[0])
        T.trivance_experts_combine_backward(x, x, places, w, y, dw[1])
        assert torch.equal(y, want) and torch.equal(dw[0], dw[1])

        state = _state(1, 2)
        T.trivance_dropout(near, want, state, 0.4, near)
        T.trivance_dropout(x, y, state, 0.4, x)
        assert torch.equal(y, want)

        ids = torch.zeros((ranks, tokens), dtype=torch.int32, device="cuda")
        ids[:, 0] = 1
        table = torch.randn((2, width), **dev).bfloat16()
        far_table = third.as_strided((2, width), (far, 1))
        far_table.copy_(table)
        T.trivance_embedding_forward(ids, table, want, 3.0)
        T.trivance_embedding_forward(ids, far_table, y, 3.0)
        assert torch.equal(y, want)
        ws = _bytes(T.trivance_embedding_workspace_bytes(ranks, tokens, width, 2))
        d = [torch.empty((ranks, 2, width), device="cuda") for _ in range(2)]
        T.trivance_embedding_backward(near, ids, d[0], ws, 3.0)
        T.trivance_embedding_backward(x, ids, d[1], ws, 3.0)
        assert torch.equal(d[0], d[1])
    wide = torch.zeros(far + 4000, device="cuda")
    d = wide.as_strided((2, 2, 77), (far, 77, 1))
    T.trivance_embedding_backward(near, ids, d, ws, 3.0)
    want = torch.empty((2, 2, 77), device="cuda")
    T.trivance_embedding_backward(near, ids, want, ws, 3.0)
    assert torch.equal(d, want)


def test_more_than_2_31_values():
    """bf16 tensors of more than 2^31 values: every call's rows at both ends have the bits of small calls."""
    import paper_2602_17254_amd as T

    ranks, tokens, width = 8, 65537, 4100
    x = torch.empty((ranks, tokens, width), dtype=torch.bfloat16, device="cuda")
    dev = _gen(1)
    for part in x:
        part.copy_(torch.randn(part.shape, **dev))
    assert x.numel() > 2 ** 31
    y, total, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty((ranks, tokens), device="cuda")
    ends = [(r, slice(a, a + 40)) for r in (0, ranks - 1) for a in (0, tokens - 40)]

    def small(r, part, t=x):
        return t[r:r + 1, part].contiguous()

    T.trivance_rmsnorm_forward(x, None, y, rstd, x, total)
    for r, part in ends:
        one = small(r, part)
        y1, t1 = torch.empty_like(one), torch.empty_like(one)
        T.trivance_rmsnorm_forward(one, None, y1, None, one, t1)
        assert torch.equal(small(r, part, y), y1) and torch.equal(small(r, part, total), t1)
    dg = torch.empty((ranks, width), device="cuda")
    T.trivance_rmsnorm_backward(x, total, None, rstd, y, dg, _bytes(T.trivance_rmsnorm_workspace_bytes(*x.shape)), x)
    for r, part in ends:
        one = small(r, part)
        d1 = torch.empty_like(one)
        T.trivance_rmsnorm_backward(one, small(r, part, total), None, rstd[r:r + 1, part].contiguous(), d1, None, None, one)
        assert torch.equal(small(r, part, y), d1)
        h = total[r].double() * rstd[r, :, None].double()
        ref.assert_within(dg[r], (x[r].double() * h).sum(0), (tokens + 40) * ref.U * (x[r].double() * h).abs().sum(0), "dgamma")
        del h

    # one slot a token, the tokens in the order of two experts, the second's first
    chosen = (torch.arange(tokens, device="cuda") % 2).flip(0).expand(ranks, -1)[..., None].to(torch.int32).contiguous()
    offsets, places = torch.empty((ranks, 3), dtype=torch.int32, device="cuda"), torch.empty_like(chosen)
    T.trivance_experts_sort(chosen, offsets, places, _bytes(T.trivance_experts_workspace_bytes(ranks, tokens, 1, 2)))
    T.trivance_experts_dispatch(x, places, total)
    w = torch.rand(places.shape, **dev)
    T.trivance_experts_combine(total, places, y, w)
    for r, part in ends:
        assert torch.equal(total[r][places[r, part, 0].long()], x[r, part])
        assert torch.equal(y[r, part], (x[r, part].float() * w[r, part]).bfloat16())
    dw = torch.empty_like(w)
    T.trivance_experts_combine_backward(x, total, places, w, total, dw)
    for r, part in ends:
        assert torch.equal(total[r][places[r, part, 0].long()], y[r, part])
        want = x[r, part].double().square().sum(1)
        ref.assert_within(dw[r, part, 0], want, (width / 64 + 24) * ref.U * want, "dweights")

    state = _state(3, 1)
    T.trivance_dropout(x, y, state, 0.25)
    for r, part in ends:
        kept = torch.from_numpy(more.kept((1, tokens, 8), 3, 1, 0.25, r)).to("cuda")[0, part]
        assert torch.equal(y[r, part, :8], torch.where(kept, (x[r, part, :8].float() / 0.75), 0.0).bfloat16())


def test_embedding_gradient_of_more_than_2_31_values():
    """A table of 9 GB: the rows at both ends and between them, and zeros everywhere else, where there was none before."""
    import paper_2602_17254_amd as T

    vocab, width = 140001, 16400
    d = torch.full((1, vocab, width), math.nan, device="cuda")
    assert d.numel() > 2 ** 31 + 2 ** 27
    ids = torch.tensor([[vocab - 1, 0, 131000, vocab - 1, -1, 77]], device="cuda")
    dy = torch.randn((1, 6, width), **_gen(1))
    T.trivance_embedding_backward(dy, ids, d, _bytes(T.trivance_embedding_workspace_bytes(1, 6, width, vocab)), 2.0)
    for v, want in ((vocab - 1, dy[0, 0] + dy[0, 3]), (0, dy[0, 1]), (131000, dy[0, 2]), (77, dy[0, 5])):
        assert torch.equal(d[0, v], 2 * want)
        d[0, v] = 0.0
    assert not any(bool(part.any()) for part in d[0].split(10000))


def test_combine_of_no_sorted_rows():
    """A capacity of zero: every slot is passed over."""
    import paper_2602_17254_amd as T

    rows, places = torch.empty((2, 0, 40), device="cuda"), torch.zeros((2, 5, 3), dtype=torch.int32, device="cuda")
    y, w, dw = torch.full((2, 5, 40), 3.0, device="cuda"), torch.ones((2, 5, 3), device="cuda"), torch.full((2, 5, 3), 3.0, device="cuda")
    T.trivance_experts_dispatch(y, places, rows)
    T.trivance_experts_combine_backward(y, rows, places, w, rows, dw)
    T.trivance_experts_combine(rows, places, y, w)
    assert bool((y == 0).all()) and bool((dw == 0).all())


@pytest.mark.parametrize("width", [24, 1030])
def test_more_ranks_than_a_grid_has_rows(width):
    """Workgroups that go on to another rank."""
    import paper_2602_17254_amd as T

    ranks, tokens, k, dev = 65535 + 70, 2, 2, _gen(width)
    some = list(range(70)) + [30000] + list(range(65535, ranks))
    x = torch.randn((ranks, tokens, width), **dev).bfloat16()

    def calls(x, chosen, ids, w, first):
        n = x.shape[0]
        out = {}
        y, total, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty((n, tokens), device="cuda")
        # rows apart, so that the ranks are not taken as one
        apart = torch.empty((n, tokens * width + 8), dtype=x.dtype, device="cuda")[:, :tokens * width].unflatten(1, (tokens, width))
        T.trivance_rmsnorm_forward(x, None, apart, rstd, x, total)
        dg = torch.empty((n, width), device="cuda")
        T.trivance_rmsnorm_backward(x, total, None, rstd, y, dg, _bytes(T.trivance_rmsnorm_workspace_bytes(n, tokens, width)))
        out |= {"y": apart, "dx": y, "dg": dg}
        offsets, places = torch.empty((n, 6), dtype=torch.int32, device="cuda"), torch.empty((n, tokens, k), dtype=torch.int32, device="cuda")
        T.trivance_experts_sort(chosen, offsets, places, _bytes(T.trivance_experts_workspace_bytes(n, tokens, k, 5)))
        rows, back, drows = (torch.zeros((n, t, width), dtype=x.dtype, device="cuda") for t in (tokens * k, tokens, tokens * k))
        dw = torch.empty_like(w)
        T.trivance_experts_dispatch(x, places, rows)
        T.trivance_experts_combine(rows, places, back, w)
        T.trivance_experts_combine_backward(x, rows, places, w, drows, dw)
        out |= {"offsets": offsets, "places": places, "rows": rows, "back": back, "drows": drows, "dw": dw}
        looked, d = torch.empty_like(x), torch.empty((n, 3, width), device="cuda")
        T.trivance_embedding_forward(ids, table, looked)
        T.trivance_embedding_backward(x, ids, d, _bytes(T.trivance_embedding_workspace_bytes(n, tokens, width, 3)))
        out |= {"looked": looked, "dtable": d}
        if first:
            drop = torch.empty_like(x)
            T.trivance_dropout(x, drop, _state(5, 6), 0.5)
            kept = torch.from_numpy(more.kept((70, tokens, width), 5, 6, 0.5, 65535)).to("cuda")
            assert torch.equal(drop[65535:], torch.where(kept, x[65535:] * 2, torch.zeros_like(x[65535:])))
        return out

    table = torch.randn((3, width), **dev)
    chosen, ids = torch.randint(-1, 5, (ranks, tokens, k), **dev), torch.randint(-1, 3, (ranks, tokens), **dev)
    w = torch.rand((ranks, tokens, k), **dev)
    every = calls(x, chosen, ids, w, True)
    few = calls(x[some].contiguous(), chosen[some].contiguous(), ids[some].contiguous(), w[some].contiguous(), False)
    for name in few:
        assert torch.equal(every[name][some], few[name]), name


@pytest.mark.parametrize("dtype", TYPES)
def test_tensors_beyond_the_caches(dtype):
    """Large tensors take other loads and stores: every row has the bits that it has in a call of its rank alone,
    which is small."""
    import paper_2602_17254_amd as T

    dt, dev = ref.DTYPES[dtype], _gen(8)
    size = torch.finfo(dt).bits // 8
    ranks, tokens, width, k = 6, 701, 12007 // size, 2
    x, _ = _place(torch.randn((ranks, tokens, width), **dev), "padded", dt)
    assert x.numel() * size > 2 ** 25 > x[:1].numel() * size * k
    places = torch.rand((ranks, tokens * k), **dev).argsort(1).to(torch.int32).view(ranks, tokens, k)
    w, ids = torch.rand(places.shape, **dev), torch.randint(-1, 300, (ranks, tokens), **dev)
    table = torch.randn((300, width), **dev)

    def calls(part):
        xs, ps, ws, n = x[part], places[part].contiguous(), w[part].contiguous(), x[part].shape[0]

        def rows(t):
            return _place(torch.zeros((n, t, width), device="cuda"), "padded", dt)

        made = {"y": rows(tokens), "total": rows(tokens), "dx": rows(tokens), "rows": rows(tokens * k), "back": rows(tokens),
                "drows": rows(tokens * k), "looked": rows(tokens)}
        o = {name: view for name, (view, _) in made.items()}
        o["rstd"], o["scales"] = torch.empty((n, tokens), device="cuda"), torch.empty((n, tokens), device="cuda")
        o["q"] = torch.empty((n, tokens, width), dtype=torch.uint8, device="cuda")
        o["dw"], o["dtable"] = torch.empty_like(ws), torch.empty((n, 300, width), device="cuda")
        T.trivance_rmsnorm_forward(xs, None, o["y"], o["rstd"], xs, o["total"])
        T.trivance_rmsnorm_forward(xs, None, o["q"].view(torch.float8_e4m3fn), None, xs, None, o["scales"])
        T.trivance_rmsnorm_backward(xs, o["total"], None, o["rstd"], o["dx"], None, None, xs)
        T.trivance_experts_dispatch(xs, ps, o["rows"])
        T.trivance_experts_combine(o["rows"], ps, o["back"], ws)
        T.trivance_experts_combine_backward(xs, o["rows"], ps, ws, o["drows"], o["dw"])
        T.trivance_embedding_forward(ids[part].contiguous(), table, o["looked"])
        T.trivance_embedding_backward(xs, ids[part].contiguous(), o["dtable"],
                                      _bytes(T.trivance_embedding_workspace_bytes(n, tokens, width, 300)))
        out = {name: t.clone() for name, t in o.items()}
        for view, base in made.values():
            _gaps_kept(view, base)
        return out

    every = calls(slice(None))
    for r in range(ranks):
        for name, t in calls(slice(r, r + 1)).items():
            assert torch.equal(every[name][r:r + 1], t), name
    drop, base = _place(torch.zeros_like(x), "padded", dt)
    T.trivance_dropout(x, drop, _state(2, 2), 0.5)
    kept = torch.from_numpy(more.kept(x.shape, 2, 2, 0.5)).to("cuda")
    assert torch.equal(drop, torch.where(kept, x * 2, torch.zeros_like(x)))
    _gaps_kept(drop, base)


@pytest.mark.parametrize("shape", [(1, 3, 40), (3, 1, 40), (1, 1, 700)], ids=_id)
def test_in_place_strides_of_a_single_rank_or_token_do_not_matter(shape):
    import paper_2602_17254_amd as T

    ranks, tokens, width = shape
    dev = _gen(width)
    other = (width if ranks > 1 else 977, width if tokens > 1 else 1013, 1)
    x, dy, state = torch.randn(shape, **dev), torch.randn(shape, **dev), _state(1, 2)
    y, dx, rstd, drop = torch.empty_like(x), torch.empty_like(x), torch.empty(shape[:2], device="cuda"), torch.empty_like(x)
    T.trivance_rmsnorm_forward(x, None, y, rstd)
    T.trivance_rmsnorm_backward(dy, x, None, rstd, dx, None)
    T.trivance_dropout(x, drop, state, 0.5)
    for call, want in ((lambda t: T.trivance_rmsnorm_forward(t, None, t.as_strided(shape, other)), y),
                       (lambda t: T.trivance_rmsnorm_backward(dy, t, None, rstd, t.as_strided(shape, other), None), dx),
                       (lambda t: T.trivance_dropout(t, t.as_strided(shape, other), state, 0.5), drop)):
        own = x.clone()
        call(own)
        assert torch.equal(own, want)
    # one token and one sorted row a rank
    if tokens == 1:
        places, w = torch.zeros((ranks, 1, 1), dtype=torch.int32, device="cuda"), torch.rand((ranks, 1, 1), **dev)
        drows, dw, own = torch.empty_like(x), torch.empty_like(w), x.clone()
        T.trivance_experts_combine_backward(dy, x, places, w, drows, dw)
        T.trivance_experts_combine_backward(dy, own, places, w, own.as_strided(shape, other), torch.empty_like(w))
        assert torch.equal(own, drows)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("width", [100003, 1 << 20, (1 << 24) - 1, 1 << 24])
def test_rmsnorm_sums_of_the_longest_rows(width, dtype):
    """Rows of values whose sums round the same way at every step, and of any: the bounds of short rows hold. A lane's sum
    of a vector passes 8 roundings, 64 lanes' 6, the waves' 16, which SUM covers whatever the width."""
    import paper_2602_17254_amd as T

    _say("rmsnorm long", width, dtype)
    dt, dev = ref.DTYPES[dtype], _gen(width)
    x = torch.randn((1, 3, width), **dev)
    x[0, 0] = 1.1
    x[0, 1] = x[0, 1].abs() + 0.3
    dy = torch.randn((1, 3, width), **dev)
    dy[0, :2] = 0.7
    x, dy, gamma = x.to(dt), dy.to(dt), 1 + 0.1 * torch.rand(width, **dev)
    y, rstd = torch.empty_like(x), torch.empty((1, 3), device="cuda")
    T.trivance_rmsnorm_forward(x, gamma, y, rstd)
    (want, by), (wr, br) = more.rmsnorm_forward(x.double(), gamma.double(), 1e-5)
    ref.assert_within(rstd, wr, br, "rstd")
    ref.assert_within(y, want, by + ref.rounding(want, dt) * 1.01, "y")
    q, scales = torch.empty(x.shape, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty_like(rstd)
    T.trivance_rmsnorm_forward(x, gamma, q, scales=scales)
    (wq, bq), (ws, bs) = more.eight_bits(want)
    ref.assert_within(scales, ws, bs, "scales")
    ref.assert_within(q.float(), wq, bq, "8 bits")
    dx, dg = torch.empty_like(x), torch.empty((1, width), device="cuda")
    T.trivance_rmsnorm_backward(dy, x, gamma, rstd, dx, dg, _bytes(T.trivance_rmsnorm_workspace_bytes(1, 3, width)))
    (wx, bx), (wg, bg) = more.rmsnorm_backward(dy.double(), x.double(), gamma.double(), rstd.double(), None)
    ref.assert_within(dx, wx, bx + ref.rounding(wx, dt) * 1.01, "dx")
    ref.assert_within(dg, wg, bg, "dgamma")


def test_more_than_2_31_values_leave_no_row_and_no_column_out():
    """Weights' gradients of whole numbers, whose sums fp32 holds, are equal to the last one; dropout's places of whole
    rows, the last block of columns, which is not full, among them."""
    import paper_2602_17254_amd as T

    ranks, tokens, width = 8, 65537, 4100
    dev = _gen(5)
    x, dy, dx = (torch.empty((ranks, tokens, width), dtype=torch.bfloat16, device="cuda") for _ in range(3))
    assert x.numel() > 2 ** 31 and tokens * 9 < 2 ** 24
    for r in range(ranks):
        for t in (x, dy):
            t[r] = torch.randint(-3, 4, (tokens, width), dtype=torch.int8, **dev)
    rstd, dg = torch.ones((ranks, tokens), device="cuda"), torch.empty((ranks, width), device="cuda")
    T.trivance_rmsnorm_backward(dy, x, None, rstd, dx, dg, _bytes(T.trivance_rmsnorm_workspace_bytes(*x.shape)))
    for r in range(ranks):
        assert torch.equal(dg[r].double(), (x[r].double() * dy[r].double()).sum(0)), r

    seed, call, rate = 7, 9, 0.25
    T.trivance_dropout(x, dx, _state(seed, call), rate)
    blocks = -(-width // 8)
    for r in (0, 3, ranks - 1):
        for t in (0, 1, tokens // 2, tokens - 1):
            words = more.philox((range(blocks), [t] * blocks, [r] * blocks, [call] * blocks), (seed, 0))
            halves = torch.tensor([[int(w[b]) >> s & 0xFFFF for w in words for s in (0, 16)] for b in range(blocks)])
            kept = (halves.flatten()[:width] >= round(rate * 65536)).to("cuda")
            assert torch.equal(dx[r, t], torch.where(kept, x[r, t].float() / 0.75, 0.0).bfloat16()), (r, t)
