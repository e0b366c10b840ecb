"""The operators of a data-parallel training step around the AllReduce, with their inputs, plain forms
and exact results.

Every operator works on the framework's layout: one row of memory per virtual rank, rank-major. A
rank's tokens pass a layer norm, whose weight gradients each rank writes straight into its row of the
vector that the AllReduce sums; a router's balance loss is formed from per-expert counts (int32) and
sums of probabilities (fp32) that the AllReduce sums as well; and a summed matrix gradient is
orthogonalised before it is applied. The fields of a case:

    op       "layernorm_forward", "layernorm_backward", "balance_counts", "balance_gradient" or
             "orthogonalize"
    dtype    "f32", "bf16" or "f16": the type of activations, logits or matrices

    ranks, tokens, width, weights, pad      layer norm: the type of the weights; elements by which a
                                            token's row is longer than its width
    ranks, tokens, experts, top_k, ids, pad, padded
                                            balance: the type of the expert numbers ("i32" or
                                            "i64"); whether tokens are masked (one rank of several
                                            then has none left) and slots are dropped (-1)
    batch, rows, cols                       orthogonalize
"""

import math

import torch

own = False

_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_EPS = 1e-5  # layer norm's
_STEPS = 5
_COEFFICIENTS = (3.4445, -4.7750, 2.0315)  # of the quintic a x + b x^3 + c x^5
_NORM_EPS = 1e-7  # added to a matrix's norm
_BALANCE = 0.01  # the weight of the balance loss


def _norm(name, op, ranks, tokens, width, dtype, weights="f32", pad=0):
    return {"name": name, "op": op, "ranks": ranks, "tokens": tokens, "width": width, "dtype": dtype,
            "weights": weights, "pad": pad}


def _balance(name, op, ranks, tokens, experts, top_k, dtype, ids="i64", pad=0, padded=False):
    return {"name": name, "op": op, "ranks": ranks, "tokens": tokens, "experts": experts,
            "top_k": top_k, "dtype": dtype, "ids": ids, "pad": pad, "padded": padded}


def _matrix(name, batch, rows, cols, dtype):
    return {"name": name, "op": "orthogonalize", "batch": batch, "rows": rows, "cols": cols,
            "dtype": dtype}


def listed():
    return [
        # one token on one rank, as in decoding: all latency
        _norm("norm_fwd_token_bf16", "layernorm_forward", 1, 1, 4096, "bf16", "bf16"),
        # a training step's activations on eight ranks
        _norm("norm_fwd_8x4096_bf16", "layernorm_forward", 8, 4096, 4096, "bf16"),
        # many ranks with few tokens each: the weight gradients weigh as much as the activations
        _norm("norm_bwd_81x16_f32", "layernorm_backward", 81, 16, 768, "f32"),
        # odd sizes, rows that no vector load fits
        _norm("norm_bwd_9x1001_f16", "layernorm_backward", 9, 1001, 2051, "f16", "f16", 2),
        # a wide model's training step; the largest layer norm
        _norm("norm_bwd_8x4096_bf16", "layernorm_backward", 8, 4096, 8192, "bf16"),
        # a small router on nine ranks
        _balance("counts_9x512_f32", "balance_counts", 9, 512, 64, 2, "f32"),
        # a long batch with many experts, part of it padding
        _balance("counts_8x32768_bf16", "balance_counts", 8, 32768, 256, 8, "bf16", "i32", 0, True),
        # ragged sizes, a rank without tokens
        _balance("balance_27x1003_f32", "balance_gradient", 27, 1003, 60, 4, "f32", "i32", 1, True),
        # a long batch with many experts; the largest
        _balance("balance_8x32768_f32", "balance_gradient", 8, 32768, 256, 8, "f32"),
        # a router's weight matrix: all latency
        _matrix("orthogonal_64x256_bf16", 1, 64, 256, "bf16"),
        # several matrices of an odd size, taller than wide
        _matrix("orthogonal_3x770x515_f32", 3, 770, 515, "f32"),
        # a feed-forward layer's weight matrix; the largest
        _matrix("orthogonal_2048x8192_bf16", 1, 2048, 8192, "bf16"),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _ragged(rng, n, step):
    """`n`, half of the time rounded up to whole steps."""
    return -(-n // step) * step if rng.random() < 0.5 else n


def draw(rng):
    op = rng.choice(["layernorm_forward", "layernorm_backward", "balance_counts", "balance_gradient",
                     "orthogonalize"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    if op.startswith("layernorm"):
        width = _ragged(rng, _log(rng, 64, 16384), 64)
        ranks = rng.choice([1, 1, 2, 3, 8, 9, 27, 64, 81, 243])
        tokens = _log(rng, 1, max(1, (1 << 27) // (ranks * width)))
        weights = rng.choice(["f32", dtype])
        c = _norm("", op, ranks, tokens, width, dtype, weights, rng.choice([0, 0, 1, 8]))
    elif op.startswith("balance"):
        experts = rng.choice([8, 16, 32, 64, 128, 256, _log(rng, 6, 512), _log(rng, 6, 512)])
        ranks = rng.choice([1, 1, 2, 3, 8, 9, 27, 64, 81, 243])
        # few experts chosen, of more tokens than one: where all are chosen alike, the gradient is zero
        tokens = _log(rng, 4, (1 << 26) // (ranks * max(experts, 32)))
        top_k = rng.randint(1, max(1, min(8, experts // 4)))
        c = _balance("", op, ranks, tokens, experts, top_k, dtype, rng.choice(["i32", "i64"]),
                     rng.choice([0, 0, 1, 8]), rng.random() < 0.5)
    else:
        rows = _ragged(rng, _log(rng, 16, 4096), 64)
        cols = _ragged(rng, _log(rng, 16, 8192), 64)
        small, large = min(rows, cols), max(rows, cols)
        batch = rng.choice([1, 1, 1, 2, 3, 8])
        while batch * small * small * (3 * large + small) > (1 << 36) + (1 << 34):
            if batch > 1:
                batch -= 1
            else:
                rows, cols = rows * 3 // 4, cols * 3 // 4
                small, large = min(rows, cols), max(rows, cols)
        c = _matrix("", batch, rows, cols, dtype)
    del c["name"]
    return c


# The inputs.


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _rows(shape, pad, dtype):
    """Uninitialised [ranks, tokens, width] rows that lie `pad` elements further apart."""
    ranks, tokens, width = shape
    return torch.empty((ranks, tokens, width + pad), dtype=dtype, device="cuda")[:, :, :width]


def _norm_inputs(case, g):
    dt, wt = _DTYPES[case["dtype"]], _DTYPES[case["weights"]]
    shape = (case["ranks"], case["tokens"], case["width"])
    dev = {"device": "cuda", "generator": g}
    # activations of a residual stream: features of their own offsets and spreads, a few far out
    spread = torch.exp(0.5 * torch.randn(shape[2], **dev))
    spread[torch.rand(shape[2], **dev) < 0.002] *= 20
    x = _rows(shape, case["pad"], dt)
    x.copy_(torch.randn(shape, **dev) * spread + 0.2 * torch.randn(shape[2], **dev))
    s = {"x": x, "gamma": (1 + 0.1 * torch.randn(shape[2], **dev)).to(wt),
         "beta": (0.1 * torch.randn(shape[2], **dev)).to(wt)}
    if case["op"] == "layernorm_backward":
        s["dy"] = _rows(shape, case["pad"], dt).copy_(torch.randn(shape, **dev) * 0.01)
        var, mean = torch.var_mean(x.double(), 2, correction=0)
        s["mean"], s["rstd"] = mean.float(), (var + _EPS).rsqrt().float()
    return s


def _balance_inputs(case, g):
    ranks, tokens, experts, k = case["ranks"], case["tokens"], case["experts"], case["top_k"]
    dev = {"device": "cuda", "generator": g}
    logits = _rows((ranks, tokens, experts), case["pad"], _DTYPES[case["dtype"]])
    # a router that prefers some experts
    logits.copy_(torch.randn((ranks, tokens, experts), **dev) * 1.5 + torch.randn(experts, **dev))
    ids = torch.topk(logits.float(), k, dim=2).indices
    s = {"logits": logits, "mask": None}
    if case["padded"]:
        # sequences that end early, and a rank that got none; slots beyond an expert's capacity
        length = torch.randint(0, tokens + 1, (ranks, 1), **dev)
        length[ranks // 2] = 0 if ranks > 1 else length[ranks // 2]
        s["mask"] = torch.arange(tokens, device="cuda") < length
        ids = ids.masked_fill(torch.rand((ranks, tokens, k), **dev) < 0.05, -1)
        # what lies in the padding is no number
        logits.masked_fill_(~s["mask"].unsqueeze(2), float("nan"))
    s["experts"] = ids.to(torch.int32 if case["ids"] == "i32" else torch.int64).contiguous()
    return s


def _tally(logits, ids, mask):
    """Counts of every expert and of the tokens [ranks, experts + 1], and the sums of probabilities."""
    ranks, _, experts = logits.shape
    live = torch.ones(logits.shape[:2], dtype=torch.bool, device="cuda") if mask is None else mask
    slot = torch.where((ids >= 0) & live.unsqueeze(2), ids, experts).long().flatten(1)
    counts = torch.zeros((ranks, experts + 1), dtype=torch.int32, device="cuda")
    counts.scatter_add_(1, slot, torch.ones_like(slot, dtype=torch.int32))
    counts[:, experts] = live.sum(1)
    f = logits.float().masked_fill(~live.unsqueeze(2), 0.0)
    e = torch.exp(f - f.amax(2, keepdim=True))
    p = e / e.sum(2, keepdim=True) * live.unsqueeze(2)
    return counts, p.sum(1)


def prepare(case, seed):
    g = _generator(seed)
    f32 = {"dtype": torch.float32, "device": "cuda"}
    if case["op"].startswith("layernorm"):
        s = _norm_inputs(case, g)
        ranks, tokens, width = s["x"].shape
        if case["op"] == "layernorm_forward":
            s["y"] = torch.empty_like(s["x"], memory_format=torch.contiguous_format)
            s["mean"], s["rstd"] = torch.empty((ranks, tokens), **f32), torch.empty((ranks, tokens), **f32)
        else:
            s["dx"] = torch.empty_like(s["x"], memory_format=torch.contiguous_format)
            # each rank's row of the vector to sum holds both gradients
            rows = torch.empty((ranks, 2 * width), **f32)
            s["dgamma"], s["dbeta"] = rows[:, :width], rows[:, width:]
    elif case["op"].startswith("balance"):
        s = _balance_inputs(case, g)
        ranks, _, experts = s["logits"].shape
        if case["op"] == "balance_counts":
            s["counts"] = torch.empty((ranks, experts + 1), dtype=torch.int32, device="cuda")
            s["probs"] = torch.empty((ranks, experts), **f32)
        else:
            # every rank holds the sums over all ranks
            counts, probs = _tally(s["logits"], s["experts"], s["mask"])
            s["counts"] = counts.sum(0, dtype=torch.int32).expand(ranks, -1).contiguous()
            s["probs"] = probs.sum(0).expand(ranks, -1).contiguous()
            s["loss"] = torch.empty(ranks, **f32)
            # the gradient of the loss: one, or in 16 bits of little range a factor that keeps the
            # gradients of a mean over many tokens in that range
            s["dloss"] = None
            if case["dtype"] == "f16":
                tokens = ranks * case["tokens"]
                s["dloss"] = torch.full((ranks,), 64.0 * 2 ** math.ceil(math.log2(tokens)), **f32)
            s["dlogits"] = torch.empty_like(s["logits"], memory_format=torch.contiguous_format)
    else:
        dev = {"device": "cuda", "generator": g}
        b, m, n = case["batch"], case["rows"], case["cols"]
        # a gradient: a few strong directions whose strengths fall off, and noise
        r = max(1, min(m, n) // 8)
        u = torch.randn((b, m, r), **dev) / torch.arange(1, r + 1, **f32).sqrt()
        x = u @ torch.randn((b, r, n), **dev) + 0.3 * torch.randn((b, m, n), **dev)
        s = {"x": (1e-3 * x).to(_DTYPES[case["dtype"]])}
        s["out"] = torch.empty_like(s["x"])
    s["case"] = case
    return s


# The plain forms: elementary operations in 32 bits, rounded once at the end.


def _plain_layernorm_forward(s):
    x = s["x"].float()
    mean = x.mean(2)
    d = x - mean.unsqueeze(2)
    rstd = 1 / torch.sqrt((d * d).mean(2) + _EPS)
    y = d * rstd.unsqueeze(2) * s["gamma"].float() + s["beta"].float()
    return {"y": y.to(s["x"].dtype), "mean": mean, "rstd": rstd}


def _plain_layernorm_backward(s):
    dy, rstd = s["dy"].float(), s["rstd"].unsqueeze(2)
    h = (s["x"].float() - s["mean"].unsqueeze(2)) * rstd
    g = dy * s["gamma"].float()
    dx = rstd * (g - g.mean(2, keepdim=True) - h * (g * h).mean(2, keepdim=True))
    return {"dx": dx.to(s["x"].dtype), "dgamma": (dy * h).sum(1), "dbeta": dy.sum(1)}


def _plain_balance_counts(s):
    counts, probs = _tally(s["logits"], s["experts"], s["mask"])
    return {"counts": counts, "probs": probs}


def _plain_balance_gradient(s):
    experts, k = s["logits"].shape[2], s["case"]["top_k"]
    n = s["counts"][:, experts:].float().clamp(min=1)
    share = s["counts"][:, :experts].float() / (k * n)
    loss = _BALANCE * experts * (share * (s["probs"] / n)).sum(1)
    w = _BALANCE * experts * share / n
    w = (w if s["dloss"] is None else w * s["dloss"].unsqueeze(1)).unsqueeze(1)
    f = s["logits"].float()
    if s["mask"] is not None:
        f = f.masked_fill(~s["mask"].unsqueeze(2), 0.0)
    e = torch.exp(f - f.amax(2, keepdim=True))
    p = e / e.sum(2, keepdim=True)
    d = p * (w - (p * w).sum(2, keepdim=True))
    if s["mask"] is not None:
        d = d * s["mask"].unsqueeze(2)
    return {"loss": loss, "dlogits": d.to(s["logits"].dtype)}


def _plain_orthogonalize(s):
    x = s["x"].float()
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2).contiguous()
    x = x / (torch.sqrt((x * x).sum((1, 2), keepdim=True)) + _NORM_EPS)
    a, b, c = _COEFFICIENTS
    for _ in range(_STEPS):
        q = x @ x.transpose(1, 2)
        x = a * x + (b * q + c * (q @ q)) @ x
    if tall:
        x = x.transpose(1, 2)
    return x.to(s["x"].dtype)


# The framework's calls. A program keeps each workspace with its buffers.


def _own_layernorm_forward(s, T):
    T.trivance_layernorm_forward(s["x"], s["gamma"], s["beta"], s["y"], s["mean"], s["rstd"], _EPS)
    return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}


def _own_layernorm_backward(s, T):
    if "workspace" not in s:
        s["workspace"] = _workspace(T.trivance_layernorm_workspace_bytes(*s["x"].shape))
    T.trivance_layernorm_backward(s["dy"], s["x"], s["gamma"], s["mean"], s["rstd"], s["dx"],
                                  s["dgamma"], s["dbeta"], s["workspace"])
    return {"dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}


def _own_balance_counts(s, T):
    if "workspace" not in s:
        s["workspace"] = _workspace(T.trivance_balance_workspace_bytes(*s["logits"].shape))
    T.trivance_balance_counts(s["logits"], s["experts"], s["counts"], s["probs"], s["workspace"],
                              s["mask"])
    return {"counts": s["counts"], "probs": s["probs"]}


def _own_balance_gradient(s, T):
    k = s["case"]["top_k"]
    T.trivance_balance_loss(s["counts"], s["probs"], k, s["loss"], _BALANCE)
    T.trivance_balance_backward(s["logits"], s["counts"], k, s["dlogits"], s["mask"], _BALANCE,
                                s["dloss"])
    return {"loss": s["loss"], "dlogits": s["dlogits"]}


def _own_orthogonalize(s, T):
    if "workspace" not in s:
        s["workspace"] = _workspace(T.trivance_orthogonalize_workspace_bytes(*s["x"].shape))
    T.trivance_orthogonalize(s["x"], s["out"], s["workspace"], [_COEFFICIENTS] * _STEPS, 1.0, _NORM_EPS)
    return s["out"]


def _workspace(nbytes):
    return torch.empty(nbytes, dtype=torch.uint8, device="cuda")


_PLAIN = {"layernorm_forward": _plain_layernorm_forward,
          "layernorm_backward": _plain_layernorm_backward, "balance_counts": _plain_balance_counts,
          "balance_gradient": _plain_balance_gradient, "orthogonalize": _plain_orthogonalize}
_OWN = {"layernorm_forward": _own_layernorm_forward, "layernorm_backward": _own_layernorm_backward,
        "balance_counts": _own_balance_counts, "balance_gradient": _own_balance_gradient,
        "orthogonalize": _own_orthogonalize}


def run(state):
    if own:
        import paper_2602_17254_amd as T

        return _OWN[state["case"]["op"]](state, T)
    return _PLAIN[state["case"]["op"]](state)


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["op"].startswith("layernorm"):
        ranks, tokens, width = case["ranks"], case["tokens"], case["width"]
        n, wsize = ranks * tokens * width, 4 if case["weights"] == "f32" else 2
        if case["op"] == "layernorm_forward":
            return {"bytes": 2 * n * size + 2 * width * wsize + 8 * ranks * tokens, "flops": 8 * n}
        return {"bytes": 3 * n * size + width * wsize + 8 * ranks * (tokens + width), "flops": 14 * n}
    if case["op"].startswith("balance"):
        ranks, tokens, experts = case["ranks"], case["tokens"], case["experts"]
        n, mask = ranks * tokens * experts, ranks * tokens * case["padded"]
        if case["op"] == "balance_counts":
            slots = ranks * tokens * case["top_k"] * (4 if case["ids"] == "i32" else 8)
            return {"bytes": n * size + slots + mask + 4 * ranks * (2 * experts + 1), "flops": 5 * n}
        return {"bytes": 2 * n * size + mask + 4 * ranks * (2 * experts + 2), "flops": 8 * n}
    b, m, n = case["batch"], case["rows"], case["cols"]
    small = min(m, n)
    # two symmetric products, of which half is computed, and a full one
    flops = _STEPS * b * (small * m * n + small ** 3 + 2 * small * m * n)
    return {"bytes": 2 * b * m * n * size, "flops": flops}


# The operators' definitions in 64 bits.


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "layernorm_forward":
        x = s["x"].double()
        var, mean = torch.var_mean(x, 2, correction=0)
        y = torch.nn.functional.layer_norm(x, x.shape[2:], s["gamma"].double(), s["beta"].double(), _EPS)
        return {"y": y, "mean": mean, "rstd": (var + _EPS).rsqrt()}
    if case["op"] == "layernorm_backward":
        dx = torch.empty(s["x"].shape, dtype=torch.float64, device="cuda")
        dgamma = torch.empty(s["dgamma"].shape, dtype=torch.float64, device="cuda")
        dbeta = torch.empty_like(dgamma)
        gamma, width = s["gamma"].double(), case["width"]
        for r in range(case["ranks"]):
            dy = s["dy"][r].double()
            rstd = s["rstd"][r].double()
            h = torch.addcmul(-(s["mean"][r].double() * rstd)[:, None], s["x"][r].double(), rstd[:, None])
            # the gradient through y = gamma h + beta: what lies along 1 and along h is taken out
            along_one = dy @ gamma / width
            along_h = (dy * h) @ gamma / width
            dx[r] = (dy * gamma - torch.stack((along_one, along_h), 1).unsqueeze(1).matmul(
                torch.stack((torch.ones_like(h), h), 1)).squeeze(1)) * rstd[:, None]
            dgamma[r] = torch.sum(torch.mul(dy, h), 0)
            dbeta[r] = torch.sum(dy, 0)
        return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    if case["op"].startswith("balance"):
        ranks, tokens, experts = s["logits"].shape
        live = torch.ones((ranks, tokens), dtype=torch.bool, device="cuda") if s["mask"] is None else s["mask"]
        if case["op"] == "balance_counts":
            counts = torch.zeros((ranks, experts + 1), dtype=torch.int32, device="cuda")
            probs = torch.zeros((ranks, experts), dtype=torch.float64, device="cuda")
            for r in range(ranks):
                ids = s["experts"][r][live[r]].flatten().long()
                counts[r, :experts] = torch.bincount(ids[ids >= 0], minlength=experts)
                counts[r, experts] = int(live[r].sum())
                probs[r] = torch.softmax(s["logits"][r][live[r]].double(), 1).sum(0)
            return {"counts": counts, "probs": probs}
        c = s["counts"].double()
        n = c[:, experts].clamp(min=1)
        w = c[:, :experts] * (_BALANCE * experts / case["top_k"]) / n[:, None] ** 2
        loss = torch.einsum("re,re->r", w, s["probs"].double())
        if s["dloss"] is not None:
            w = w * s["dloss"].double()[:, None]
        d = torch.zeros((ranks, tokens, experts), dtype=torch.float64, device="cuda")
        for r in range(ranks):
            p = torch.softmax(s["logits"][r][live[r]].double(), 1)
            d[r][live[r]] = p * w[r] - p * (p @ w[r])[:, None]
        return {"loss": loss, "dlogits": d}
    a, b, c = _COEFFICIENTS
    out = torch.empty(s["x"].shape, dtype=torch.float64, device="cuda")
    for i in range(case["batch"]):
        x = s["x"][i].double()
        x /= torch.linalg.matrix_norm(x) + _NORM_EPS
        for _ in range(_STEPS):
            # x (a + b g + c g^2) with g the smaller of the two Gram matrices, by Horner's rule
            g = x.T @ x if x.shape[0] > x.shape[1] else x @ x.T
            p = c * g
            p.diagonal().add_(b)
            p = p @ g
            p.diagonal().add_(a)
            x = x @ p if x.shape[0] > x.shape[1] else p @ x
        out[i] = x
    return out
