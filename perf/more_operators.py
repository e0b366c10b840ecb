"""More operators of a data-parallel training step: a root-mean-square norm with the residual's addition,
tokens sorted by expert and back, an embedding and dropout, with their inputs, plain forms and exact results.

Activations are rows [ranks][tokens][width], one rank's after another's, as the framework's other operators
have them; what the AllReduce sums, the gradients of the norm's weights and of the embedding's table, is
written straight into one row of memory per rank. The fields of a case:

    op       "rmsnorm", "experts", "embedding" or "dropout"
    step     which of its passes: "forward" or "backward"; of "experts" "dispatch" (sort the slots by
             expert, copy the tokens into that order), "combine" (weighted sums back) or "gradient" (of
             those sums)
    dtype    "f32", "bf16" or "f16": the type of activations
    ranks, tokens, width, pad
             pad: elements by which a token's row is longer than its width

    weights, residual, out8
             rmsnorm: the type of the weights; whether a residual is added (forward) or another gradient of
             the sum arrives (backward); whether the result is held in 8 bits with a scale for each token
    experts, top_k, ids, dropped
             experts: the type of the expert numbers ("i32" or "i64"); whether slots are empty (-1) and
             tokens masked (one rank of several then has none left)
    vocab, table, ids, dropped
             embedding: the type of the table; whether positions are padding (-1)
    residual, rate
             dropout: whether the result is added to a residual; the share that is dropped
"""

import math

import torch

own = False

_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_EPS = 1e-5
_LARGEST_8 = 448.0  # of a number of 8 bits, four of them exponent
_SMALLEST_SCALE = 2.0 ** -126
_WORD = (1 << 32) - 1


def _norm(name, step, ranks, tokens, width, dtype, weights="f32", pad=0, residual=True, out8=False):
    return {"name": name, "op": "rmsnorm", "step": step, "ranks": ranks, "tokens": tokens, "width": width,
            "dtype": dtype, "weights": weights, "pad": pad, "residual": residual, "out8": out8}


def _experts(name, step, ranks, tokens, width, experts, top_k, dtype, ids="i64", pad=0, dropped=False):
    return {"name": name, "op": "experts", "step": step, "ranks": ranks, "tokens": tokens, "width": width,
            "experts": experts, "top_k": top_k, "dtype": dtype, "ids": ids, "pad": pad, "dropped": dropped}


def _embedding(name, step, ranks, tokens, vocab, width, dtype, table="f32", ids="i64", dropped=False):
    return {"name": name, "op": "embedding", "step": step, "ranks": ranks, "tokens": tokens, "vocab": vocab,
            "width": width, "dtype": dtype, "table": table, "ids": ids, "dropped": dropped}


def _dropout(name, ranks, tokens, width, dtype, rate, pad=0, residual=False):
    return {"name": name, "op": "dropout", "ranks": ranks, "tokens": tokens, "width": width,
            "dtype": dtype, "rate": rate, "pad": pad, "residual": residual}


def listed():
    return [
        # one token on one rank, as in decoding: all latency
        _norm("rms_fwd_token_bf16", "forward", 1, 1, 4096, "bf16", "bf16"),
        # a training step's activations on eight ranks, the result for a product in 8 bits
        _norm("rms_fwd_8x4096_out8", "forward", 8, 4096, 4096, "bf16", out8=True),
        # odd sizes, rows that no vector load fits, no residual
        _norm("rms_bwd_9x777_f16", "backward", 9, 777, 1283, "f16", "f16", 2, False),
        # a wide model's training step
        _norm("rms_bwd_8x4096_bf16", "backward", 8, 4096, 8192, "bf16"),
        # a few sequences of a small model on nine ranks
        _experts("dispatch_9x128_f32", "dispatch", 9, 128, 768, 64, 2, "f32"),
        # a long batch with many experts; the most bytes of all
        _experts("dispatch_8x16384_bf16", "dispatch", 8, 16384, 2048, 256, 8, "bf16", "i32"),
        # ragged sizes, empty slots, a rank without tokens
        _experts("combine_27x1003_f16", "combine", 27, 1003, 515, 60, 4, "f16", "i32", 1, True),
        # the way back through the sums of a long batch
        _experts("gradient_8x8192_bf16", "gradient", 8, 8192, 2048, 64, 4, "bf16"),
        # tokens of a training step from a table in 32 bits
        _embedding("lookup_8x4096_bf16", "forward", 8, 4096, 32000, 2048, "bf16", ids="i32", dropped=True),
        # and their gradient, into each rank's row of the vector to sum
        _embedding("table_grad_8x8192_bf16", "backward", 8, 8192, 32000, 1024, "bf16"),
        # a small model's activations
        _dropout("dropout_9x256_f32", 9, 256, 515, "f32", 0.1),
        # a wide model's, added to its residual
        _dropout("dropout_8x4096_bf16", 8, 4096, 8192, "bf16", 0.1, residual=True),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(max(low, high))))))


def _ragged(rng, n, step):
    """`n`, half of the time rounded up to whole steps."""
    return -(-n // step) * step if rng.random() < 0.5 else n


def draw(rng):
    op = rng.choice(["rmsnorm", "rmsnorm", "experts", "experts", "embedding", "dropout"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    ranks = rng.choice([1, 1, 2, 3, 8, 9, 27, 81, 243])
    pad = rng.choice([0, 0, 1, 8])
    ids = rng.choice(["i32", "i64"])
    dropped = rng.random() < 0.5
    if op == "rmsnorm":
        width = _ragged(rng, _log(rng, 64, 16384), 64)
        tokens = _log(rng, 1, (1 << 27) // (ranks * width))
        step = rng.choice(["forward", "backward"])
        c = _norm("", step, ranks, tokens, width, dtype, rng.choice(["f32", dtype]), pad, rng.random() < 0.7,
                  step == "forward" and rng.random() < 0.4)
    elif op == "experts":
        experts = rng.choice([8, 16, 64, 256, _log(rng, 4, 512)])
        top_k = rng.randint(1, min(8, experts))
        width = _ragged(rng, _log(rng, 32, 8192), 64)
        # a router's scores for all experts are made with the inputs
        tokens = _log(rng, 1, (1 << 27) // (ranks * max(width * top_k, 2 * experts)))
        c = _experts("", rng.choice(["dispatch", "combine", "gradient"]), ranks, tokens, width, experts, top_k,
                     dtype, ids, pad, dropped)
    elif op == "embedding":
        vocab = _log(rng, 100, 130000)
        width = _ragged(rng, _log(rng, 32, 8192), 64)
        width = min(width, (1 << 27) // vocab)
        if rng.random() < 0.5:
            c = _embedding("", "forward", ranks, _log(rng, 1, (1 << 26) // (ranks * width)), vocab, width, dtype,
                           rng.choice(["f32", dtype]), ids, dropped)
        else:
            ranks = min(ranks, max(1, (1 << 28) // (vocab * width)))
            c = _embedding("", "backward", ranks, _log(rng, 1, (1 << 26) // (ranks * width)), vocab, width, dtype,
                           "f32", ids, dropped)
    else:
        width = _ragged(rng, _log(rng, 64, 16384), 64)
        tokens = _log(rng, 1, (1 << 27) // (ranks * width))
        c = _dropout("", ranks, tokens, width, dtype, rng.choice([0.02, 0.1, 0.25, 0.5]), pad, rng.random() < 0.5)
    del c["name"]
    return c


# The inputs.


def _rows(shape, pad, dtype):
    """Uninitialised [ranks, tokens, width] rows that lie `pad` elements further apart."""
    ranks, tokens, width = shape
    return torch.empty((ranks, tokens, width + pad), dtype=dtype, device="cuda")[:, :, :width]


def _activations(case, dev, spread=1.0):
    shape = (case["ranks"], case["tokens"], case["width"])
    x = _rows(shape, case.get("pad", 0), _DTYPES[case["dtype"]])
    return x.copy_(torch.randn(shape, **dev) * spread)


def _norm_inputs(case, dev):
    width, f32 = case["width"], {"dtype": torch.float32, "device": "cuda"}
    # a residual stream: features of their own spreads, a few far out
    spread = torch.exp(0.5 * torch.randn(width, **dev))
    spread[torch.rand(width, **dev) < 0.002] *= 20
    shape = (case["ranks"], case["tokens"], width)
    s = {"gamma": (1 + 0.1 * torch.randn(width, **dev)).to(_DTYPES[case["weights"]]), "residual": None,
         "total": None, "scales": None, "dtotal": None}
    if case["step"] == "forward":
        s["x"] = _activations(case, dev, 0.3 if case["residual"] else spread)
        s["rstd"] = torch.empty(shape[:2], **f32)
        s["y"] = torch.empty(shape, dtype=torch.float8_e4m3fn if case["out8"] else s["x"].dtype, device="cuda")
        if case["residual"]:
            s["residual"] = _activations(case, dev, spread)
            s["total"] = torch.empty(shape, dtype=s["x"].dtype, device="cuda")
        if case["out8"]:
            s["scales"] = torch.empty(shape[:2], **f32)
    else:
        s["total"] = _activations(case, dev, spread)
        s["rstd"] = (s["total"].double().square().mean(2) + _EPS).rsqrt().float()
        s["dy"] = _activations(case, dev, 0.01)
        if case["residual"]:
            s["dtotal"] = _activations(case, dev, 0.01)
        s["dx"] = torch.empty(shape, dtype=s["dy"].dtype, device="cuda")
        # each rank's row of the vector to sum holds other gradients too
        s["dgamma"] = torch.empty((case["ranks"], 2 * width), **f32)[:, width:]
    return s


def _experts_inputs(case, dev):
    ranks, tokens, width, k = case["ranks"], case["tokens"], case["width"], case["top_k"]
    # a router that prefers some experts
    scores = torch.randn((ranks, tokens, case["experts"]), **dev) * 1.5 + torch.randn(case["experts"], **dev)
    best, ids = torch.topk(scores, k, dim=2)
    s = {"weights": torch.softmax(best, 2), "mask": None}
    if case["dropped"]:
        # sequences that end early, and a rank that got none; slots beyond an expert's capacity
        length = torch.randint(0, tokens + 1, (ranks, 1), **dev)
        length[ranks // 2] = 0 if ranks > 1 else length[ranks // 2]
        s["mask"] = torch.arange(tokens, device="cuda") < length
        ids = ids.masked_fill(torch.rand((ranks, tokens, k), **dev) < 0.05, -1)
    s["chosen"] = ids.to(torch.int32 if case["ids"] == "i32" else torch.int64).contiguous()
    sorted_shape, dt = (ranks, tokens * k, width), _DTYPES[case["dtype"]]
    if case["step"] == "dispatch":
        s["x"] = _activations(case, dev)
        # rows behind a rank's last stay as they are
        s["rows"] = torch.zeros(sorted_shape, dtype=dt, device="cuda")
        s["offsets"] = torch.empty((ranks, case["experts"] + 1), dtype=torch.int32, device="cuda")
        s["places"] = torch.empty((ranks, tokens, k), dtype=torch.int32, device="cuda")
        return s
    s["places"] = _plain_sort(s["chosen"], s["mask"], case["experts"])[2]
    s["rows"] = _rows(sorted_shape, case["pad"], dt).copy_(torch.randn(sorted_shape, **dev))
    if case["step"] == "combine":
        s["y"] = torch.empty((ranks, tokens, width), dtype=dt, device="cuda")
    else:
        s["dy"] = _activations(case, dev, 0.01)
        s["drows"] = torch.zeros(sorted_shape, dtype=dt, device="cuda")
        s["dweights"] = torch.empty_like(s["weights"])
    return s


def _embedding_inputs(case, dev):
    ranks, tokens, vocab, width = case["ranks"], case["tokens"], case["vocab"], case["width"]
    # the n-th most frequent number is n times rarer than the first
    ids = (vocab ** torch.rand((ranks, tokens), dtype=torch.float64, **dev)).long() - 1
    if case["dropped"]:
        ids[torch.rand((ranks, tokens), **dev) < 0.1] = -1
    s = {"ids": ids.clamp(max=vocab - 1).to(torch.int32 if case["ids"] == "i32" else torch.int64),
         "scale": math.sqrt(width)}
    if case["step"] == "forward":
        s["table"] = (0.02 * torch.randn((vocab, width), **dev)).to(_DTYPES[case["table"]])
        s["y"] = torch.empty((ranks, tokens, width), dtype=_DTYPES[case["dtype"]], device="cuda")
    else:
        s["dy"] = _activations(case, dev, 0.01)
        s["dtable"] = torch.empty((ranks, vocab, width), dtype=torch.float32, device="cuda")
    return s


def _dropout_inputs(case, dev):
    s = {"x": _activations(case, dev), "residual": _activations(case, dev) if case["residual"] else None}
    s["y"] = torch.empty(s["x"].shape, dtype=s["x"].dtype, device="cuda")
    # the seed and the number of the call, which a program counts up
    s["state"] = torch.randint(-(1 << 62), 1 << 62, (2,), **dev)
    s["state"][1] &= _WORD
    return s


_INPUTS = {"rmsnorm": _norm_inputs, "experts": _experts_inputs, "embedding": _embedding_inputs,
           "dropout": _dropout_inputs}


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return {**_INPUTS[case["op"]](case, {"device": "cuda", "generator": g}), "case": case}


# The plain forms: elementary operations in 32 bits, rounded once at the end.


def _plain_norm_forward(s):
    total = s["x"].float() if s["residual"] is None else s["x"].float() + s["residual"].float()
    rstd = 1 / torch.sqrt((total * total).mean(2) + _EPS)
    y = total * rstd.unsqueeze(2) * s["gamma"].float()
    out = {"rstd": rstd}
    if s["total"] is not None:
        out["total"] = total.to(s["x"].dtype)
    if s["scales"] is None:
        return {**out, "y": y.to(s["x"].dtype)}
    scales = (y.abs().amax(2) / _LARGEST_8).clamp(min=_SMALLEST_SCALE)
    y = (y / scales.unsqueeze(2)).clamp(-_LARGEST_8, _LARGEST_8)
    return {**out, "y": y.to(torch.float8_e4m3fn), "scales": scales}


def _plain_norm_backward(s):
    rstd, dy = s["rstd"].unsqueeze(2), s["dy"].float()
    h = s["total"].float() * rstd
    g = dy * s["gamma"].float()
    dx = rstd * (g - h * (g * h).mean(2, keepdim=True))
    if s["dtotal"] is not None:
        dx = dx + s["dtotal"].float()
    return {"dx": dx.to(s["dy"].dtype), "dgamma": (dy * h).sum(1)}


def _plain_sort(chosen, mask, experts):
    """First row of each expert and the number of rows [ranks, experts + 1], the slots in the order of
    their experts [ranks, tokens * top_k], and each slot's row, -1 for none [ranks, tokens, top_k]."""
    ranks, tokens, k = chosen.shape
    used = (chosen >= 0) & (chosen < experts)
    if mask is not None:
        used = used & mask.unsqueeze(2)
    key = torch.where(used, chosen, experts).long().flatten(1)
    counts = torch.zeros((ranks, experts + 1), dtype=torch.int64, device="cuda")
    counts.scatter_add_(1, key, torch.ones_like(key))
    offsets = counts.cumsum(1) - counts
    order = torch.sort(key, dim=1, stable=True).indices
    row = torch.arange(tokens * k, device="cuda").expand(ranks, -1)
    places = torch.empty_like(order).scatter_(1, order, row).view(ranks, tokens, k)
    return offsets.int(), order, torch.where(used, places, -1).int()


def _plain_dispatch(s):
    x, k = s["x"], s["case"]["top_k"]
    offsets, order, places = _plain_sort(s["chosen"], s["mask"], s["case"]["experts"])
    rank = torch.arange(x.shape[0], device="cuda").unsqueeze(1)
    live = torch.arange(order.shape[1], device="cuda") < offsets[:, -1:]
    rows = x[rank, order // k].masked_fill(~live.unsqueeze(2), 0.0)
    return {"rows": rows, "offsets": offsets, "places": places}


def _picked(rows, places):
    """Every slot's row [ranks, tokens, top_k, width] in 32 bits, and which slots have one."""
    rank = torch.arange(rows.shape[0], device="cuda").view(-1, 1, 1)
    return rows[rank, places.clamp(min=0).long()].float(), (places >= 0).unsqueeze(3)


def _plain_combine(s):
    rows, live = _picked(s["rows"], s["places"])
    y = torch.where(live, rows * s["weights"].unsqueeze(3), 0.0).sum(2)
    return {"y": y.to(s["rows"].dtype)}


def _plain_gradient(s):
    rows, live = _picked(s["rows"], s["places"])
    ranks, tokens, k, width = rows.shape
    dy = s["dy"].float().unsqueeze(2)
    dweights = torch.where(live, rows * dy, 0.0).sum(3)
    drows = torch.zeros((ranks, tokens * k + 1, width), device="cuda")  # the last row takes the empty slots'
    to = torch.where(s["places"] >= 0, s["places"], tokens * k).long()
    drows[torch.arange(ranks, device="cuda").view(-1, 1, 1), to] = dy * s["weights"].unsqueeze(3)
    return {"drows": drows[:, :-1].to(s["dy"].dtype), "dweights": dweights}


def _plain_lookup(s):
    live = (s["ids"] >= 0).unsqueeze(2)
    y = s["table"][s["ids"].clamp(min=0).long()].float() * s["scale"]
    return {"y": torch.where(live, y, 0.0).to(s["y"].dtype)}


def _plain_table_gradient(s):
    ranks, vocab, width = s["dtable"].shape
    rank = torch.arange(ranks, device="cuda").unsqueeze(1)
    to = torch.where(s["ids"] >= 0, rank * vocab + s["ids"], ranks * vocab).long()
    d = torch.zeros((ranks * vocab + 1, width), device="cuda")  # the last row takes the padding's
    d.index_add_(0, to.flatten(), s["dy"].float().flatten(0, 1))
    return {"dtable": (d[:-1] * s["scale"]).view(ranks, vocab, width)}


def _times(a, m):
    """High and low words of the products of the words `a` and the constant word `m`."""
    low, high = a * (m & 0xFFFF), a * (m >> 16)
    low = low + ((high & 0xFFFF) << 16)
    return (low >> 32) + (high >> 16), low & _WORD


def _random_words(state, ranks, tokens, blocks):
    """Ten rounds of Philox-4x32 (Salmon, Moraes, Dror, Shaw 2011) on the counters (block, token, rank,
    call) with the seed as key: four words for each block of each token."""
    k0, k1 = state[0] & _WORD, (state[0] >> 32) & _WORD
    shape = (ranks, tokens, blocks)
    c0 = torch.arange(blocks, device="cuda").expand(shape)
    c1 = torch.arange(tokens, device="cuda").view(1, -1, 1).expand(shape)
    c2 = torch.arange(ranks, device="cuda").view(-1, 1, 1).expand(shape)
    c3 = (state[1] & _WORD).expand(shape)
    for _ in range(10):
        h0, l0 = _times(c0, 0xD2511F53)
        h1, l1 = _times(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & _WORD, (k1 + 0xBB67AE85) & _WORD
    return torch.stack((c0, c1, c2, c3), 3)


def _threshold(case):
    """The rate in units of 2^-16."""
    return round(case["rate"] * 65536)


def _plain_dropout(s):
    ranks, tokens, width = s["x"].shape
    words = _random_words(s["state"], ranks, tokens, (width + 7) // 8)
    # eight values from each block, low half of a word first
    halves = torch.stack((words & 0xFFFF, words >> 16), 4).flatten(2)[:, :, :width]
    limit = _threshold(s["case"])
    y = torch.where(halves >= limit, s["x"].float() * (65536 / (65536 - limit)), 0.0)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return {"y": y.to(s["x"].dtype)}


# The framework's calls. A program keeps each workspace with its buffers.


def _workspace(s, nbytes):
    if "workspace" not in s:
        s["workspace"] = torch.empty(nbytes(), dtype=torch.uint8, device="cuda")
    return s["workspace"]


def _own_norm_forward(s, T):
    T.trivance_rmsnorm_forward(s["x"], s["gamma"], s["y"], s["rstd"], s["residual"], s["total"], s["scales"], _EPS)
    out = {"rstd": s["rstd"], "total": s["total"], "y": s["y"], "scales": s["scales"]}
    return {name: t for name, t in out.items() if t is not None}


def _own_norm_backward(s, T):
    work = _workspace(s, lambda: T.trivance_rmsnorm_workspace_bytes(*s["dy"].shape))
    T.trivance_rmsnorm_backward(s["dy"], s["total"], s["gamma"], s["rstd"], s["dx"], s["dgamma"], work, s["dtotal"])
    return {"dx": s["dx"], "dgamma": s["dgamma"]}


def _own_dispatch(s, T):
    work = _workspace(s, lambda: T.trivance_experts_workspace_bytes(*s["chosen"].shape, s["case"]["experts"]))
    T.trivance_experts_sort(s["chosen"], s["offsets"], s["places"], work, s["mask"])
    T.trivance_experts_dispatch(s["x"], s["places"], s["rows"])
    return {"rows": s["rows"], "offsets": s["offsets"], "places": s["places"]}


def _own_combine(s, T):
    T.trivance_experts_combine(s["rows"], s["places"], s["y"], s["weights"])
    return {"y": s["y"]}


def _own_gradient(s, T):
    T.trivance_experts_combine_backward(s["dy"], s["rows"], s["places"], s["weights"], s["drows"], s["dweights"])
    return {"drows": s["drows"], "dweights": s["dweights"]}


def _own_lookup(s, T):
    T.trivance_embedding_forward(s["ids"], s["table"], s["y"], s["scale"])
    return {"y": s["y"]}


def _own_table_gradient(s, T):
    work = _workspace(s, lambda: T.trivance_embedding_workspace_bytes(*s["dy"].shape, s["case"]["vocab"]))
    T.trivance_embedding_backward(s["dy"], s["ids"], s["dtable"], work, s["scale"])
    return {"dtable": s["dtable"]}


def _own_dropout(s, T):
    T.trivance_dropout(s["x"], s["y"], s["state"], s["case"]["rate"], s["residual"])
    return {"y": s["y"]}


_PLAIN = {("rmsnorm", "forward"): _plain_norm_forward, ("rmsnorm", "backward"): _plain_norm_backward,
          ("experts", "dispatch"): _plain_dispatch, ("experts", "combine"): _plain_combine,
          ("experts", "gradient"): _plain_gradient, ("embedding", "forward"): _plain_lookup,
          ("embedding", "backward"): _plain_table_gradient, ("dropout", None): _plain_dropout}
_OWN = {("rmsnorm", "forward"): _own_norm_forward, ("rmsnorm", "backward"): _own_norm_backward,
        ("experts", "dispatch"): _own_dispatch, ("experts", "combine"): _own_combine,
        ("experts", "gradient"): _own_gradient, ("embedding", "forward"): _own_lookup,
        ("embedding", "backward"): _own_table_gradient, ("dropout", None): _own_dropout}


def run(state):
    which = state["case"]["op"], state["case"].get("step")
    if own:
        import paper_2602_17254_amd as T

        return _OWN[which](state, T)
    return _PLAIN[which](state)


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    ranks, tokens, width = case["ranks"], case["tokens"], case["width"]
    t = ranks * tokens
    n = t * width
    id_size = 4 if case.get("ids") == "i32" else 8
    if case["op"] == "rmsnorm":
        weights = width * (4 if case["weights"] == "f32" else 2)
        if case["step"] == "forward":
            read = n * size * (2 if case["residual"] else 1) + weights
            written = n * (1 if case["out8"] else size) + 4 * t * (2 if case["out8"] else 1)
            return {"bytes": read + written + (n * size if case["residual"] else 0), "flops": (6 if case["out8"] else 5) * n}
        return {"bytes": n * size * (4 if case["residual"] else 3) + weights + 4 * t + 4 * ranks * width,
                "flops": 10 * n}
    if case["op"] == "experts":
        slots = t * case["top_k"]
        # of `dropped` cases about half of the tokens and 95 slots in 100 of those are in use
        used = 0.475 if case["dropped"] else 1.0
        tokens_used = 0.5 if case["dropped"] else 1.0
        rows = used * slots * width * size
        if case["step"] == "dispatch":
            index = slots * (id_size + 4) + 4 * ranks * (case["experts"] + 1) + (t if case["dropped"] else 0)
            return {"bytes": int(tokens_used * n * size + rows) + index, "flops": 0}
        if case["step"] == "combine":
            return {"bytes": int(rows + used * 4 * slots) + 4 * slots + n * size, "flops": int(2 * used * slots * width)}
        return {"bytes": int(2 * rows + tokens_used * n * size + used * 4 * slots) + 8 * slots,
                "flops": int(3 * used * slots * width)}
    if case["op"] == "embedding":
        if case["step"] == "forward":
            # rows of the table that are wanted twice are read once: of ids of that distribution the
            # expected number of different ones
            each = 4 if case["table"] == "f32" else 2
            rows = min(t, int(_distinct(case["vocab"], t * (0.9 if case["dropped"] else 1.0))))
            return {"bytes": rows * width * each + n * size + t * id_size, "flops": n}
        live = 0.9 if case["dropped"] else 1.0
        return {"bytes": int(live * n * size) + t * id_size + 4 * ranks * case["vocab"] * width, "flops": 2 * n}
    return {"bytes": n * size * (3 if case["residual"] else 2) + 16, "flops": 2 * n}


def _distinct(vocab, drawn):
    """The expected number of different ones among `drawn` numbers of which n turns up in proportion to
    log((n + 1) / n)."""
    n = torch.arange(1, vocab, dtype=torch.float64)
    share = torch.log1p(1 / n) / math.log(vocab)
    return float((1 - torch.exp(drawn * torch.log1p(-share.clamp(max=1 - 1e-12)))).sum())


# The operators' definitions in 64 bits.


def _exact_norm(s, case):
    if case["step"] == "forward":
        total = s["x"].double()
        if case["residual"]:
            total += s["residual"].double()
        rstd = (torch.linalg.vector_norm(total, dim=2).square() / case["width"] + _EPS).rsqrt()
        y = torch.einsum("rtw,rt,w->rtw", total, rstd, s["gamma"].double())
        out = {"rstd": rstd}
        if case["residual"]:
            out["total"] = total
        if case["out8"]:
            scales = torch.linalg.vector_norm(y, ord=math.inf, dim=2) / _LARGEST_8
            return {**out, "y": y / scales[..., None], "scales": scales}
        return {**out, "y": y}
    dx = torch.empty(s["dy"].shape, dtype=torch.float64, device="cuda")
    dgamma = torch.empty(s["dgamma"].shape, dtype=torch.float64, device="cuda")
    gamma = s["gamma"].double()
    for r in range(case["ranks"]):
        dy, rstd = s["dy"][r].double(), s["rstd"][r].double()[:, None]
        h = s["total"][r].double().mul_(rstd)
        # through y = gamma h: what lies along h is taken out
        along = (dy * h) @ gamma / case["width"]
        dx[r] = rstd * torch.addcmul(dy * gamma, h, along[:, None], value=-1)
        if case["residual"]:
            dx[r] += s["dtotal"][r].double()
        dgamma[r] = torch.einsum("tw,tw->w", dy, h)
    return {"dx": dx, "dgamma": dgamma}


def _exact_experts(s, case):
    ranks, tokens, k, experts = case["ranks"], case["tokens"], case["top_k"], case["experts"]
    out = {}
    for r in range(ranks):
        if case["step"] == "dispatch":
            expert = s["chosen"][r].flatten()
            live = expert >= 0
            if s["mask"] is not None:
                live &= s["mask"][r].repeat_interleave(k)
            slot = live.nonzero().flatten()
            # one number for each slot in use, by its expert and then its own number
            slot = (expert[slot].long() * (tokens * k) + slot).sort().values % (tokens * k)
            rows = torch.zeros(s["rows"].shape[1:], dtype=torch.float64, device="cuda")
            rows[:slot.numel()] = s["x"][r].double()[torch.div(slot, k, rounding_mode="floor")]
            places = torch.full((tokens * k,), -1, dtype=torch.int32, device="cuda")
            places[slot] = torch.arange(slot.numel(), dtype=torch.int32, device="cuda")
            first = torch.bincount(expert[live].long(), minlength=experts)[:experts].cumsum(0)
            one = {"rows": rows, "places": places.view(tokens, k),
                   "offsets": torch.cat((torch.zeros_like(first[:1]), first)).int()}
        else:
            p = s["places"][r].flatten().long()
            slot = (p >= 0).nonzero().flatten()
            weight = s["weights"][r].double().flatten()[slot, None]
            token = torch.div(slot, k, rounding_mode="floor")
            if case["step"] == "combine":
                y = torch.zeros((tokens, case["width"]), dtype=torch.float64, device="cuda")
                one = {"y": y.index_add_(0, token, s["rows"][r].double()[p[slot]] * weight)}
            else:
                dy = s["dy"][r].double()[token]
                drows = torch.zeros(s["rows"].shape[1:], dtype=torch.float64, device="cuda")
                drows[p[slot]] = dy * weight
                dweights = torch.zeros(tokens * k, dtype=torch.float64, device="cuda")
                dweights[slot] = torch.linalg.vecdot(dy, s["rows"][r].double()[p[slot]])
                one = {"drows": drows, "dweights": dweights.view(tokens, k)}
        for name, t in one.items():
            out.setdefault(name, []).append(t)
    return {name: torch.stack(t) for name, t in out.items()}


def _exact_embedding(s, case):
    if case["step"] == "forward":
        # a row of zeros for the padding, whose number is -1
        table = torch.cat((s["table"].double() * s["scale"], torch.zeros((1, case["width"]), dtype=torch.float64, device="cuda")))
        return {"y": table[s["ids"].long()]}
    d = torch.zeros((case["ranks"], case["vocab"] + 1, case["width"]), dtype=torch.float64, device="cuda")
    for r in range(case["ranks"]):
        d[r].index_add_(0, s["ids"][r].long() % (case["vocab"] + 1), s["dy"][r].double(), alpha=s["scale"])
    return {"dtable": d[:, :-1]}


def _exact_dropout(s, case):
    ranks, tokens, width = s["x"].shape
    seed, call = s["state"].tolist()
    limit = _threshold(case)
    y = torch.empty(s["x"].shape, dtype=torch.float64, device="cuda")
    at = {"dtype": torch.int64, "device": "cuda"}
    for r in range(ranks):
        block, token = torch.meshgrid(torch.arange(-(-width // 8), **at), torch.arange(tokens, **at), indexing="xy")
        c = [block, token, torch.full_like(block, r), torch.full_like(block, call)]
        for i in range(10):
            # products of 64 bits that wrap around; the shift copies the sign, which the mask takes off
            p, q = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
            key = (seed + i * 0x9E3779B9) & _WORD, ((seed >> 32) + i * 0xBB67AE85) & _WORD
            c = [(q >> 32 & _WORD) ^ c[1] ^ key[0], q & _WORD, (p >> 32 & _WORD) ^ c[3] ^ key[1], p & _WORD]
        kept = torch.stack([w >> shift & 0xFFFF for w in c for shift in (0, 16)], 2).view(tokens, -1)[:, :width] >= limit
        y[r] = s["x"][r].double() * kept / (1 - limit / 65536)
        if s["residual"] is not None:
            y[r] += s["residual"][r].double()
    return {"y": y}


def exact(case, seed):
    s = prepare(case, seed)
    return {"rmsnorm": _exact_norm, "experts": _exact_experts, "embedding": _exact_embedding,
            "dropout": _exact_dropout}[case["op"]](s, case)
