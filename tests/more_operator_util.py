"""Plain implementations in 64 bits of the RMS norm, the experts' calls, the embedding and dropout, and the
bounds their kernels are held to, which follow from the arithmetic as those of operator_util do (U, SUM and
the rounding of 16-bit results are its)."""

import numpy as np
import torch

from operator_util import SUM, U


def rmsnorm_forward(total, gamma, eps):
    """(y, bound), (rstd, bound) of double rows of the sum. A square has its sum's rounding twice and its own,
    the row's sum SUM more, and the root halves their number."""
    rstd = 1 / torch.sqrt((total * total).mean(-1) + eps)
    y = total * rstd[..., None] * gamma
    rel = (SUM / 2 + 8) * U
    return (y, (rel + 4 * U) * y.abs() + 1e-45), (rstd, rel * rstd)


def eight_bits(y):
    """The numbers of 8 bits that stand for y with their bound, and (scales, bound): half a step of three
    bits behind the leading one, or of the smallest numbers, 2^-9; and the factor's roundings."""
    scales = (y.abs().amax(-1) / 448).clamp(min=2.0 ** -126)
    q = y / scales[..., None]
    rel = (SUM + 30) * U
    return (q, (2.0 ** -4 + rel) * q.abs() + 2.0 ** -10), (scales, rel * scales)


def rmsnorm_backward(dy, total, gamma, rstd, dtotal):
    """(dx, bound), (dgamma, bound) [ranks, width] of double rows; rstd is the fp32 value that the kernel reads."""
    r = rstd[..., None]
    h, g = total * r, dy * gamma
    along = (g * h).mean(-1, keepdim=True)
    size = (g * h).abs().mean(-1, keepdim=True)
    dx = r * (g - h * along)
    bound = r * U * (8 * g.abs() + (SUM + 16) * h.abs() * size)
    if dtotal is not None:
        dx = dx + dtotal
        bound = bound + 2 * U * dtotal.abs()
    n = (total.shape[1] + 40) * U  # a lane adds its rows one by one, and a workgroup its at most 32 groups
    return (dx, bound + 1e-45), ((dy * h).sum(1), n * (dy * h).abs().sum(1) + 1e-45)


def experts_sort(chosen, mask, experts):
    """offsets, places, slots as nested lists of whole numbers, rank by rank, by Python's own stable sort."""
    ranks, tokens, k = chosen.shape
    ids = chosen.cpu().numpy()
    live = np.ones((ranks, tokens), bool) if mask is None else mask.cpu().numpy().astype(bool)
    offsets = np.zeros((ranks, experts + 1), np.int64)
    places = np.full((ranks, tokens * k), -1, np.int64)
    slots = np.full((ranks, tokens * k), -1, np.int64)
    for r in range(ranks):
        flat = ids[r].reshape(-1).astype(np.int64)
        used = np.nonzero((flat >= 0) & (flat < experts) & np.repeat(live[r], k))[0].tolist()
        used.sort(key=lambda s: int(flat[s]))
        slots[r, :len(used)] = used
        places[r, used] = np.arange(len(used))
        count = np.bincount(flat[used], minlength=experts) if used else np.zeros(experts, np.int64)
        offsets[r, 1:] = np.cumsum(count)
    return offsets, places.reshape(ranks, tokens, k), slots


def picked(rows, places):
    """Every slot's row [ranks, tokens, top_k, width] of double rows, zeros for those without one."""
    rank = torch.arange(rows.shape[0], device=rows.device).view(-1, 1, 1)
    live = (places >= 0) & (places < rows.shape[1])
    return torch.where(live[..., None], rows[rank, torch.where(live, places, 0).long()], 0.0), live


def combine(rows, places, weights):
    """(y, bound) of double rows and weights: a product and a sum for each slot."""
    v, live = picked(rows, places)
    w = torch.where(live, weights, 0.0)[..., None]
    return (v * w).sum(2), (places.shape[2] + 2) * U * (v * w).abs().sum(2) + 1e-45


def combine_backward(dy, rows, places, weights, drows):
    """((drows, bound), (dweights, bound)); drows is what lies there before. A lane adds up its values one
    by one: 64 lanes at least hold rows of more than 64 vectors."""
    v, live = picked(rows, places)
    d = dy[:, :, None]
    want, bound = drows.clone(), torch.zeros_like(drows)
    rank = torch.arange(rows.shape[0], device=rows.device).view(-1, 1, 1).expand(places.shape)[live]
    to = places[live].long()
    part = (d * weights[..., None])[live]
    want[rank, to] = part
    bound[rank, to] = U * part.abs() + 1e-45
    n = (rows.shape[2] / 64 + 24) * U
    return (want, bound), ((v * d).sum(3), n * (v * d).abs().sum(3) + 1e-45)


def table_gradient(dy, ids, vocab, scale, piece):
    """(dtable, bound) of double rows: sums of a number's tokens in fp32, at most `piece` of them in one."""
    ranks, tokens, width = dy.shape
    d = torch.zeros((ranks, vocab, width), dtype=torch.float64, device=dy.device)
    size = torch.zeros_like(d)
    count = torch.zeros((ranks, vocab), dtype=torch.float64, device=dy.device)
    for r in range(ranks):
        live = (ids[r] >= 0) & (ids[r] < vocab)
        to = ids[r][live].long()
        d[r].index_add_(0, to, dy[r][live])
        size[r].index_add_(0, to, dy[r][live].abs())
        count[r].index_add_(0, to, torch.ones(to.shape, dtype=torch.float64, device=dy.device))
    n = (count.clamp(max=piece) + 4)[..., None] * U
    return d * scale, n * size * abs(scale) + 1e-45


def piece_of(tokens):
    """The smallest power of two from 32 on, the 64-fold of whose square is not less than the number of tokens."""
    p = 32
    while 64 * p * p < tokens:
        p *= 2
    return p


def philox(counter, key):
    """Ten rounds of Philox-4x32 on four arrays of words and a key of two, in numpy's 64 bits."""
    mask = np.uint64(0xFFFFFFFF)
    c = [np.asarray(x, np.uint64) for x in counter]
    k = [int(x) for x in key]
    for _ in range(10):
        p, q = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(q >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), q & mask, (p >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), p & mask]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def kept(shape, seed, call, rate, first_rank=0):
    """Which values dropout keeps, a numpy array of truth values."""
    ranks, tokens, width = shape
    blocks = -(-width // 8)
    r, t, b = np.meshgrid(np.arange(ranks) + first_rank, np.arange(tokens), np.arange(blocks), indexing="ij")
    seed %= 1 << 64
    words = philox((b, t, r, np.full(b.shape, call % (1 << 32))), (seed & 0xFFFFFFFF, seed >> 32))
    halves = np.stack([w >> np.uint64(s) & np.uint64(0xFFFF) for w in words for s in (0, 16)], -1)
    return halves.reshape(ranks, tokens, blocks * 8)[:, :, :width] >= round(rate * 65536)
