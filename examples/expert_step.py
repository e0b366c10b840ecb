"""A data-parallel training step of a small model with experts, on virtual ranks, from the tokens' numbers to
the summed gradients.

Every rank holds its own sequences; all hold the same parameters: an embedding, the weights of two norms, a
router, a matrix for each expert and the output's matrix. In a step each rank looks its tokens up, drops a share
of the values, normalises the rows, sends each token to the experts its router chooses, adds what comes back to
the row, and predicts the next number. The gradients of a rank lie in one row of a buffer, the AllReduce sums the
rows, and the experts' matrices move by their orthogonalised momentum. Padding (number -1) is left out everywhere.

    python examples/expert_step.py [--steps 30] [--ranks 9] [--tokens 128]
"""

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2602_17254_amd as T  # noqa: E402


class Step:
    """The parameters, and the buffers that a training program keeps from step to step."""

    def __init__(self, ranks, tokens, vocab, width, experts, top_k, seed=0, rate=0.1, balance=0.01):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        dev = {"device": "cuda"}
        n, t, v, w, e, k = ranks, tokens, vocab, width, experts, top_k
        self.experts, self.top_k, self.rate, self.balance = e, k, rate, balance
        self.scale = math.sqrt(w)
        self.params = {"table": torch.randn((v, w), generator=g, **dev) / self.scale,
                       "gamma1": torch.ones(w, **dev), "gamma2": torch.ones(w, **dev),
                       "router": torch.randn((e, w), generator=g, **dev) / self.scale,
                       "matrices": torch.randn((e, w, w), generator=g, **dev) / self.scale,
                       "head": torch.randn((v, w), generator=g, **dev) / self.scale}
        # the seed of dropout, and the number of the step
        self.state = torch.tensor([seed, 0], dtype=torch.int64, **dev)
        self.momentum = torch.zeros((e, w, w), **dev)
        self.update = torch.empty_like(self.momentum)

        def rows(count=t):
            return torch.empty((n, count, w), **dev)

        self.h, self.y, self.mixed, self.total, self.y2 = rows(), rows(), rows(), rows(), rows()
        self.sorted, self.out, self.dout, self.dsorted = (rows(t * k).zero_() for _ in range(4))
        self.dtotal, self.dy, self.dh = rows(), rows(), rows()
        self.rstd, self.rstd2 = torch.empty((n, t), **dev), torch.empty((n, t), **dev)
        i32 = {"dtype": torch.int32, **dev}
        self.offsets, self.places = torch.empty((n, e + 1), **i32), torch.empty((n, t, k), **i32)
        self.dweights, self.dlogits = torch.empty((n, t, k), **dev), torch.empty((n, t, e), **dev)
        self.counts, self.probs = torch.empty((n, e + 1), **i32), torch.empty((n, e), **dev)
        self.balance_loss = torch.empty(n, **dev)
        # a rank's row of the buffer: all its gradients
        self.rows = torch.zeros((n, sum(p.numel() for p in self.params.values())), **dev)
        self.grads, at = {}, 0
        for name, p in self.params.items():
            self.grads[name] = self.rows[:, at:at + p.numel()].unflatten(1, p.shape)
            at += p.numel()
        self.plan, self.counts_plan = T.trivance_plan((n,), "B"), T.trivance_plan((n,), "L")
        self.work = {name: torch.empty(size, dtype=torch.uint8, **dev) for name, size in (
            ("norm", T.trivance_rmsnorm_workspace_bytes(n, t, w)),
            ("sort", T.trivance_experts_workspace_bytes(n, t, k, e)),
            ("table", T.trivance_embedding_workspace_bytes(n, t, w, v)),
            ("counts", T.trivance_balance_workspace_bytes(n, t, e)),
            ("sums", T.trivance_workspace_bytes(self.counts_plan, e + 1)),
            ("matrices", T.trivance_orthogonalize_workspace_bytes(e, w, w)))}

    def _segments(self):
        """Every rank's and expert's sorted rows (the program waits for the GPU here)."""
        for r, first in enumerate(self.offsets.tolist()):
            for e in range(self.experts):
                if first[e] < first[e + 1]:
                    yield r, e, slice(first[e], first[e + 1])

    def gradients(self, ids, target):
        """Every rank's gradients, summed over the ranks in every row of `grads`; the two losses."""
        p, g, mask = self.params, self.grads, ids >= 0
        T.trivance_embedding_forward(ids, p["table"], self.h, self.scale)
        T.trivance_dropout(self.h, self.h, self.state, self.rate)
        T.trivance_rmsnorm_forward(self.h, p["gamma1"], self.y, self.rstd)

        # to the experts and back
        logits = self.y @ p["router"].T
        best, chosen = torch.topk(logits, self.top_k, dim=2)
        weights = torch.softmax(best, 2)
        T.trivance_experts_sort(chosen, self.offsets, self.places, self.work["sort"], mask)
        T.trivance_experts_dispatch(self.y, self.places, self.sorted)
        segments = list(self._segments())
        for r, e, rows in segments:
            torch.mm(self.sorted[r, rows], p["matrices"][e], out=self.out[r, rows])
        T.trivance_experts_combine(self.out, self.places, self.mixed, weights)
        T.trivance_rmsnorm_forward(self.mixed, p["gamma2"], self.y2, self.rstd2, self.h, self.total)

        # the balance loss is that of all ranks' tokens: counts and sums of probabilities are summed first
        T.trivance_balance_counts(logits, chosen, self.counts, self.probs, self.work["counts"], mask)
        T.trivance_allreduce_emulated_ws(self.counts, self.counts_plan, self.work["sums"])
        T.trivance_allreduce_emulated_ws(self.probs, self.counts_plan, self.work["sums"])
        T.trivance_balance_loss(self.counts, self.probs, self.top_k, self.balance_loss, self.balance)
        T.trivance_balance_backward(logits, self.counts, self.top_k, self.dlogits, mask, self.balance)

        # the mean cross entropy over all ranks' tokens
        live = mask.to(torch.float32) / self.counts[:, -1].to(torch.float32).clamp(min=1)[:, None]
        logp = torch.log_softmax(self.y2 @ p["head"].T, 2)
        aim = target.clamp(min=0)[..., None]
        entropy = -(logp.gather(2, aim)[..., 0] * live).sum()
        dhead = logp.exp()
        dhead.scatter_add_(2, aim, torch.full_like(dhead[..., :1], -1.0))
        dhead *= live[..., None]
        g["head"].copy_(dhead.transpose(1, 2).contiguous() @ self.y2)

        # back through the second norm: its gradient goes to what the experts gave and to the row itself
        T.trivance_rmsnorm_backward(dhead @ p["head"], self.total, p["gamma2"], self.rstd2, self.dtotal,
                                    g["gamma2"], self.work["norm"])
        T.trivance_experts_combine_backward(self.dtotal, self.out, self.places, weights, self.dout, self.dweights)
        g["matrices"].zero_()
        for r, e, rows in segments:
            torch.mm(self.sorted[r, rows].T, self.dout[r, rows], out=g["matrices"][r, e])
            torch.mm(self.dout[r, rows], p["matrices"][e].T, out=self.dsorted[r, rows])
        T.trivance_experts_combine(self.dsorted, self.places, self.dy)
        dbest = weights * (self.dweights - (weights * self.dweights).sum(2, keepdim=True))
        self.dlogits.scatter_add_(2, chosen, dbest)
        g["router"].copy_(self.dlogits.transpose(1, 2).contiguous() @ self.y)
        self.dy += self.dlogits @ p["router"]
        # through the first norm, with what reached its row by the other way
        T.trivance_rmsnorm_backward(self.dy, self.h, p["gamma1"], self.rstd, self.dh, g["gamma1"], self.work["norm"],
                                    self.dtotal)
        T.trivance_dropout(self.dh, self.dh, self.state, self.rate)
        T.trivance_embedding_backward(self.dh, ids, g["table"], self.work["table"], self.scale)
        T.trivance_allreduce_emulated(self.rows, self.plan)
        return entropy, self.balance_loss[0]

    def apply(self, rate):
        """Moves the parameters by any rank's row of the summed gradients: they are equal."""
        self.momentum.mul_(0.9).add_(self.grads["matrices"][0])
        T.trivance_orthogonalize(self.momentum, self.update, self.work["matrices"])
        for name, p in self.params.items():
            p.sub_(self.update if name == "matrices" else self.grads[name][0], alpha=0.1 * rate if name == "matrices" else rate)
        self.state[1] += 1


def batch(ranks, tokens, vocab, seed):
    """Numbers in sequences that end early, each followed by a number that it decides."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    ids = torch.randint(0, vocab, (ranks, tokens), device="cuda", generator=g)
    length = torch.randint(1, tokens + 1, (ranks, 1), device="cuda", generator=g)
    ids[torch.arange(tokens, device="cuda") >= length] = -1
    return ids, torch.where(ids >= 0, (7 * ids + 3) % vocab, -1)


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--ranks", type=int, default=9)
    ap.add_argument("--tokens", type=int, default=128)
    ap.add_argument("--vocab", type=int, default=50)
    ap.add_argument("--width", type=int, default=64)
    ap.add_argument("--experts", type=int, default=8)
    ap.add_argument("--rate", type=float, default=1.0)
    a = ap.parse_args()
    step = Step(a.ranks, a.tokens, a.vocab, a.width, a.experts, top_k=2)
    for i in range(a.steps):
        entropy, balance = step.gradients(*batch(a.ranks, a.tokens, a.vocab, i))
        step.apply(a.rate)
        if i % 5 == 0 or i == a.steps - 1:
            print(f"step {i:3d}  cross entropy {float(entropy):.4f}  balance loss {float(balance):.4f}", flush=True)


if __name__ == "__main__":
    main()
