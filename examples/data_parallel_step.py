"""A data-parallel training step on virtual ranks: what the ranks put into the AllReduce and what is done with
the sum.

Every rank holds its own tokens; all hold the same parameters: the weights of a layer norm and a router's
matrix. In a step each rank normalises its tokens, scores the experts, and forms its gradients of the mean
cross entropy to the experts its tokens should go to and of the balance loss over all ranks' tokens. The
gradients of a rank lie in one row of a buffer, the AllReduce sums the rows, and the router's matrix
moves by the orthogonalised momentum of its summed gradient.

    python examples/data_parallel_step.py [--steps 30] [--ranks 9] [--tokens 256]
"""

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2602_17254_amd as T  # noqa: E402


class Step:
    """The parameters, and the buffers that a training program keeps from step to step."""

    def __init__(self, ranks, tokens, width, experts, top_k, seed=0, balance=0.1):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        dev = {"device": "cuda"}
        self.ranks, self.tokens, self.width, self.experts, self.top_k = ranks, tokens, width, experts, top_k
        self.balance = balance
        self.gamma = torch.ones(width, **dev)
        self.beta = torch.zeros(width, **dev)
        self.router = torch.randn((experts, width), generator=g, **dev) / width ** 0.5
        self.momentum = torch.zeros((1, experts, width), **dev)
        self.update = torch.empty_like(self.momentum)
        self.plan = T.trivance_plan((ranks,), "B")
        self.counts_plan = T.trivance_plan((ranks,), "L")

        n, t, e, w = ranks, tokens, experts, width
        self.y = torch.empty((n, t, w), **dev)
        self.mean, self.rstd = torch.empty((n, t), **dev), torch.empty((n, t), **dev)
        self.dx, self.dbalance = torch.empty((n, t, w), **dev), torch.empty((n, t, e), **dev)
        self.counts = torch.empty((n, e + 1), dtype=torch.int32, **dev)
        self.probs, self.balance_loss = torch.empty((n, e), **dev), torch.empty(n, **dev)
        # a rank's row: the router's gradient, the layer norm's two
        self.grads = torch.empty((n, e * w + 2 * w), **dev)
        self.drouter = self.grads[:, :e * w].unflatten(1, (e, w))
        self.dgamma, self.dbeta = self.grads[:, e * w:e * w + w], self.grads[:, e * w + w:]
        self.work = {name: torch.empty(size, dtype=torch.uint8, **dev) for name, size in (
            ("norm", T.trivance_layernorm_workspace_bytes(n, t, w)),
            ("counts", T.trivance_balance_workspace_bytes(n, t, e)),
            ("sums", T.trivance_workspace_bytes(self.counts_plan, e + 1)),
            ("matrix", T.trivance_orthogonalize_workspace_bytes(1, e, w)))}

    def _sum_counts(self, rows):
        T.trivance_allreduce_emulated_ws(rows, self.counts_plan, self.work["sums"])

    def gradients(self, x, target, mask):
        """Every rank's gradients, summed over the ranks in every row of `grads`; the two losses."""
        T.trivance_layernorm_forward(x, self.gamma, self.beta, self.y, self.mean, self.rstd)
        logits = self.y @ self.router.T
        chosen = torch.topk(logits, self.top_k, dim=2).indices

        # the balance loss is that of all ranks' tokens: counts and sums of probabilities are summed first
        T.trivance_balance_counts(logits, chosen, self.counts, self.probs, self.work["counts"], mask)
        self._sum_counts(self.counts)
        self._sum_counts(self.probs)
        T.trivance_balance_loss(self.counts, self.probs, self.top_k, self.balance_loss, self.balance)
        T.trivance_balance_backward(logits, self.counts, self.top_k, self.dbalance, mask, self.balance)

        # the mean cross entropy over all ranks' tokens, whose number every rank now knows
        tokens = self.counts[:, -1].to(torch.float32).clamp(min=1)[:, None]
        logp = torch.log_softmax(logits, dim=2)
        live = mask.to(torch.float32) / tokens
        entropy = -(logp.gather(2, target[..., None])[..., 0] * live).sum()
        dlogits = logp.exp()
        dlogits.scatter_add_(2, target[..., None], torch.full_like(dlogits[..., :1], -1.0))
        dlogits = dlogits * live[..., None] + self.dbalance

        self.drouter.copy_(dlogits.transpose(1, 2).contiguous() @ self.y)
        T.trivance_layernorm_backward(dlogits @ self.router, x, self.gamma, self.mean, self.rstd, self.dx,
                                      self.dgamma, self.dbeta, self.work["norm"])
        T.trivance_allreduce_emulated(self.grads, self.plan)
        return entropy, self.balance_loss[0]

    def apply(self, rate):
        """Moves the parameters by any rank's row of the summed gradients: they are equal."""
        self.momentum.mul_(0.9).add_(self.drouter[:1])
        T.trivance_orthogonalize(self.momentum, self.update, self.work["matrix"])
        self.router.sub_(self.update[0], alpha=rate)
        self.gamma.sub_(self.dgamma[0], alpha=rate)
        self.beta.sub_(self.dbeta[0], alpha=rate)


def batch(ranks, tokens, width, experts, seed):
    """Tokens of every rank, the expert that each should go to (by directions that are the same for all),
    and a mask: sequences end early."""
    g = torch.Generator(device="cuda")
    g.manual_seed(123)
    directions = torch.randn((experts, width), device="cuda", generator=g)
    g.manual_seed(seed)
    x = torch.randn((ranks, tokens, width), device="cuda", generator=g)
    length = torch.randint(1, tokens + 1, (ranks, 1), device="cuda", generator=g)
    return x, (x @ directions.T).argmax(2), torch.arange(tokens, device="cuda") < length


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--ranks", type=int, default=9)
    ap.add_argument("--tokens", type=int, default=256)
    ap.add_argument("--width", type=int, default=128)
    ap.add_argument("--experts", type=int, default=16)
    ap.add_argument("--rate", type=float, default=0.05)
    a = ap.parse_args()
    step = Step(a.ranks, a.tokens, a.width, a.experts, top_k=2)
    for i in range(a.steps):
        entropy, balance = step.gradients(*batch(a.ranks, a.tokens, a.width, a.experts, i))
        step.apply(a.rate)
        if i % 5 == 0 or i == a.steps - 1:
            print(f"step {i:3d}  cross entropy {float(entropy):.4f}  balance loss {float(balance):.4f}", flush=True)


if __name__ == "__main__":
    main()
