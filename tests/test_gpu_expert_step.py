"""GPU: examples/expert_step.py: the embedding, dropout, the norm, the experts' calls, the balance loss and the
AllReduce together. One step's summed gradients against autograd in 64 bits on all ranks' tokens at once, twice, as
dropout draws anew in the second; and that the example runs."""

import importlib.util
import os
import subprocess
import sys

import pytest

import more_operator_util as more

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EXAMPLE = os.path.join(ROOT, "examples", "expert_step.py")


def _example():
    spec = importlib.util.spec_from_file_location("expert_step", EXAMPLE)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _losses(s, p, ids, target, chosen):
    """The two losses in 64 bits; the experts chosen and their counts are constants, the kernels' own."""
    mask = ids >= 0
    kept = torch.from_numpy(more.kept(s.h.shape, *s.state.tolist(), s.rate)).to("cuda")
    keep = kept / (1 - round(s.rate * 65536) / 65536)
    h = torch.where(mask[..., None], p["table"][ids.clamp(min=0)], 0.0) * s.scale * keep

    def norm(x, gamma):
        return x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-5) * gamma

    y = norm(h, p["gamma1"])
    logits = y @ p["router"].T
    weights = torch.softmax(logits.gather(2, chosen), 2)
    given = torch.stack([y @ m for m in p["matrices"]], 2)  # of every expert
    picked = given.gather(2, chosen[..., None].expand(-1, -1, -1, y.shape[2]))
    mixed = (weights[..., None] * picked).sum(2) * mask[..., None]
    out = norm(h + mixed, p["gamma2"]) @ p["head"].T
    n = int(mask.sum())
    ce = torch.nn.functional.cross_entropy(out[mask], target[mask])
    f = torch.bincount(chosen[mask].flatten(), minlength=s.experts).double()
    bal = s.balance * s.experts * (f / (s.top_k * n) * torch.softmax(logits[mask], 1).sum(0) / n).sum()
    return ce, bal


@pytest.mark.parametrize("ranks,tokens,vocab,width,experts,top_k", [(9, 40, 60, 96, 8, 2), (4, 65, 1500, 130, 12, 3),
                                                                    (1, 30, 17, 64, 6, 1)])
def test_summed_gradients_are_those_of_all_tokens(ranks, tokens, vocab, width, experts, top_k):
    m = _example()
    s = m.Step(ranks, tokens, vocab, width, experts, top_k, seed=3, rate=0.2)
    g = torch.Generator("cuda").manual_seed(1)
    for name in ("gamma1", "gamma2"):
        s.params[name].add_(0.1 * torch.randn(width, device="cuda", generator=g))
    for turn in range(2):
        ids, target = m.batch(ranks, tokens, vocab, 5)
        entropy, balance = s.gradients(ids, target)
        torch.cuda.synchronize()
        print("[step] losses", float(entropy), float(balance), flush=True)
        chosen = torch.topk(s.y @ s.params["router"].T, top_k, dim=2).indices
        p = {name: t.double().requires_grad_() for name, t in s.params.items()}
        ce, bal = _losses(s, p, ids, target, chosen)
        grads = torch.autograd.grad(ce + bal, list(p.values()))
        ce, bal = ce.detach(), bal.detach()
        # fp32 throughout: two norms, some three products and sums over at most some hundred tokens or columns in
        # a row, of which each is off by some tens of units at most, 200 in all, of 2^-24, relative to the largest
        assert abs(float(entropy) - float(ce)) <= 2e-5 * abs(float(ce))
        assert abs(float(balance) - float(bal)) <= 2e-5 * abs(float(bal))
        for name, want in zip(p, grads):
            got = s.grads[name]
            assert torch.equal(got, got[:1].expand_as(got)), "every rank holds the same sum"
            err, most = float((got[0].double() - want).abs().max()), float(want.abs().max())
            print("[step]", name, err, most, flush=True)
            assert err <= 4e-5 * most, (name, err, most)
        s.state[1] += 1


def test_example_runs():
    res = subprocess.run([sys.executable, EXAMPLE, "--steps", "7", "--tokens", "64"], capture_output=True, text=True,
                         timeout=100)
    print(res.stdout, flush=True)
    assert res.returncode == 0, res.stdout + res.stderr
    assert res.stdout.splitlines()[-1].startswith("step   6")
