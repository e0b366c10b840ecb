"""GPU: examples/data_parallel_step.py: the operators together with the AllReduce. One step's summed
gradients against autograd in 64 bits on all ranks' tokens at once, and the example's losses going down."""

import importlib.util
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EXAMPLE = os.path.join(ROOT, "examples", "data_parallel_step.py")


def _example():
    spec = importlib.util.spec_from_file_location("data_parallel_step", EXAMPLE)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("ranks,tokens,width,experts,top_k", [(9, 40, 96, 8, 2), (4, 65, 130, 12, 3), (1, 30, 64, 6, 1)])
def test_summed_gradients_are_those_of_all_tokens(ranks, tokens, width, experts, top_k):
    m = _example()
    s = m.Step(ranks, tokens, width, experts, top_k, seed=3)
    x, target, mask = m.batch(ranks, tokens, width, experts, 5)
    s.gamma.add_(0.1 * torch.randn(width, device="cuda", generator=torch.Generator("cuda").manual_seed(1)))
    entropy, balance = s.gradients(x, target, mask)
    torch.cuda.synchronize()
    print("[step] losses", float(entropy), float(balance), flush=True)

    p = [t.double().requires_grad_() for t in (s.router, s.gamma, s.beta)]
    rows, aims = x[mask].double(), target[mask]
    d = rows - rows.mean(1, keepdim=True)
    y = d / torch.sqrt((d * d).mean(1, keepdim=True) + 1e-5) * p[1] + p[2]
    logits = y @ p[0].T
    # the choice is a constant of the balance loss: the kernel's own, which ties or near ties may decide
    f = s.counts[0, :experts].double()
    n = rows.shape[0]
    assert int(s.counts[0, experts]) == n and int(f.sum()) == n * top_k
    ce = torch.nn.functional.cross_entropy(logits, aims)
    bal = s.balance * experts * (f / (top_k * n) * torch.softmax(logits, 1).sum(0) / n).sum()
    grads = torch.autograd.grad(ce + bal, p)
    # fp32 throughout: sums over some hundred tokens and a hundred columns, relative to the largest
    # gradient of a tensor
    assert abs(float(entropy) - float(ce)) <= 1e-5 * abs(float(ce))
    assert abs(float(balance) - float(bal)) <= 1e-5 * abs(float(bal))
    for got, want in zip((s.drouter, s.dgamma, s.dbeta), grads):
        assert torch.equal(got, got[:1].expand_as(got)), "every rank holds the same sum"
        err = float((got[0].double() - want).abs().max())
        assert err <= 2e-5 * float(want.abs().max()), (err, float(want.abs().max()))


def test_example_learns():
    res = subprocess.run([sys.executable, EXAMPLE, "--steps", "21", "--tokens", "128"], capture_output=True, text=True,
                         timeout=100)
    print(res.stdout, flush=True)
    assert res.returncode == 0, res.stdout + res.stderr
    lines = [line.split() for line in res.stdout.splitlines() if line.startswith("step")]
    first, last = float(lines[0][4]), float(lines[-1][4])
    assert last < 0.8 * first, (first, last)
