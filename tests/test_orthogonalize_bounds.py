"""The limits that the precision of orthogonalised matrices is held to pass the arithmetic of two fp16
planes and reject it with a lower plane missing in any single product."""

import pytest

torch = pytest.importorskip("torch")

import orthogonalize_util as ref

SIZES = [(40, 40), (64, 256), (96, 200)]
KINDS = ["even", "steep", "falling", "strong", "thin"]


def _case(size, kind):
    g = torch.Generator()
    g.manual_seed(sum(size))
    x = ref.spectrum(kind, (1, *size), g, "cpu")[0]
    return x, ref.steps(x, ref.QUINTIC, 1.0, 0.0, torch.float64), ref.steps(x, ref.QUINTIC, 1.0, 0.0, torch.float32)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_two_planes_pass(size, kind):
    x, want, plain = _case(size, kind)
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        assert ref.excess(ref.simulated(x, ref.QUINTIC, dtype), want, plain, ref.FAR_SUMS) <= 1.0


@pytest.mark.parametrize("step", range(5))
@pytest.mark.parametrize("what", ["gram", "square", "update"])
@pytest.mark.parametrize("side", ["l", "r"])
def test_a_plane_missing_anywhere_shows(step, what, side):
    """In some spectrum: where P is small beside a, or a later step covers an error, a single one has nothing to
    show. 16-bit results show those from the second step on."""
    worst = {torch.float32: 0.0, torch.bfloat16: 0.0}
    for size in SIZES:
        for kind in KINDS:
            x, want, plain = _case(size, kind)
            for dtype in worst:
                out = ref.simulated(x, ref.QUINTIC, dtype, (step, what, side))
                worst[dtype] = max(worst[dtype], ref.excess(out, want, plain, ref.NEAR))
    assert worst[torch.float32] > 1.0
    assert worst[torch.bfloat16] > 1.0 or step == 0
