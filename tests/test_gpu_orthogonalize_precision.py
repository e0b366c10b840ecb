"""GPU: how near trivance_orthogonalize comes to its definition in 64 bits, held to what plain fp32
products of the same matrices reach. Limits: orthogonalize_util."""

import pytest

import orthogonalize_util as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
KINDS = ["even", "steep", "falling", "strong", "thin"]


def _measure(size, kind, dtype, coefficients=ref.QUINTIC, factor=1.0, eps=1e-7):
    """The excess of every matrix of a call, with `near` as its size asks."""
    import paper_2602_17254_amd as T

    g = torch.Generator(device="cuda")
    g.manual_seed(sum(size))
    x = (factor * ref.spectrum(kind, size, g, "cuda")).to(TYPES[dtype])
    out = torch.empty_like(x)
    ws = torch.full((T.trivance_orthogonalize_workspace_bytes(*size),), 255, dtype=torch.uint8, device="cuda")
    T.trivance_orthogonalize(x, out, ws, coefficients, 1.0, eps)
    torch.cuda.synchronize()
    near = ref.FAR_SUMS if min(size[1:]) >= 512 else ref.NEAR
    worst = 0.0
    for b in range(size[0]):
        want = ref.steps(x[b], coefficients, 1.0, eps, torch.float64)
        plain = ref.steps(x[b], coefficients, 1.0, eps, torch.float32)
        worst = max(worst, ref.excess(out[b], want, plain, near))
    print("[orthogonalize]", size, kind, dtype, "excess %.2f of the limit" % worst, flush=True)
    return worst


# one workgroup, strips, and the product kernels with little to fill their tiles; a limit that rests on chance wants many values
SMALL = [(2, 64, 250), (1, 48, 3001), (3, 130, 77), (1, 257, 130), (2, 515, 300)]
# single steps whose last product stands alone
SQUARE = [(1, 600, 640), (3, 770, 515), (1, 1030, 1500)]
# the larger side twice the smaller or more
WIDE = [(1, 600, 5000), (1, 1024, 4096), (1, 4100, 1030), (1, 2033, 8100)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("size", SMALL + SQUARE + WIDE, ids=lambda s: "x".join(map(str, s)))
def test_as_near_as_fp32_products(size, kind, dtype):
    assert _measure(size, kind, dtype) <= 1.0


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("steps", [1, 5])
@pytest.mark.parametrize("form", ref.FORMS)
def test_every_form(form, steps, dtype):
    assert _measure(ref.FORMS[form], "falling", dtype, ref.QUINTIC[:steps]) <= 1.0


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", [(1, 2176, 1600), (3, 1030, 1030), (1, 3990, 4010), (1, 8100, 2033)],
                         ids=lambda s: "x".join(map(str, s)))
def test_large(size, dtype):
    assert _measure(size, "falling", dtype, ref.QUINTIC[:1]) <= 1.0
    assert _measure(size, "steep", dtype) <= 1.0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(2, 64, 250), (1, 48, 3001), (1, 130, 300), (1, 600, 1300)],
                         ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("factor,eps", [(1e-8, 1e-7), (1e-10, 1e-7), (1e-13, 1e-7), (1e-17, 1e-7), (1e-30, 1e-20),
                                        (1.0, 1e25)])
def test_norms_far_below_eps(size, factor, eps, dtype):
    """X starts far below one, and the steps raise it by their a."""
    assert _measure(size, "falling", dtype, ref.QUINTIC, factor, eps) <= 1.0
    assert _measure(size, "even", dtype, ((1.5, -0.5, 0.0),) * 12, factor, eps) <= 1.0


def test_more_than_2_31_values():
    import paper_2602_17254_amd as T

    size = (520, 2049, 2030)
    x = torch.empty(size, dtype=torch.bfloat16, device="cuda")
    assert x.numel() > 2 ** 31
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    for part in x:
        part.copy_(ref.spectrum("falling", (1, *size[1:]), g, "cuda")[0])
    out = torch.empty_like(x)
    ws = torch.empty(T.trivance_orthogonalize_workspace_bytes(*size), dtype=torch.uint8, device="cuda")
    T.trivance_orthogonalize(x, out, ws, ref.QUINTIC[:2])
    for b in (0, 263, 519):
        want = ref.steps(x[b], ref.QUINTIC[:2], 1.0, 1e-7, torch.float64)
        plain = ref.steps(x[b], ref.QUINTIC[:2], 1.0, 1e-7, torch.float32)
        assert ref.excess(out[b], want, plain, ref.FAR_SUMS) <= 1.0
