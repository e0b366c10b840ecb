"""What the binding of the operators around the AllReduce hands to the library and what it refuses, without a
GPU: host tensors that say they are on one, and a library that records its arguments."""

import pytest

torch = pytest.importorskip("torch")

import paper_2602_17254_amd as T

B = T.binding


class OnGpu(torch.Tensor):
    """A host tensor that passes for one on GPU 0."""

    is_cuda = True

    def get_device(self):
        return 0


class OnOtherGpu(OnGpu):
    def get_device(self):
        return 1


def gpu(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnGpu)


class Library:
    """Takes every call, launches nothing."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return 0

        return call


@pytest.fixture
def library(monkeypatch):
    lib = Library()
    monkeypatch.setattr(B, "_lib", lambda: lib)
    monkeypatch.setattr(B, "_stream_ptr", lambda stream: 0)
    monkeypatch.setattr(B, "_current_device", lambda: 0, raising=False)
    return lib


def _backward(dgamma, dbeta):
    x, s = gpu(4, 3, 8), gpu(4, 3)
    T.trivance_layernorm_backward(x, x, None, s, s, x, dgamma, dbeta)


GRAD_STRIDE = 17  # the place of grad_rank_stride among the C call's arguments


def test_gradient_rows_with_strides_of_their_own(library):
    apart, dense = gpu(4, 20)[:, :8], gpu(4, 8)
    for dgamma, dbeta, stride in ((apart, gpu(4, 20)[:, 8:16], 20), (apart, None, 20), (None, dense, 8)):
        _backward(dgamma, dbeta)
        assert library.calls[-1][1][GRAD_STRIDE] == stride
    _backward(None, None)
    for dgamma, dbeta in ((apart, dense), (dense, apart)):
        with pytest.raises(ValueError):
            _backward(dgamma, dbeta)


def test_one_gradient_row_for_all_ranks_is_refused(library):
    """A stride of zero is a stride: beside another it is unequal, and alone it reaches the library, which
    refuses rows that overlap."""
    one, rows = gpu(1, 8).expand(4, 8), gpu(4, 8)
    for dgamma, dbeta in ((one, rows), (rows, one)):
        with pytest.raises(ValueError):
            _backward(dgamma, dbeta)
    assert not library.calls
    for dgamma, dbeta in ((one, None), (None, one), (one, one)):
        _backward(dgamma, dbeta)
        assert library.calls[-1][1][GRAD_STRIDE] == 0


COEFFICIENTS, STEPS = 9, 10  # their places among the arguments


def _orthogonalize(library, steps):
    x = gpu(1, 4, 4)
    T.trivance_orthogonalize(x, x, gpu(8), steps)
    args = library.calls[-1][1]
    return list(args[COEFFICIENTS])[:3 * args[STEPS]]


def test_coefficients_are_those_of_the_call(library):
    """Also where the same numbers' objects held other values in the call before."""
    a, b, c = (torch.tensor(v, dtype=torch.float64) for v in (3.0, -4.0, 2.0))
    steps = ((a, b, c), (1.5, b, 0))
    assert _orthogonalize(library, steps) == [3.0, -4.0, 2.0, 1.5, -4.0, 0.0]
    b.fill_(-0.5)
    assert _orthogonalize(library, steps) == [3.0, -0.5, 2.0, 1.5, -0.5, 0.0]
    assert _orthogonalize(library, [[1, 2, 3]]) == [1.0, 2.0, 3.0]
    assert len(_orthogonalize(library, T.QUINTIC_5)) == 15


@pytest.mark.parametrize("steps", [((1, 2), (3, 4, 5, 6)), ((1, 2, 3, 4),), ((1, 2),), [[1.0, 2.0, 3.0], []]], ids=str)
def test_each_step_has_three_coefficients(library, steps):
    with pytest.raises(ValueError):
        _orthogonalize(library, steps)
    assert not library.calls


def _calls():
    """Every call of the operators, as (name, call of its arguments, the arguments)."""
    x, s, w, g = gpu(2, 3, 8), gpu(2, 3), gpu(8), gpu(2, 8)
    counts, ids = gpu(2, 9, dtype=torch.int32), gpu(2, 3, 2, dtype=torch.int64)
    return [("forward", T.trivance_layernorm_forward, [x, w, w, x, s, s]),
            ("backward", T.trivance_layernorm_backward, [x, x, w, s, s, x, g, g, gpu(8)]),
            ("counts", T.trivance_balance_counts, [x, ids, counts, g, gpu(8), s.bool()]),
            ("loss", T.trivance_balance_loss, [counts, g, 2, gpu(2)]),
            ("gradient", T.trivance_balance_backward, [x, counts, 2, x, s.bool(), 1.0, gpu(2)]),
            ("orthogonalize", T.trivance_orthogonalize, [x, x, gpu(8)])]


def test_tensors_of_several_gpus_are_refused(library):
    """Any one tensor elsewhere, the workspace among them, and all of them on a GPU that is not the current
    one, on whose stream the kernels would run."""
    for name, call, args in _calls():
        call(*args)
        launched = len(library.calls)
        tensors = [i for i, a in enumerate(args) if isinstance(a, torch.Tensor)]
        for i in tensors:
            other = list(args)
            other[i] = args[i].as_subclass(OnOtherGpu)
            with pytest.raises((TypeError, ValueError)):
                call(*other)
        with pytest.raises((TypeError, ValueError)):
            call(*[a.as_subclass(OnOtherGpu) if i in tensors else a for i, a in enumerate(args)])
        assert len(library.calls) == launched, name
