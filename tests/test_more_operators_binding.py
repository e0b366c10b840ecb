"""What the binding of the RMS norm, the experts' calls, the embedding and dropout hands to the library and what it
refuses, without a GPU: host tensors that say they are on one, and a library that records its arguments."""

import pytest

torch = pytest.importorskip("torch")

import paper_2602_17254_amd as T
from test_operators_binding import Library, OnOtherGpu, gpu

B = T.binding


@pytest.fixture
def library(monkeypatch):
    lib = Library()
    monkeypatch.setattr(B, "_lib", lambda: lib)
    monkeypatch.setattr(B, "_stream_ptr", lambda stream: 0)
    monkeypatch.setattr(B, "_current_device", lambda: 0, raising=False)
    return lib


def _calls():
    """Every call, as (name, call of its arguments, the arguments)."""
    x, s, w, rows = gpu(2, 3, 8), gpu(2, 3), gpu(8), gpu(2, 6, 8)
    q = torch.zeros((2, 3, 8), dtype=torch.float8_e4m3fn).as_subclass(type(x))
    places, slots = gpu(2, 3, 2, dtype=torch.int32), gpu(2, 6, dtype=torch.int32)
    chosen, weights = gpu(2, 3, 2, dtype=torch.int64), gpu(2, 3, 2)
    ids, table, state = gpu(2, 3, dtype=torch.int64), gpu(5, 8), gpu(2, dtype=torch.int64)
    return [("norm", T.trivance_rmsnorm_forward, [x, w, x, s, x, x]),
            ("norm of 8 bits", T.trivance_rmsnorm_forward, [x, w, q, s, x, x, s]),
            ("norm backward", T.trivance_rmsnorm_backward, [x, x, w, s, x, gpu(2, 8), gpu(8), x]),
            ("sort", T.trivance_experts_sort, [chosen, gpu(2, 5, dtype=torch.int32), places, gpu(8), s.bool(), slots]),
            ("dispatch", T.trivance_experts_dispatch, [x, places, rows]),
            ("combine", T.trivance_experts_combine, [rows, places, x, weights]),
            ("combine backward", T.trivance_experts_combine_backward, [x, rows, places, weights, rows, weights]),
            ("lookup", T.trivance_embedding_forward, [ids, table, x, 1.0]),
            ("table", T.trivance_embedding_backward, [x, ids, gpu(2, 5, 8), gpu(8), 1.0]),
            ("dropout", T.trivance_dropout, [x, x, state, 0.1, x])]


def test_tensors_of_several_gpus_are_refused(library):
    """Any one tensor elsewhere, the workspace among them, and all of them on a GPU that is not the current one."""
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


# Workspaces, by their place among the arguments, may be larger and of any type; a last dimension of one expert or one slot
# more is another call's.
WORKSPACES = {"norm backward": 6, "sort": 3, "table": 3}
FREE = {"sort": 1, "dispatch": 1}


def test_tensors_of_other_shapes_and_types_are_refused(library):
    """Every tensor with one value more in its last dimension, or of a type that it cannot have."""
    for name, call, args in _calls():
        for i, a in enumerate(args):
            if not isinstance(a, torch.Tensor) or WORKSPACES.get(name) == i:
                continue
            longer, complex_ = torch.zeros((*a.shape[:-1], a.shape[-1] + 1), dtype=a.dtype), torch.zeros(a.shape, dtype=torch.complex64)
            for other in [complex_] if FREE.get(name) == i else [longer, complex_]:
                bad = list(args)
                bad[i] = other.as_subclass(type(a))
                with pytest.raises((TypeError, ValueError)):
                    call(*bad)
                    print(name, i, other.dtype)
    assert not library.calls


def test_what_is_handed_on(library):
    x, w, s = gpu(2, 3, 12)[:, :, 2:10], gpu(8, dtype=torch.bfloat16), gpu(2, 3)
    T.trivance_rmsnorm_forward(x, w, gpu(2, 3, 8), s, None, None, eps=0.5)
    args = library.calls[-1][1]
    assert args[1] is None and args[3] is None and args[6] is None
    assert args[7:18] == (2, 3, 8, 36, 12, 0, 0, 0, 0, 24, 8) and args[18:22] == (0.5, T.F32, T.F32, T.BF16)
    rows, places = gpu(2, 7, 9)[:, :, 1:], gpu(2, 3, 2, dtype=torch.int32)
    T.trivance_experts_combine(rows, places, gpu(2, 3, 8), None)
    args = library.calls[-1][1]
    assert args[2] is None and args[4:13] == (2, 3, 2, 8, 7, 63, 9, 24, 8)
    # the rank stride of one rank's table does not matter, nor the row stride of a table of one row
    T.trivance_embedding_backward(gpu(1, 3, 8), gpu(1, 3, dtype=torch.int32), gpu(1, 99)[:, 9:49].unflatten(1, (5, 8)), gpu(8), 2.0)
    assert library.calls[-1][1][3:12] == (1, 3, 8, 5, 24, 8, 40, 2.0, T.F32)
    with pytest.raises(ValueError):  # rows that do not follow one another
        T.trivance_embedding_backward(gpu(2, 3, 8), gpu(2, 3, dtype=torch.int32), gpu(2, 5, 9)[:, :, :8], gpu(8))
    with pytest.raises(ValueError):
        T.trivance_experts_sort(gpu(2, 6, 2, dtype=torch.int32)[:, ::2], gpu(2, 5, dtype=torch.int32), places)
