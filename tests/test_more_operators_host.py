"""The refusals of the RMS norm, the experts' calls, the embedding and dropout, through the C ABI and the
binding, without a GPU: every case here is turned away, or has nothing to do, before any kernel is launched."""

import ctypes
import math
import os
import re

import numpy as np
import pytest

import more_operator_util as more
import paper_2602_17254_amd as T

OK, EINVAL, EUNSUPPORTED, ESIZE = 0, -1, -2, -5
P, Q = 4096, 8192  # addresses that are never followed
BIG = 1 << 40


def _lib():
    return T.binding._lib()


def norm(**kw):
    a = dict(x=P, residual=P, gamma=P, total=P, y=Q, rstd=P, scales=None, ranks=2, tokens=3, width=8, xr=24, xt=8,
             rr=24, rt=8, tr=24, tt=8, yr=24, yt=8, eps=1e-5, dtype=T.F32, ytype=T.F32, wtype=T.F32, stream=None)
    a.update(kw)
    return _lib().trivance_rmsnorm_forward(*a.values())


def norm_backward(**kw):
    a = dict(dy=P, total=P, gamma=P, rstd=P, dtotal=P, dx=P, dgamma=P, ranks=2, tokens=3, width=8, dyr=24, dyt=8,
             tr=24, tt=8, mr=24, mt=8, dxr=24, dxt=8, gr=8, dtype=T.F32, wtype=T.F32, ws=P, wsb=BIG, stream=None)
    a.update(kw)
    return _lib().trivance_rmsnorm_backward(*a.values())


def sort(**kw):
    a = dict(chosen=P, mask=None, offsets=P, places=P, slots=P, ranks=2, tokens=3, k=2, experts=8, ids=T.I32, ws=P,
             wsb=BIG, stream=None)
    a.update(kw)
    return _lib().trivance_experts_sort(*a.values())


def dispatch(**kw):
    a = dict(x=P, places=P, rows=Q, ranks=2, tokens=3, k=2, width=8, capacity=6, xr=24, xt=8, rr=48, rs=8, dtype=T.F32,
             stream=None)
    a.update(kw)
    return _lib().trivance_experts_dispatch(*a.values())


def combine(**kw):
    a = dict(rows=P, places=P, weights=P, y=Q, ranks=2, tokens=3, k=2, width=8, capacity=6, rr=48, rs=8, yr=24, yt=8,
             dtype=T.F32, wtype=T.F32, stream=None)
    a.update(kw)
    return _lib().trivance_experts_combine(*a.values())


def gradient(**kw):
    a = dict(dy=P, rows=P, places=P, weights=P, drows=Q, dweights=P, ranks=2, tokens=3, k=2, width=8, capacity=6,
             yr=24, yt=8, rr=48, rs=8, dr=48, ds=8, dtype=T.F32, wtype=T.F32, stream=None)
    a.update(kw)
    return _lib().trivance_experts_combine_backward(*a.values())


def lookup(**kw):
    a = dict(ids=P, table=P, y=Q, ranks=2, tokens=3, width=8, vocab=10, row=8, yr=24, yt=8, scale=1.0, dtype=T.F32,
             ttype=T.BF16, ids_type=T.I64, stream=None)
    a.update(kw)
    return _lib().trivance_embedding_forward(*a.values())


def table(**kw):
    a = dict(dy=P, ids=P, dtable=Q, ranks=2, tokens=3, width=8, vocab=10, dyr=24, dyt=8, tr=80, scale=1.0, dtype=T.F32,
             ids_type=T.I64, ws=P, wsb=BIG, stream=None)
    a.update(kw)
    return _lib().trivance_embedding_backward(*a.values())


def dropout(**kw):
    a = dict(x=P, residual=P, y=Q, state=P, ranks=2, tokens=3, width=8, xr=24, xt=8, rr=24, rt=8, yr=24, yt=8, rate=0.1,
             dtype=T.F32, stream=None)
    a.update(kw)
    return _lib().trivance_dropout(*a.values())


@pytest.mark.parametrize("kw", [
    dict(dtype=T.I32), dict(dtype=9), dict(dtype=T.E4M3, ytype=T.E4M3), dict(wtype=T.I64), dict(wtype=T.E4M3),
    dict(ytype=T.BF16), dict(ytype=T.E4M3), dict(scales=P), dict(ranks=0), dict(tokens=-1), dict(width=0),
    dict(width=(1 << 24) + 1), dict(eps=-1.0), dict(eps=math.nan), dict(x=None), dict(y=None), dict(total=Q),
    dict(xr=-1), dict(xt=-8), dict(rr=-1), dict(rt=-1), dict(tr=0), dict(tt=7), dict(yr=-1), dict(yt=7), dict(yr=23),
    dict(yr=0), dict(yt=0), dict(xr=1 << 60), dict(ranks=1 << 40, tokens=1 << 40), dict(yr=8, yt=8),
    dict(ytype=T.E4M3, scales=P, x=Q), dict(ytype=T.E4M3, scales=P, residual=Q)], ids=str)
def test_rmsnorm_forward_refuses(kw):
    assert norm(**kw) == EINVAL


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=T.I32), EINVAL), (dict(dtype=T.E4M3), EINVAL), (dict(wtype=5), EINVAL), (dict(ranks=0), EINVAL),
    (dict(width=0), EINVAL), (dict(tokens=-1), EINVAL), (dict(dy=None), EINVAL), (dict(total=None), EINVAL),
    (dict(rstd=None), EINVAL), (dict(dx=None), EINVAL), (dict(dxt=4), EINVAL), (dict(mr=-1), EINVAL),
    (dict(tt=-1), EINVAL), (dict(dyr=-1), EINVAL), (dict(gr=7), EINVAL), (dict(gr=-1), EINVAL), (dict(ws=P + 2), EINVAL),
    (dict(tokens=1 << 20, tr=1 << 23, dyr=1 << 23, dxr=1 << 23, mr=1 << 23, wsb=64), ESIZE),
    (dict(tokens=1 << 20, tr=1 << 23, dyr=1 << 23, dxr=1 << 23, mr=1 << 23, ws=None), ESIZE)], ids=str)
def test_rmsnorm_backward_refuses(kw, status):
    assert norm_backward(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(ids=T.F32), EINVAL), (dict(ranks=0), EINVAL), (dict(tokens=-1), EINVAL), (dict(k=0), EINVAL),
    (dict(experts=0), EINVAL), (dict(experts=4097), EUNSUPPORTED), (dict(tokens=1 << 30), EINVAL),
    (dict(chosen=None), EINVAL), (dict(offsets=None), EINVAL), (dict(places=None), EINVAL), (dict(ws=P + 1), EINVAL),
    (dict(tokens=1 << 20, wsb=64), ESIZE), (dict(tokens=1 << 20, ws=None), ESIZE)], ids=str)
def test_experts_sort_refuses(kw, status):
    assert sort(**kw) == status


BAD_ROWS = [dict(dtype=T.I32), dict(dtype=T.E4M3), dict(ranks=0), dict(tokens=-1), dict(k=0), dict(width=0),
            dict(width=1 << 25), dict(capacity=-1), dict(capacity=1 << 31), dict(rows=None), dict(places=None),
            dict(rr=-1), dict(rs=-1), dict(tokens=1 << 30), dict(ranks=1 << 40)]


@pytest.mark.parametrize("kw", BAD_ROWS + [dict(x=None), dict(xr=-1), dict(xt=-1), dict(rs=7), dict(rr=47),
                                           dict(rr=0), dict(rows=P)], ids=str)
def test_experts_dispatch_refuses(kw):
    assert dispatch(**kw) == EINVAL


@pytest.mark.parametrize("kw", BAD_ROWS + [dict(y=None), dict(yr=-1), dict(yt=7), dict(yr=8), dict(wtype=T.I32),
                                           dict(y=P)], ids=str)
def test_experts_combine_refuses(kw):
    assert combine(**kw) == EINVAL


@pytest.mark.parametrize("kw", BAD_ROWS + [dict(dy=None), dict(yr=-1), dict(drows=None), dict(dweights=None), dict(dr=47),
                                           dict(ds=7), dict(ds=-1), dict(wtype=9), dict(drows=P)], ids=str)
def test_experts_combine_backward_refuses(kw):
    assert gradient(**kw) == EINVAL


@pytest.mark.parametrize("kw", [
    dict(dtype=T.I32), dict(ttype=T.E4M3), dict(ids_type=T.F32), dict(ranks=0), dict(tokens=-1), dict(tokens=1 << 30),
    dict(width=0), dict(width=1 << 25), dict(vocab=0), dict(ids=None), dict(table=None), dict(y=None), dict(row=-1),
    dict(yr=-1), dict(yt=7), dict(yr=8), dict(row=1 << 60)], ids=str)
def test_embedding_forward_refuses(kw):
    assert lookup(**kw) == EINVAL


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=T.I32), EINVAL), (dict(ids_type=T.F32), EINVAL), (dict(ranks=0), EINVAL), (dict(tokens=-1), EINVAL),
    (dict(tokens=1 << 30), EINVAL), (dict(width=0), EINVAL), (dict(vocab=0), EINVAL),
    (dict(vocab=(1 << 24) + 1, tr=1 << 28), EUNSUPPORTED), (dict(dy=None), EINVAL), (dict(ids=None), EINVAL),
    (dict(dtable=None), EINVAL), (dict(dyr=-1), EINVAL), (dict(dyt=-1), EINVAL), (dict(tr=79), EINVAL),
    (dict(tr=-1), EINVAL), (dict(ws=None), ESIZE), (dict(wsb=16), ESIZE), (dict(ws=P + 2), EINVAL)], ids=str)
def test_embedding_backward_refuses(kw, status):
    assert table(**kw) == status


@pytest.mark.parametrize("kw", [
    dict(dtype=T.I32), dict(dtype=T.E4M3), dict(rate=-0.1), dict(rate=1.0), dict(rate=1.5), dict(rate=math.nan),
    dict(rate=1 - 2.0 ** -18), dict(ranks=0), dict(ranks=1 << 32), dict(tokens=-1), dict(tokens=1 << 32), dict(width=0),
    dict(width=1 << 25), dict(x=None), dict(y=None), dict(state=None), dict(state=P + 4), dict(xr=-1), dict(rt=-1),
    dict(yt=7), dict(yr=8)], ids=str)
def test_dropout_refuses(kw):
    assert dropout(**kw) == EINVAL


def test_nothing_to_do():
    assert norm(tokens=0, x=None, y=None) == OK
    assert norm_backward(tokens=0, dy=None, total=None, rstd=None, dx=None, dgamma=None) == OK
    assert dispatch(tokens=0, x=None, rows=None) == OK
    assert dispatch(capacity=0, rows=None) == OK
    assert combine(tokens=0, y=None) == OK
    assert gradient(tokens=0, dy=None) == OK
    assert lookup(tokens=0, y=None) == OK
    assert dropout(tokens=0, x=None, y=None, state=None) == OK


def test_workspace_sizes():
    assert T.trivance_rmsnorm_workspace_bytes(81, 1, 768) == 0
    # half of what the layer norm's two gradients take
    assert T.trivance_rmsnorm_workspace_bytes(1, 4096, 4096) * 2 == T.trivance_layernorm_workspace_bytes(1, 4096, 4096) > 0
    assert T.trivance_experts_workspace_bytes(9, 100, 2, 64) == 0
    assert T.trivance_experts_workspace_bytes(1, 1 << 20, 8, 4096) > 0
    # sorted keys and slots, twice in two passes, where each digit's run starts, and two parts of 32 pieces
    assert T.trivance_embedding_workspace_bytes(3, 1000, 64, 1000) >= 3 * (2 * 1000 + 1001 + 32 * 2 * 64) * 4
    assert T.trivance_embedding_workspace_bytes(3, 1000, 64, 50000) >= 3 * (4 * 1000 + 257 + 32 * 2 * 64) * 4
    for call, args in ((T.trivance_rmsnorm_workspace_bytes, (0, 1, 1)), (T.trivance_rmsnorm_workspace_bytes, (1, 1, 0)),
                       (T.trivance_experts_workspace_bytes, (1, 1, 0, 8)), (T.trivance_experts_workspace_bytes, (1, 1, 1, 0)),
                       (T.trivance_experts_workspace_bytes, (1, 1, 1, 4097)),
                       (T.trivance_embedding_workspace_bytes, (1, 1, 1, 0)),
                       (T.trivance_embedding_workspace_bytes, (1, 1, 1, 1 << 25))):
        with pytest.raises(T.TrivanceError):
            call(*args)


def test_binding_declares_the_arguments_of_the_header():
    """The ctypes signature of every function against the prototypes of the C header."""
    with open(os.path.join(os.path.dirname(T.__file__), "..", "include", "trivance.h")) as f:
        text = re.sub(r"/\*.*?\*/", "", f.read(), flags=re.S)
    kinds = {"int": ctypes.c_int, "int64_t": ctypes.c_int64, "double": ctypes.c_double, "uint64_t": ctypes.c_uint64,
             "unsigned": ctypes.c_uint}
    found = 0
    for name, params in re.findall(r"\b(trivance_(?:rmsnorm|experts|embedding|dropout)\w*)\s*\(([^)]*)\)", text):
        declared = getattr(_lib(), name).argtypes
        want = [ctypes.c_void_p if "*" in p else kinds[p.split()[0]] for p in params.split(",")]
        assert declared == want, name
        found += 1
    assert found == 12


def test_binding_refuses_host_tensors():
    torch = pytest.importorskip("torch")
    x, s = torch.zeros((2, 3, 8)), torch.zeros((2, 3))
    ids, i32 = torch.zeros((2, 3, 2), dtype=torch.int64), torch.zeros((2, 9), dtype=torch.int32)
    places, w = torch.zeros((2, 3, 2), dtype=torch.int32), torch.zeros((2, 3, 2))
    for call, args in ((T.trivance_rmsnorm_forward, (x, None, x)), (T.trivance_rmsnorm_backward, (x, x, None, s, x, None)),
                       (T.trivance_experts_sort, (ids, i32, places)), (T.trivance_experts_dispatch, (x, places, x)),
                       (T.trivance_experts_combine, (x, places, x)),
                       (T.trivance_experts_combine_backward, (x, x, places, w, x, w)),
                       (T.trivance_embedding_forward, (ids[..., 0], x[0], x)),
                       (T.trivance_embedding_backward, (x, ids[..., 0], x, s)),
                       (T.trivance_dropout, (x, x, ids[0, 0], 0.1))):
        with pytest.raises(TypeError):
            call(*args)


@pytest.mark.parametrize("counter,key,want", [
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
     (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))], ids=["zeros", "ones", "pi"])
def test_generator_gives_its_published_words(counter, key, want):
    """The plain generator that the kernel is held to, against the known answers of Philox-4x32 with ten
    rounds that its authors publish."""
    assert tuple(int(w) for w in more.philox(counter, key)) == want


def test_generator_keeps_the_share():
    for rate in (0.0, 0.1, 0.5, 0.9):
        share = more.kept((3, 200, 1001), 12345, 7, rate).mean()
        n = 3 * 200 * 1001
        assert abs(share - (1 - round(rate * 65536) / 65536)) <= 5 * math.sqrt(rate * (1 - rate) / n)
    a, b = more.kept((2, 9, 40), 5, 1, 0.5), more.kept((2, 9, 40), 5, 2, 0.5)
    assert (a != b).any() and np.array_equal(a, more.kept((2, 9, 40), 5, 1 + (1 << 32), 0.5))


@pytest.mark.parametrize("kw", [dict(total=P, tr=48), dict(total=P, tt=12, tr=36), dict(residual=8 * P, total=P, tr=48),
                                dict(x=8 * P, total=P, tr=48), dict(total=None, y=P, yr=48), dict(total=None, y=P, yt=9, yr=27),
                                dict(total=8 * P, x=9 * P, y=P, yr=48), dict(total=8 * P, y=P, ranks=1, yt=9),
                                dict(total=8 * P, y=P, tokens=1, yr=25)], ids=str)
def test_rmsnorm_forward_refuses_other_strides_in_place(kw):
    assert norm(**kw) == EINVAL


@pytest.mark.parametrize("kw", [dict(dxr=48), dict(dxt=9, dxr=27), dict(dx=Q, dy=Q, dxr=48), dict(dx=Q, total=Q, dxr=48),
                                dict(dx=Q, dtotal=Q, dxr=48), dict(ranks=1, dxt=9), dict(tokens=1, dxr=25)], ids=str)
def test_rmsnorm_backward_refuses_other_strides_in_place(kw):
    assert norm_backward(**kw) == EINVAL


@pytest.mark.parametrize("kw", [dict(dr=96), dict(ds=9, dr=54), dict(ranks=1, ds=9), dict(capacity=1, dr=96)], ids=str)
def test_experts_combine_backward_refuses_other_strides_in_place(kw):
    assert gradient(drows=Q, rows=Q, **kw) == EINVAL


@pytest.mark.parametrize("kw", [dict(yr=48), dict(yt=9, yr=27), dict(x=P, residual=Q, yr=48), dict(x=Q, residual=P, yr=48),
                                dict(x=Q, residual=None, yr=48), dict(ranks=1, yt=9), dict(tokens=1, yr=25)], ids=str)
def test_dropout_refuses_other_strides_in_place(kw):
    assert dropout(**{**dict(x=Q, residual=Q), **kw}) == EINVAL


@pytest.mark.parametrize("scale", [math.inf, -math.inf, math.nan, 1e39, -3.5e38], ids=str)
def test_embedding_refuses_scales_that_are_no_numbers(scale):
    """They would make NaN of the zeros of padding, and of sums that are zero."""
    assert lookup(scale=scale) == EINVAL
    assert table(scale=scale) == EINVAL


def test_embedding_refuses_outputs_in_place():
    """Rows of the table, or of dy, would be overwritten before they are read."""
    assert lookup(y=P, ttype=T.F32) == EINVAL
    assert table(dtable=P) == EINVAL
    assert table(dtable=P, ranks=1, tokens=200, dyr=1600) == EINVAL


def test_few_tokens_ask_for_no_parts():
    """The sums of pieces, two rows for each, are most of a workspace; up to 128 tokens of a rank have no pieces."""
    few = T.trivance_embedding_workspace_bytes(243, 128, 8192, 1000)
    assert 0 < few < 2 * 4 * (243 * (1000 + 1 + 2 * 128) + 12)
    assert T.trivance_embedding_workspace_bytes(243, 129, 8192, 1000) > 243 * 5 * 2 * 8192 * 4
