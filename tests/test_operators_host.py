"""The refusals of the operators around the AllReduce, through the C ABI and the binding, without a GPU:
every case here is turned away, or has nothing to do, before any kernel is launched."""

import ctypes
import math

import pytest

import paper_2602_17254_amd as T

OK, EINVAL, EUNSUPPORTED, ESIZE = 0, -1, -2, -5
P = 4096  # an address that is never followed


def _lib():
    return T.binding._lib()


def forward(**kw):
    a = dict(x=P, gamma=P, beta=P, y=P, mean=P, rstd=P, ranks=2, tokens=3, width=8, xr=24, xt=8, yr=24,
             yt=8, eps=1e-5, dtype=T.F32, wtype=T.F32, stream=None)
    a.update(kw)
    return _lib().trivance_layernorm_forward(*a.values())


def backward(**kw):
    a = dict(dy=P, x=P, gamma=P, mean=P, rstd=P, dx=P, dgamma=P, dbeta=P, ranks=2, tokens=3, width=8,
             dyr=24, dyt=8, xr=24, xt=8, dxr=24, dxt=8, gr=16, dtype=T.F32, wtype=T.F32, ws=P,
             wsb=1 << 40, stream=None)
    a.update(kw)
    return _lib().trivance_layernorm_backward(*a.values())


def counts(**kw):
    a = dict(logits=P, chosen=P, mask=None, counts=P, probs=P, ranks=2, tokens=3, experts=8, k=2, lr=24,
             lt=8, cr=9, pr=8, dtype=T.F32, ids=T.I32, ws=P, wsb=1 << 40, stream=None)
    a.update(kw)
    return _lib().trivance_balance_counts(*a.values())


def loss(**kw):
    a = dict(counts=P, probs=P, loss=P, ranks=2, experts=8, k=2, cr=9, pr=8, scale=1.0, stream=None)
    a.update(kw)
    return _lib().trivance_balance_loss(*a.values())


def gradient(**kw):
    a = dict(logits=P, counts=P, mask=None, dloss=None, dlogits=P, ranks=2, tokens=3, experts=8, k=2, lr=24,
             lt=8, dr=24, dt=8, cr=9, scale=1.0, dtype=T.F32, stream=None)
    a.update(kw)
    return _lib().trivance_balance_backward(*a.values())


def orthogonalize(k=((3.4445, -4.7750, 2.0315),) * 5, **kw):
    flat = [v for abc in k for v in abc]
    a = dict(x=P, out=P, batch=2, rows=70, cols=80, xb=5600, xr=80, ob=5600, orow=80,
             k=(ctypes.c_float * max(1, len(flat)))(*flat), steps=len(k), scale=1.0, eps=1e-7,
             dtype=T.F32, ws=P, wsb=1 << 40, stream=None)
    a.update(kw)
    return _lib().trivance_orthogonalize(*a.values())


@pytest.mark.parametrize("kw", [
    dict(dtype=T.I32), dict(dtype=9), dict(wtype=T.I64), dict(ranks=0), dict(tokens=-1), dict(width=0),
    dict(width=(1 << 24) + 1), dict(eps=-1.0), dict(eps=math.nan), dict(x=None), dict(y=None),
    dict(xr=-1), dict(xt=-8), dict(yr=-1), dict(yt=7), dict(yr=23), dict(yr=0), dict(yt=0),
    dict(xr=1 << 60), dict(ranks=1 << 40, tokens=1 << 40), dict(yr=8, yt=8)], ids=str)
def test_layernorm_forward_refuses(kw):
    assert forward(**kw) == EINVAL


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=T.I32), EINVAL), (dict(wtype=5), EINVAL), (dict(ranks=0), EINVAL), (dict(width=0), EINVAL),
    (dict(dy=None), EINVAL), (dict(x=None), EINVAL), (dict(mean=None), EINVAL), (dict(rstd=None), EINVAL),
    (dict(dx=None), EINVAL), (dict(dxt=4), EINVAL), (dict(gr=7), EINVAL), (dict(gr=-1), EINVAL),
    (dict(ws=P + 2), EINVAL), (dict(tokens=1 << 20, xr=1 << 23, dyr=1 << 23, dxr=1 << 23, wsb=64), ESIZE),
    (dict(tokens=1 << 20, xr=1 << 23, dyr=1 << 23, dxr=1 << 23, ws=None), ESIZE)], ids=str)
def test_layernorm_backward_refuses(kw, status):
    assert backward(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=T.I32), EINVAL), (dict(ids=T.F32), EINVAL), (dict(ranks=0), EINVAL), (dict(tokens=-1), EINVAL),
    (dict(experts=0), EINVAL), (dict(k=0), EINVAL), (dict(experts=4097), EUNSUPPORTED),
    (dict(tokens=1 << 30), EINVAL), (dict(logits=None), EINVAL), (dict(chosen=None), EINVAL),
    (dict(counts=None), EINVAL), (dict(probs=None), EINVAL), (dict(cr=8), EINVAL), (dict(pr=7), EINVAL),
    (dict(lt=-1), EINVAL), (dict(ws=P + 1), EINVAL), (dict(tokens=1 << 20, wsb=64), ESIZE),
    (dict(tokens=1 << 20, ws=None), ESIZE)], ids=str)
def test_balance_counts_refuses(kw, status):
    assert counts(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(ranks=0), EINVAL), (dict(experts=0), EINVAL), (dict(experts=5000), EUNSUPPORTED), (dict(k=0), EINVAL),
    (dict(counts=None), EINVAL), (dict(probs=None), EINVAL), (dict(loss=None), EINVAL),
    (dict(cr=-1), EINVAL)], ids=str)
def test_balance_loss_refuses(kw, status):
    assert loss(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=T.I64), EINVAL), (dict(ranks=-1), EINVAL), (dict(k=0), EINVAL), (dict(experts=5000), EUNSUPPORTED),
    (dict(logits=None), EINVAL), (dict(counts=None), EINVAL), (dict(dlogits=None), EINVAL), (dict(dt=7), EINVAL),
    (dict(dr=8), EINVAL), (dict(cr=-1), EINVAL), (dict(lr=-1), EINVAL)], ids=str)
def test_balance_backward_refuses(kw, status):
    assert gradient(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=T.I32), EINVAL), (dict(batch=-1), EINVAL), (dict(rows=-1), EINVAL), (dict(k=()), EINVAL),
    (dict(x=None), EINVAL), (dict(out=None), EINVAL), (dict(eps=-1.0), EINVAL), (dict(scale=math.inf), EINVAL),
    (dict(orow=79), EINVAL), (dict(ob=5599), EINVAL), (dict(xr=-80), EINVAL), (dict(wsb=64), ESIZE),
    (dict(ws=None), ESIZE), (dict(rows=1 << 17, xb=1 << 24, ob=1 << 24), EUNSUPPORTED),
    (dict(batch=1 << 16), EUNSUPPORTED), (dict(k=((1.0, 0.0, 0.0),) * 65), EUNSUPPORTED),
    (dict(k=((16.0, 0.0, 0.0),)), EUNSUPPORTED), (dict(k=((2.0, 0.0, 0.0),) * 3), EUNSUPPORTED),
    (dict(k=((math.nan, 0.0, 0.0),)), EUNSUPPORTED)], ids=str)
def test_orthogonalize_refuses(kw, status):
    assert orthogonalize(**kw) == status


def test_nothing_to_do():
    assert forward(tokens=0, x=None, y=None) == OK
    assert gradient(tokens=0, logits=None, dlogits=None) == OK
    for empty in ("batch", "rows", "cols"):
        assert orthogonalize(**{empty: 0}, x=None, out=None, ws=None, wsb=0) == OK


def test_workspace_sizes():
    assert T.trivance_layernorm_workspace_bytes(81, 1, 768) == 0
    assert T.trivance_layernorm_workspace_bytes(1, 4096, 4096) > 0
    assert T.trivance_balance_workspace_bytes(81, 1, 64) == 0
    assert T.trivance_orthogonalize_workspace_bytes(0, 5, 5) == 0
    # a step's matrices both ways round and twice, and the products of the smaller side
    assert T.trivance_orthogonalize_workspace_bytes(1, 2048, 512) >= 16 * 2048 * 512 + 8 * 512 * 512
    for call, args in ((T.trivance_layernorm_workspace_bytes, (0, 1, 1)),
                       (T.trivance_balance_workspace_bytes, (1, 1, 0)),
                       (T.trivance_balance_workspace_bytes, (1, 1, 9999)),
                       (T.trivance_orthogonalize_workspace_bytes, (1, -1, 1))):
        with pytest.raises(T.TrivanceError):
            call(*args)


def test_allreduce_still_takes_its_two_types():
    plan = T.trivance_plan((9,), "L")
    for dtype in (T.BF16, T.F16, T.I64):
        assert _lib().trivance_allreduce_emulated(P, 9, 64, dtype, plan.handle, None) == EINVAL
        assert _lib().trivance_workspace_bytes(plan.handle, 64, dtype) == EINVAL


def test_binding_refuses_host_tensors():
    torch = pytest.importorskip("torch")
    x = torch.zeros((2, 3, 8))
    row = torch.zeros((2, 8))
    c = torch.zeros((2, 9), dtype=torch.int32)
    with pytest.raises(TypeError):
        T.trivance_layernorm_forward(x, None, None, x)
    with pytest.raises(TypeError):
        T.trivance_layernorm_backward(x, x, None, row, row, x, row, row)
    with pytest.raises(TypeError):
        T.trivance_balance_counts(x, c, c, row)
    with pytest.raises(TypeError):
        T.trivance_balance_loss(c, row, 2, row[0])
    with pytest.raises(TypeError):
        T.trivance_balance_backward(x, c, 2, x)
    with pytest.raises(TypeError):
        T.trivance_orthogonalize(x, x, None)


@pytest.mark.parametrize("scale", [1e39, -1e300, math.nan, -math.inf])
def test_orthogonalize_refuses_scales_that_fp32_does_not_hold(scale):
    assert orthogonalize(scale=scale) == EINVAL


@pytest.mark.parametrize("size,shared", [((1, 512, 512), 0), ((4, 256, 512), 0), ((1, 2048, 8192), 136 + 256),
                                         ((64, 256, 768), 0)], ids=str)
def test_orthogonalize_workspace_holds_what_the_call_uses(size, shared):
    """X both ways round twice and two products of its smaller side, in two fp16 numbers; where symmetric products
    are shared (tiles of 128 here), a part for each tile and worker; norms and coefficients."""
    b, m, n = size
    need = b * (16 * m * n + 8 * m * m) + 4 * shared * 128 * 128
    got = T.trivance_orthogonalize_workspace_bytes(*size)
    assert need <= got <= need + b * (1024 * 8 + 16) + 4096
