"""Host-only checks of the calls for 8-bit layers and of what stands around a layer: bad arguments are refused before any GPU work
is attempted, and the callable objects behave like the others."""
import copy
import inspect
import pickle
import weakref

import numpy as np
import pytest

import paper_2406_11235_amd as q
from paper_2406_11235_amd import binding

buf = np.zeros(4096 + 64, dtype=np.uint8)
P = buf.ctypes.data + (-buf.ctypes.data) % 256  # 256-byte aligned; never dereferenced

QUANTIZE = dict(x=P, up=None, type=q.F16, rows=2, n=64, ldx=64, signs=None, block=0, q=P, ldq=64, scale=P)
MATMUL = dict(W=P, ldw=64, w_scale=P, m=5, n=50, X=P, ldx=64, x_scale=P, B=3, bias=None, Y=P, ldy=5, y_type=q.F32, workspace=P,
              workspace_bytes=1 << 40)
NORM = dict(y=P, ldy=64, y_type=q.F16, h=P, ldh=64, h_type=q.F16, gate=None, ldgate=0, rows=2, n=64, norm=q.NORM_RMS,
            post_weight=P, post_bias=None, pre_weight=P, pre_bias=None, eps=1e-6, res_scale=1.0, signs=None, block=0, h_out=P,
            x=P, ldx=64, x_type=q.F16, x_scale=None)
MOE = dict(x=P, ldx=64, type=q.BF16, T=2, n=64, router=P, router_bias=None, E=8, top_k=2, renormalize=1, W_up=P, up_scale=P,
           f=32, W_down=P, down_scale=P, y=P, ldy=64, ids=None, weights=None, workspace=P, workspace_bytes=1 << 40)
EINVAL, EUNSUPPORTED = -1, -2


def refused(entry, base, code, **change):
    with pytest.raises(q.QtipError) as e:
        entry(**{**base, **change}, stream=0)
    assert e.value.code == code, (change, str(e.value))
    assert entry.__name__ in str(e.value)


@pytest.mark.parametrize("code,change", [
    (EINVAL, dict(x=None)), (EINVAL, dict(q=None)), (EINVAL, dict(scale=None)), (EUNSUPPORTED, dict(type=q.I8)),
    (EUNSUPPORTED, dict(type=9)), (EINVAL, dict(rows=0)), (EINVAL, dict(n=0)), (EINVAL, dict(n=-4)), (EINVAL, dict(n=32769, ldx=32769, ldq=32769)),
    (EINVAL, dict(ldx=63)), (EINVAL, dict(ldq=63)), (EINVAL, dict(ldx=-64)), (EINVAL, dict(x=P + 1)), (EINVAL, dict(up=P + 1)),
    (EINVAL, dict(scale=P + 2)), (EINVAL, dict(signs=P, block=8)), (EINVAL, dict(signs=P, block=48)), (EINVAL, dict(signs=P, block=128)),
    (EINVAL, dict(signs=P, block=0)), (EINVAL, dict(signs=P + 2, block=64)), (EINVAL, dict(signs=P, block=32768, n=32768, ldx=32768, ldq=32768))])
def test_quantize_rows_refuses(code, change):
    refused(q.qtip_quantize_rows_i8, QUANTIZE, code, **change)


@pytest.mark.parametrize("code,change", [
    (EINVAL, dict(W=None)), (EINVAL, dict(X=None)), (EINVAL, dict(Y=None)), (EINVAL, dict(w_scale=None)), (EINVAL, dict(x_scale=None)),
    (EUNSUPPORTED, dict(y_type=q.I8)), (EINVAL, dict(m=0)), (EINVAL, dict(n=0)), (EINVAL, dict(B=0)), (EINVAL, dict(B=-1)),
    (EINVAL, dict(n=131072, ldw=131072, ldx=131072)), (EINVAL, dict(B=65535 * 16 + 1)), (EINVAL, dict(m=(1 << 28) + 1, ldy=1 << 29)), (EINVAL, dict(ldw=(1 << 24) + 16)), (EINVAL, dict(ldx=(1 << 24) + 16)), (EINVAL, dict(ldw=48)), (EINVAL, dict(ldx=48)),
    (EINVAL, dict(ldy=4)), (EINVAL, dict(ldw=72)), (EINVAL, dict(ldx=56)), (EINVAL, dict(W=P + 8)), (EINVAL, dict(X=P + 1)),
    (EINVAL, dict(Y=P + 2)), (EINVAL, dict(bias=P + 2)), (EINVAL, dict(w_scale=P + 1)), (EINVAL, dict(x_scale=P + 3))])
def test_matmul_refuses(code, change):
    refused(q.qtip_matmul_i8, MATMUL, code, **change)


def test_matmul_workspace():
    assert q.qtip_matmul_i8_workspace(0, 16, 1) == q.qtip_matmul_i8_workspace(16, 0, 1) == q.qtip_matmul_i8_workspace(16, 16, 0) == 0
    assert q.qtip_matmul_i8_workspace(16, 131072, 1) == 0
    for m, n, B in ((64, 131071, 3), (4096, 14336, 48), (4096, 14336, 130), (512, 28672, 256), (8192, 8192, 64)):
        need = q.qtip_matmul_i8_workspace(m, n, B)
        sizes = dict(m=m, n=n, B=B, ldw=1 << 17, ldx=1 << 17, ldy=m)
        if need:
            refused(q.qtip_matmul_i8, MATMUL, EINVAL, workspace=None, **sizes)
            refused(q.qtip_matmul_i8, MATMUL, EINVAL, workspace=P + 128, **sizes)
            refused(q.qtip_matmul_i8, MATMUL, EINVAL, workspace_bytes=need - 1, **sizes)


@pytest.mark.parametrize("code,change", [
    (EINVAL, dict(y=None, h=None)), (EINVAL, dict(h_out=None, x=None, pre_weight=None)), (EUNSUPPORTED, dict(norm=2)),
    (EUNSUPPORTED, dict(y_type=q.I8)), (EUNSUPPORTED, dict(h_type=q.BF16)), (EUNSUPPORTED, dict(y_type=q.F32)),
    (EINVAL, dict(rows=0)), (EINVAL, dict(n=0)), (EINVAL, dict(n=32769, ldy=32769, ldh=32769, ldx=32769)),
    (EINVAL, dict(y=None)), (EINVAL, dict(y=None, post_weight=None, gate=P)), (EINVAL, dict(post_weight=None, post_bias=P)),
    (EINVAL, dict(pre_weight=None, pre_bias=P)), (EINVAL, dict(ldy=63)), (EINVAL, dict(ldh=63)), (EINVAL, dict(gate=P, ldgate=63)),
    (EINVAL, dict(ldx=63)), (EUNSUPPORTED, dict(x_type=4)), (EINVAL, dict(x_type=q.I8)), (EINVAL, dict(x_type=q.I8, x_scale=P + 1)),
    (EINVAL, dict(x=None)), (EINVAL, dict(x=None, pre_weight=None, signs=P, block=64)), (EINVAL, dict(signs=P, block=128)),
    (EINVAL, dict(eps=-1e-6)), (EINVAL, dict(eps=float("nan"))), (EINVAL, dict(y=P + 1)), (EINVAL, dict(h_out=P + 1)),
    (EINVAL, dict(post_weight=P + 2)), (EINVAL, dict(x=P + 1))])
def test_norm_residual_refuses(code, change):
    refused(q.qtip_norm_residual, NORM, code, **change)


@pytest.mark.parametrize("code,change", [
    (EINVAL, dict(x=None)), (EINVAL, dict(router=None)), (EINVAL, dict(W_up=None)), (EINVAL, dict(up_scale=None)),
    (EINVAL, dict(W_down=None)), (EINVAL, dict(down_scale=None)), (EINVAL, dict(y=None)), (EINVAL, dict(workspace=None)),
    (EUNSUPPORTED, dict(type=q.F32)), (EINVAL, dict(T=0)), (EINVAL, dict(T=65)), (EINVAL, dict(E=0)), (EINVAL, dict(E=257)),
    (EINVAL, dict(top_k=0)), (EINVAL, dict(top_k=9)), (EINVAL, dict(top_k=17, E=64)), (EINVAL, dict(n=56)), (EINVAL, dict(f=24)),
    (EINVAL, dict(f=0)), (EINVAL, dict(n=0)), (EINVAL, dict(n=32784, ldx=32784, ldy=32784)), (EINVAL, dict(f=32784)),
    (EINVAL, dict(ldx=56)), (EINVAL, dict(ldy=63)), (EINVAL, dict(ldx=68)), (EINVAL, dict(ldx=(1 << 24) + 8)), (EINVAL, dict(x=P + 8)), (EINVAL, dict(router=P + 8)),
    (EINVAL, dict(W_up=P + 4)), (EINVAL, dict(W_down=P + 4)), (EINVAL, dict(up_scale=P + 4)), (EINVAL, dict(down_scale=P + 8)),
    (EINVAL, dict(y=P + 1)), (EINVAL, dict(ids=P + 2)), (EINVAL, dict(weights=P + 2)), (EINVAL, dict(router_bias=P + 2)),
    (EINVAL, dict(workspace=P + 64)), (EINVAL, dict(workspace_bytes=q.qtip_moe_i8_workspace(2, 64, 32, 8, 2) - 1))])
def test_moe_refuses(code, change):
    refused(q.qtip_moe_i8, MOE, code, **change)


def test_moe_workspace():
    assert q.qtip_moe_i8_workspace(1, 16, 16, 1, 1) > 0
    for wrong in ((0, 16, 16, 1, 1), (65, 16, 16, 1, 1), (1, 16, 16, 257, 1), (1, 16, 16, 4, 5), (1, 16, 0, 1, 1), (1, 0, 16, 1, 1)):
        assert q.qtip_moe_i8_workspace(*wrong) == 0
    assert q.qtip_moe_i8_workspace(64, 4096, 32768, 256, 16) < 1 << 30


@pytest.mark.parametrize("name,base", [("qtip_quantize_rows_i8", QUANTIZE), ("qtip_matmul_i8", MATMUL),
                                       ("qtip_norm_residual", NORM), ("qtip_moe_i8", MOE)])
def test_entry_points_are_like_functions(name, base):
    assert name in binding._LAYER_ENTRIES
    f = getattr(q, name)
    assert (f.__name__, f.__qualname__, f.__module__) == (name, name, binding.__name__) and f.__doc__
    assert pickle.loads(pickle.dumps(f)) is f and copy.copy(f) is f and weakref.ref(f)() is f
    parameters = inspect.signature(f).parameters
    assert list(parameters) == list(base) + ["stream"]
    assert [p.name for p in parameters.values() if p.default is not p.empty] == ["stream"]
    with pytest.raises(q.QtipError):
        f(*[0] * len(parameters))
    with pytest.raises(TypeError, match="at most"):
        f(*[None] * 28)
    with pytest.raises(TypeError, match="unexpected keyword"):
        f(nonsense=1)
    for p in base:
        with pytest.raises(TypeError, match=f"missing required argument '{p}'"):
            f(**{o: 0 for o in parameters if o != p})


def test_real_arguments():
    refused(q.qtip_norm_residual, NORM, EINVAL, eps=-1)                     # a whole number is one
    refused(q.qtip_norm_residual, NORM, EINVAL, eps=np.float64(-0.5))
    with pytest.raises(TypeError):
        q.qtip_norm_residual(**{**NORM, "eps": "1e-6"}, stream=0)
