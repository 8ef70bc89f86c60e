"""Layer operators without a GPU: the library exports what include/bsr_layer_ops.h declares, invalid arguments are refused before
anything is launched, and the plain implementation that the GPU tests compare with has the gradients that differences of its own
forward pass give."""
import ctypes as C
import re
from pathlib import Path

import numpy as np
import pytest
import torch

import layer_plain as P
from paper_2311_16883_amd import binding as B

ROOT = Path(__file__).resolve().parent.parent


def test_library_exports_every_declared_layer_symbol():
    text = re.sub(r"/\*.*?\*/", "", (ROOT / "include" / "bsr_layer_ops.h").read_text(), flags=re.S)
    declared = set(re.findall(r"\b(bsr_[a-z_0-9]+)\s*\(", text))
    assert declared == set(B.LAYER_EXPORTS)
    for name in declared:
        assert getattr(B.lib(), name) is not None and callable(getattr(B, name))


FAKE, ODD = C.c_void_p(0x1000), C.c_void_p(0x1001)          # never dereferenced: validation fails first
FAR = C.c_void_p(0x100000)


def test_norm_refusals():
    lib, big = B.lib(), 1 << 31

    def norm(X=FAKE, dtype=0, M=4, D=16, ldx=16, gamma=FAKE, beta=FAKE, pt=0, eps=1e-5, Y=FAR, ldy=16, stats=FAKE):
        return lib.bsr_layer_norm(X, dtype, M, D, ldx, gamma, beta, pt, eps, Y, ldy, stats, None)
    assert norm(dtype=2) == norm(pt=-1) == B.BSR_ERR_DTYPE
    assert norm(ldx=15) == norm(ldy=15) == norm(M=-1) == norm(D=-1) == norm(M=big) == norm(D=big, ldx=big, ldy=big) == B.BSR_ERR_SHAPE
    assert norm(Y=FAKE, ldy=17) == B.BSR_ERR_SHAPE
    for eps in (0.0, -1.0, float("nan"), float("inf"), 1e-39):
        assert norm(eps=eps) == B.BSR_ERR_VALUE
    assert norm(X=None) == norm(Y=None) == B.BSR_ERR_NULL
    assert norm(X=ODD) == norm(Y=ODD) == norm(gamma=ODD) == norm(beta=ODD) == norm(stats=ODD) == B.BSR_ERR_ALIGN
    assert norm(gamma=C.c_void_p(0x1002)) == B.BSR_ERR_ALIGN and norm(M=0, X=None, Y=None) == norm(D=0, ldx=0, ldy=0) == B.BSR_OK

    def grad(X=FAKE, dtype=0, M=4, D=16, ldx=16, gamma=FAKE, pt=0, stats=FAKE, dY=FAKE, lddy=16, dX=FAR, lddx=16, dg=FAKE, db=FAKE,
             acc=0, ws=FAKE, nbytes=1 << 20):
        return lib.bsr_layer_norm_grad(X, dtype, M, D, ldx, gamma, pt, stats, dY, lddy, dX, lddx, dg, db, acc, ws, nbytes, None)
    assert grad(dtype=9) == grad(pt=9) == B.BSR_ERR_DTYPE
    assert grad(ldx=15) == grad(lddy=15) == grad(lddx=15) == grad(M=-1) == B.BSR_ERR_SHAPE
    assert grad(dX=FAKE, lddx=17) == grad(dX=FAKE, lddx=17, X=FAR) == B.BSR_ERR_SHAPE
    assert grad(X=None) == grad(stats=None) == grad(dY=None) == grad(dX=None) == B.BSR_ERR_NULL
    assert grad(X=ODD) == grad(dY=ODD) == grad(dX=ODD) == grad(dg=ODD) == grad(db=ODD) == grad(stats=ODD) == grad(ws=C.c_void_p(0x1008)) == B.BSR_ERR_ALIGN
    assert grad(ws=None) == grad(nbytes=8) == B.BSR_ERR_WORKSPACE
    assert grad(D=0, ldx=0, lddy=0, lddx=0) == grad(M=0, acc=1) == grad(M=0, dg=None, db=None, ws=None) == B.BSR_OK
    assert B.bsr_layer_norm_grad_workspace_bytes(0, 8) == B.bsr_layer_norm_grad_workspace_bytes(-1, 8) == 0
    assert B.bsr_layer_norm_grad_workspace_bytes(10, 8) >= 10 * 8 * 2 * 4 // 10


def test_gated_refusals():
    lib, big = B.lib(), 1 << 31

    def ff(X=FAKE, dtype=0, M=4, D=16, ldx=16, W=FAKE, F=8, ldw=16, act=0, H=FAR, ldh=8, GU=FAR, ldgu=16, ws=FAKE, nbytes=1 << 30):
        return lib.bsr_gated_ff(X, dtype, M, D, ldx, W, F, ldw, act, H, ldh, GU, ldgu, ws, nbytes, None)
    assert ff(dtype=2) == B.BSR_ERR_DTYPE
    assert ff(ldx=15) == ff(ldw=15) == ff(ldh=7) == ff(ldgu=15) == ff(M=-1) == ff(F=-1) == ff(M=big) == ff(F=1 << 30, ldw=big) == B.BSR_ERR_SHAPE
    wide = (1 << 20) + 2
    assert ff(D=wide, ldx=wide) == ff(F=wide // 2, ldw=wide, ldh=wide, ldgu=wide) == B.BSR_ERR_LIMIT
    assert ff(act=-1) == ff(act=4) == B.BSR_ERR_VALUE
    assert ff(X=None) == ff(W=None) == ff(H=None) == B.BSR_ERR_NULL
    assert ff(X=ODD) == ff(W=ODD) == ff(H=ODD) == ff(GU=ODD) == B.BSR_ERR_ALIGN
    assert ff(M=0, X=None, H=None) == ff(F=0, W=None, H=None) == B.BSR_OK
    need = lib.bsr_gated_ff_workspace_bytes(FAKE, 0, 4, 16, 16, FAKE, 8, 16)
    assert need == 0 or ff(nbytes=need - 1) == ff(ws=None) == B.BSR_ERR_WORKSPACE
    assert lib.bsr_gated_ff_workspace_bytes(FAKE, 7, 4, 16, 16, FAKE, 8, 16) == lib.bsr_gated_ff_workspace_bytes(FAKE, 0, 0, 16, 16, FAKE, 8, 16) == 0

    def grad(GU=FAKE, dtype=0, M=4, F=8, ldgu=16, dH=FAKE, lddh=8, act=0, W=FAKE, D=16, ldw=16, dGU=FAR, lddgu=16, dX=FAR, lddx=16, ws=FAKE,
             nbytes=1 << 30):
        return lib.bsr_gated_ff_grad(GU, dtype, M, F, ldgu, dH, lddh, act, W, D, ldw, dGU, lddgu, dX, lddx, ws, nbytes, None)
    assert grad(dtype=2) == grad(dtype=2, dX=None) == B.BSR_ERR_DTYPE
    assert grad(ldgu=15) == grad(lddh=7) == grad(ldw=15) == grad(lddgu=15) == grad(lddx=15) == grad(M=-1) == grad(dX=None, F=-1) == B.BSR_ERR_SHAPE
    assert grad(dGU=FAKE, lddgu=17) == B.BSR_ERR_SHAPE
    assert grad(act=4) == grad(act=4, dX=None) == B.BSR_ERR_VALUE
    assert grad(GU=None) == grad(dH=None) == grad(W=None) == grad(dGU=None) == B.BSR_ERR_NULL
    assert grad(GU=ODD) == grad(dH=ODD) == grad(W=ODD) == grad(dGU=ODD) == grad(dX=ODD) == B.BSR_ERR_ALIGN
    assert grad(M=0) == B.BSR_OK


class Options(C.Structure):
    _fields_ = [("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double), ("grad_scale", C.c_double),
                ("step", C.c_int64), ("seed", C.c_uint64), ("lr_device", C.c_void_p), ("grad_scale_device", C.c_void_p),
                ("step_device", C.c_void_p)]


def test_adamw_refusals():
    lib = B.lib()

    def call(n_items=1, pt=0, gt=0, moments=0, options=True, item=None, **numbers):
        o = Options(1e-3, 0.9, 0.999, 1e-8, 1.0, 1, 0, None, None, None)
        for k, v in numbers.items():
            setattr(o, k, v)
        it = B._AdamWItem(0x1000, 0x1000, 0x1000, 0x1000, 0x1000, None, 300, 3, 0.0)
        for k, v in (item or {}).items():
            setattr(it, k, v)
        return lib.bsr_adamw_batched(C.byref(it) if n_items else None, n_items, pt, gt, moments, C.byref(o) if options else None, None)
    assert call(pt=2) == call(gt=2) == call(moments=2) == B.BSR_ERR_DTYPE
    assert call(n_items=-1) == B.BSR_ERR_SHAPE and call(options=False) == B.BSR_ERR_NULL and call(n_items=0) == B.BSR_OK
    inf, nan = float("inf"), float("nan")
    for bad in (dict(lr=nan), dict(lr=inf), dict(lr=1e300), dict(beta1=1.0), dict(beta1=-0.1), dict(beta1=nan), dict(beta2=1.0), dict(beta2=2.0),
                dict(eps=0.0), dict(eps=-1.0), dict(eps=inf), dict(eps=nan), dict(grad_scale=inf), dict(step=0), dict(step=-3),
                dict(item=dict(weight_decay=nan))):
        assert call(**bad) == B.BSR_ERR_VALUE, bad
    for bad in (dict(n=-1), dict(n=(1 << 40) + 1)):
        assert call(item=bad) == B.BSR_ERR_SHAPE, bad
    assert call(moments=1, item=dict(scales_stride=2)) == B.BSR_ERR_SHAPE
    for name in ("param", "grad", "m", "v"):
        assert call(item={name: None}) == B.BSR_ERR_NULL and call(item={name: 0x1001}) == B.BSR_ERR_ALIGN
    assert call(moments=1, item=dict(scales=None)) == B.BSR_ERR_NULL and call(item=dict(copy=0x1001)) == B.BSR_ERR_ALIGN
    assert call(lr_device=0x1002) == call(step_device=0x1004) == call(grad_scale_device=0x1001) == B.BSR_ERR_ALIGN
    assert call(item=dict(n=0, param=None, m=None)) == B.BSR_OK
    assert [B.bsr_adamw_blocks(n) for n in (0, 1, 128, 129)] == [0, 1, 1, 2]
    with pytest.raises(B.BsrError):
        B.bsr_adamw_blocks(-1)

    def values(codes=FAKE, scales=FAKE, n=5, which=0, out=FAKE, dtype=0):
        return lib.bsr_adamw_state_values(codes, scales, n, which, out, dtype, None)
    assert values(dtype=3) == B.BSR_ERR_DTYPE and values(n=-1) == B.BSR_ERR_SHAPE and values(which=2) == B.BSR_ERR_VALUE
    assert values(codes=None) == values(scales=None) == values(out=None) == B.BSR_ERR_NULL and values(out=ODD) == B.BSR_ERR_ALIGN
    assert values(n=0, codes=None) == B.BSR_OK


@pytest.mark.parametrize("call", [lambda x: B.bsr_layer_norm(x), lambda x: B.bsr_layer_norm_grad(x, None, x, x),
                                  lambda x: B.bsr_gated_ff(x, x), lambda x: B.bsr_gated_ff_grad(x, x, x)])
def test_native_layer_calls_refuse_what_is_no_device_matrix(call):
    with pytest.raises(ValueError, match="2-D device tensor"):
        call(torch.zeros(4, 4))
    with pytest.raises(TypeError, match="must be a tensor"):
        call([[0.0]])


def test_adamw_batch_and_names_are_checked():
    x = torch.zeros(4)
    with pytest.raises(ValueError, match="on one device"):
        B.AdamWBatch([x], [x])
    for bad in (dict(params=[], grads=[]), dict(params=[x], grads=[]), dict(params=[x], grads=[x], bits=16), dict(params=[x], grads=[x], weight_decay=[1, 2]),
                dict(params=[x], grads=[x], states=[])):
        with pytest.raises(ValueError):
            B.AdamWBatch(**bad)
    with pytest.raises(B.BsrError):
        B.AdamWBatch([x.double()], [x])
    with pytest.raises(ValueError, match="which"):
        B.bsr_adamw_state_values(x, x, "v")
    with pytest.raises(ValueError, match="act must be"):
        B.bsr_gated_ff(x, x, act="tanh")


# ---- the plain implementation against differences of its own forward pass ----

def test_plain_norm_gradient_against_differences():
    rng = np.random.default_rng(0)
    x, gamma, beta, dy, h = rng.standard_normal((3, 7)), rng.standard_normal(7), rng.standard_normal(7), rng.standard_normal((3, 7)), 1e-6

    def loss(x, gamma, beta):
        return (P.layer_norm(x, gamma, beta, 1e-3)[0] * dy).sum()
    dx, _, dg, _, db, _ = P.layer_norm_grad(x, gamma, P.layer_norm(x, gamma, beta, 1e-3)[2], dy)
    for args, k, grad in (((x, gamma, beta), 0, dx), ((x, gamma, beta), 1, dg), ((x, gamma, beta), 2, db)):
        for i in np.ndindex(grad.shape):
            up, down = [a.copy() for a in args], [a.copy() for a in args]
            up[k][i] += h
            down[k][i] -= h
            assert abs((loss(*up) - loss(*down)) / (2 * h) - grad[i]) < 1e-7


@pytest.mark.parametrize("name", ["silu", "gelu", "gelu_tanh", "relu"])
def test_plain_gated_gradient_against_differences(name):
    rng = np.random.default_rng(1)
    x, w, dh, h = rng.standard_normal((4, 5)), rng.standard_normal((5, 6)), rng.standard_normal((4, 3)), 1e-6
    dgu, _ = P.gated_slopes(x @ w, dh, name)
    dx, dw = dgu @ w.T, x.T @ dgu

    def loss(x, w):
        return (P.gated(x, w, name, "bf16")[0] * dh).sum()
    for grad, k in ((dx, 0), (dw, 1)):
        for i in np.ndindex(grad.shape):
            up, down = [x.copy(), w.copy()], [x.copy(), w.copy()]
            up[k][i] += h
            down[k][i] -= h
            assert abs((loss(*up) - loss(*down)) / (2 * h) - grad[i]) < 1e-6


def test_plain_codes_cover_their_range_evenly():
    for bits in (3, 4):
        k = [P.magnitude(c, bits) for c in range(128 if bits == 3 else 256)]
        assert k[0] == 0 and k[1] == 1 and k[-1] == ((2 << bits) - 1) * 2.0 ** 14
        assert all(1.0 < b / a <= 1 + 2.0 ** -bits for a, b in zip(k[1 << bits:], k[(1 << bits) + 1:]))
        x = np.random.default_rng(2).lognormal(0, 3, 128)
        _, step = P.steps_of(x, bits)
        assert x.max() / step[x.argmax()] < (2 << bits)
    u, v = P.uniform(1 << 33, 1 << 18, 12345, 7)
    for z in (u, v, (u + 0.5 * v) % 1.0):
        assert abs(np.histogram(z, 64, (0, 1))[0] / 4096 - 1).max() < 0.1          # 4096 +- 64 in each: six of those
    assert abs(np.corrcoef(u, v)[0, 1]) < 0.012 and abs(np.corrcoef(u[1:], u[:-1])[0, 1]) < 0.012
