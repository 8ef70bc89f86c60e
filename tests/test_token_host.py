"""Token operators without a GPU: the library exports what include/bsr_token_step.h declares, the host functions agree with
the definitions, invalid arguments are refused before anything is launched, and the plain implementation that the GPU tests
compare with has the gradients that differences of its own forward pass give."""
import ctypes as C
import itertools
import re
from pathlib import Path

import numpy as np
import pytest
import torch

import token_plain as P
from paper_2311_16883_amd import binding as B

ROOT = Path(__file__).resolve().parent.parent


def test_library_exports_every_declared_token_symbol():
    text = re.sub(r"/\*.*?\*/", "", (ROOT / "include" / "bsr_token_step.h").read_text(), flags=re.S)
    declared = set(re.findall(r"\b(bsr_[a-z_0-9]+)\s*\(", text))
    assert declared == set(B.TOKEN_EXPORTS)
    for name in declared:
        assert getattr(B.lib(), name) is not None and callable(getattr(B, name))
    assert B.lib().bsr_error_string(B.BSR_ERR_VALUE) == b"BSR_ERR_VALUE"


def test_capacity_is_the_most_that_any_routing_needs():
    for n, E, align in itertools.product(range(0, 8), range(1, 4), range(1, 6)):
        need = 0
        for counts in itertools.product(range(n + 1), repeat=E):
            if sum(counts) <= n:
                need = max(need, sum(-(-c // align) * align for c in counts))
        assert B.bsr_expert_capacity(n, E, align) == need == P.capacity(n, E, align)
    for bad in [(-1, 4, 1), (4, 0, 1), (4, 4, 0), (2 ** 31, 4, 1), (1000, 1000, 2 ** 30)]:
        assert B.lib().bsr_expert_capacity(*bad) == -1
        with pytest.raises(B.BsrError):
            B.bsr_expert_capacity(*bad)


def test_workspaces():
    assert B.bsr_embedding_grad_workspace_bytes(0, 1000, 64) == 0
    assert B.bsr_embedding_grad_workspace_bytes(-1, 1000, 64) == 0
    assert B.bsr_embedding_grad_workspace_bytes(10, 2 ** 30, 64) == 0
    assert B.bsr_embedding_grad_workspace_bytes(10000, 1000, 64) >= 8 * 10000
    assert B.bsr_expert_sort_workspace_bytes(100, 8) == 0
    assert B.bsr_expert_sort_workspace_bytes(1 << 20, 8) > 0
    assert B.bsr_expert_sort_workspace_bytes(1 << 20, 1025) == 0
    assert B.bsr_distill_workspace_bytes(0, 1000, 4) == 0
    assert B.bsr_distill_workspace_bytes(10, 1000, 4) >= 10 * 8
    assert B.bsr_distill_workspace_bytes(10, 1000, 1025) == 0


FAKE, ODD = C.c_void_p(0x1000), C.c_void_p(0x1001)          # never dereferenced: validation fails first


def test_invalid_arguments_are_refused_on_the_host():
    lib, big = B.lib(), 1 << 40

    def lookup(table=FAKE, dtype=0, V=8, D=16, ldt=16, tokens=FAKE, index=0, T=4, scale=1.0, out=FAKE, ldo=16):
        return lib.bsr_embedding_lookup(table, dtype, V, D, ldt, tokens, index, T, scale, out, ldo, None)
    assert lookup(dtype=2) == B.BSR_ERR_DTYPE and lookup(index=2) == B.BSR_ERR_DTYPE
    assert lookup(ldt=15) == lookup(ldo=15) == lookup(T=-1) == lookup(V=-1) == lookup(T=big) == B.BSR_ERR_SHAPE
    assert lookup(scale=float("nan")) == lookup(scale=float("inf")) == B.BSR_ERR_VALUE
    assert lookup(table=None) == lookup(tokens=None) == lookup(out=None) == B.BSR_ERR_NULL
    assert lookup(table=ODD) == lookup(out=ODD) == lookup(tokens=ODD) == B.BSR_ERR_ALIGN
    assert lookup(tokens=C.c_void_p(0x1004), index=1) == B.BSR_ERR_ALIGN
    assert lookup(T=0, tokens=None, out=None) == lookup(D=0, ldt=0, ldo=0) == B.BSR_OK

    def grad(tokens=FAKE, index=0, T=4, dY=FAKE, dtype=1, D=16, lddy=16, scale=1.0, V=8, dE=FAKE, ldde=16, acc=0, ws=FAKE,
             nbytes=1 << 20):
        return lib.bsr_embedding_grad(tokens, index, T, dY, dtype, D, lddy, scale, V, dE, ldde, acc, ws, nbytes, None)
    assert grad(dtype=7) == grad(index=-1) == B.BSR_ERR_DTYPE
    assert grad(lddy=15) == grad(ldde=15) == grad(T=-1) == grad(V=1 << 30) == B.BSR_ERR_SHAPE
    assert grad(scale=float("-inf")) == B.BSR_ERR_VALUE
    assert grad(tokens=None) == grad(dY=None) == grad(dE=None) == B.BSR_ERR_NULL
    assert grad(dE=C.c_void_p(0x1002)) == grad(dY=ODD) == grad(ws=C.c_void_p(0x1008)) == B.BSR_ERR_ALIGN
    assert grad(ws=None) == grad(nbytes=8) == B.BSR_ERR_WORKSPACE
    assert grad(V=0, dE=None) == grad(T=0, acc=1) == B.BSR_OK

    def sort(ids=FAKE, index=0, n=8, E=4, align=1, offsets=FAKE, counts=FAKE, order=FAKE, slots=FAKE, ws=None, nbytes=0):
        return lib.bsr_expert_sort(ids, index, n, E, align, offsets, counts, order, slots, ws, nbytes, None)
    assert sort(index=3) == B.BSR_ERR_DTYPE
    assert sort(n=-1) == sort(E=0) == sort(align=0) == sort(n=1 << 31) == B.BSR_ERR_SHAPE
    assert sort(E=1025) == B.BSR_ERR_LIMIT
    assert sort(ids=None) == sort(offsets=None) == sort(counts=None) == sort(order=None) == sort(slots=None) == B.BSR_ERR_NULL
    assert sort(ids=ODD) == sort(order=ODD) == B.BSR_ERR_ALIGN
    assert sort(n=1 << 20) == B.BSR_ERR_WORKSPACE

    def gather(X=FAKE, dtype=0, T=4, D=16, ldx=16, slots=FAKE, k=2, order=FAKE, rows=8, Xs=FAKE, ldxs=16):
        return lib.bsr_expert_gather(X, dtype, T, D, ldx, slots, k, order, rows, Xs, ldxs, None)
    assert gather(dtype=5) == B.BSR_ERR_DTYPE
    assert gather(ldx=15) == gather(ldxs=15) == gather(k=-1) == gather(rows=-1) == gather(T=1 << 30, k=8) == B.BSR_ERR_SHAPE
    assert gather(X=None) == gather(slots=None) == gather(order=None) == gather(Xs=None) == B.BSR_ERR_NULL
    assert gather(X=ODD) == gather(slots=ODD) == B.BSR_ERR_ALIGN

    def combine(Ys=FAKE, dtype=0, rows=8, D=16, ldys=16, slots=FAKE, T=4, k=2, w=None, out=FAKE, ldo=16):
        return lib.bsr_expert_combine(Ys, dtype, rows, D, ldys, slots, T, k, w, out, ldo, None)
    assert combine(dtype=5) == B.BSR_ERR_DTYPE
    assert combine(ldys=15) == combine(ldo=15) == combine(T=-1) == B.BSR_ERR_SHAPE
    assert combine(Ys=None) == combine(slots=None) == combine(out=None) == B.BSR_ERR_NULL
    assert combine(w=ODD) == combine(out=ODD) == B.BSR_ERR_ALIGN

    def cgrad(Ys=FAKE, dtype=0, rows=8, D=16, ldys=16, slots=FAKE, order=FAKE, T=4, k=2, w=FAKE, dOut=FAKE, lddo=16, dYs=FAKE,
              lddys=16, dw=FAKE):
        return lib.bsr_expert_combine_grad(Ys, dtype, rows, D, ldys, slots, order, T, k, w, dOut, lddo, dYs, lddys, dw, None)
    assert cgrad(dtype=5) == B.BSR_ERR_DTYPE
    assert cgrad(ldys=15) == cgrad(lddo=15) == cgrad(lddys=15) == B.BSR_ERR_SHAPE
    assert cgrad(Ys=None) == cgrad(slots=None) == cgrad(order=None) == cgrad(w=None) == cgrad(dOut=None) == B.BSR_ERR_NULL
    assert cgrad(dYs=None) == cgrad(dw=None) == B.BSR_ERR_NULL
    assert cgrad(dw=ODD) == cgrad(dOut=ODD) == B.BSR_ERR_ALIGN

    def loss(z=FAKE, dtype=0, N=4, V=16, ldz=16, ids=FAKE, index=0, t=FAKE, tt=0, K=2, tau=1.0, out=FAKE, stats=FAKE, ws=FAKE,
             nbytes=1 << 20):
        return lib.bsr_distill_loss(z, dtype, N, V, ldz, ids, index, t, tt, K, tau, out, stats, ws, nbytes, None)

    def dgrad(z=FAKE, dtype=0, N=4, V=16, ldz=16, ids=FAKE, index=0, t=FAKE, tt=0, K=2, tau=1.0, stats=FAKE, dloss=FAKE,
              out=FAKE, ldd=16):
        return lib.bsr_distill_grad(z, dtype, N, V, ldz, ids, index, t, tt, K, tau, stats, dloss, out, ldd, None)

    def both(z=FAKE, dtype=0, N=4, V=16, ldz=16, ids=FAKE, index=0, t=FAKE, tt=0, K=2, tau=1.0, dloss=FAKE, loss=FAKE,
             out=C.c_void_p(0x2000), ldd=16, ws=FAKE, nbytes=1 << 20):
        return lib.bsr_distill_loss_grad(z, dtype, N, V, ldz, ids, index, t, tt, K, tau, dloss, loss, out, ldd, ws, nbytes, None)
    for call in (loss, dgrad, both):
        assert call(dtype=5) == call(index=5) == call(tt=5) == B.BSR_ERR_DTYPE
        assert call(ldz=15) == call(N=-1) == call(V=-1) == call(K=-1) == call(V=1 << 31, ldz=1 << 31) == B.BSR_ERR_SHAPE
        assert call(K=1025) == B.BSR_ERR_LIMIT
        for tau in (0.0, -1.0, float("nan"), float("inf"), 1e-30):
            assert call(tau=tau) == B.BSR_ERR_VALUE
        assert call(z=None) == call(ids=None) == call(t=None) == call(out=None) == B.BSR_ERR_NULL
        assert call(z=ODD) == call(ids=ODD) == call(t=ODD) == call(out=ODD) == B.BSR_ERR_ALIGN
        assert call(N=0) == B.BSR_OK
    assert loss(stats=None) == dgrad(stats=None) == dgrad(dloss=None) == both(dloss=None) == both(loss=None) == B.BSR_ERR_NULL
    assert loss(ws=None) == loss(nbytes=4) == both(ws=None) == both(nbytes=4) == B.BSR_ERR_WORKSPACE
    assert dgrad(ldd=15) == both(ldd=15) == B.BSR_ERR_SHAPE
    assert dgrad(out=FAKE, ldd=17) == both(out=FAKE, ldd=17) == B.BSR_ERR_SHAPE       # in place, with another pitch


@pytest.mark.parametrize("call", [
    lambda x: B.bsr_embedding_lookup(x, x), lambda x: B.bsr_embedding_grad(x, x, 4), lambda x: B.bsr_expert_gather(x, x, x),
    lambda x: B.bsr_expert_combine(x, x), lambda x: B.bsr_expert_combine_grad(x, x, x, x, x),
    lambda x: B.bsr_distill_loss(x, x, x), lambda x: B.bsr_distill_grad(x, x, x, x, x),
    lambda x: B.bsr_distill_loss_grad(x, x, x, x),
])
def test_native_token_calls_refuse_what_is_no_device_matrix(call):
    with pytest.raises(ValueError, match="2-D device tensor"):
        call(torch.zeros(4, 4))
    with pytest.raises(TypeError, match="must be a tensor"):
        call([[0.0]])


def test_native_sort_refuses_host_tensors():
    with pytest.raises(ValueError, match="device"):
        B.bsr_expert_sort(torch.zeros(4, dtype=torch.int32), 4)
    with pytest.raises(TypeError, match="must be a tensor"):
        B.bsr_expert_sort([1, 2], 4)


# ---- the plain implementation against differences of its own forward pass ----

def test_plain_gradients_against_differences():
    rng = np.random.default_rng(0)
    h = 1e-5
    # table: linear, so differences are exact up to rounding
    table, tokens, dY = rng.standard_normal((7, 5)), np.array([3, 0, 3, -1, 6, 9, 3]), rng.standard_normal((7, 5))
    dE, _ = P.table_grad(tokens, dY, 7, 1.5)
    for v in range(7):
        for d in range(5):
            up, down = table.copy(), table.copy()
            up[v, d] += h
            down[v, d] -= h
            diff = ((P.lookup(up, tokens, 1.5) - P.lookup(down, tokens, 1.5)) * dY).sum() / (2 * h)
            assert abs(diff - dE[v, d]) < 1e-8
    # experts
    ids = np.array([[2, 0], [1, -1], [2, 1]])
    offsets, counts, order, slots = P.sort_by_expert(ids, 3, 4)
    Ys, w, dOut = rng.standard_normal((len(order), 4)), rng.random((3, 2)), rng.standard_normal((3, 4))
    dYs, dw, _ = P.combine_grad(Ys, slots, order, w, dOut)
    for s in range(len(order)):
        for d in range(4):
            up, down = Ys.copy(), Ys.copy()
            up[s, d] += h
            down[s, d] -= h
            diff = ((P.combine(up, slots, w)[0] - P.combine(down, slots, w)[0]) * dOut).sum() / (2 * h)
            assert abs(diff - dYs[s, d]) < 1e-8
    for t in range(3):
        for j in range(2):
            up, down = w.copy(), w.copy()
            up[t, j] += h
            down[t, j] -= h
            diff = ((P.combine(Ys, slots, up)[0] - P.combine(Ys, slots, down)[0]) * dOut).sum() / (2 * h)
            assert abs(diff - dw[t, j]) < 1e-8
    X = rng.standard_normal((3, 4))
    dXs = rng.standard_normal((len(order), 4))
    dX, _ = P.combine(dXs, slots, None)
    assert abs((P.gather(X, order, 2) * dXs).sum() - (X * dX).sum()) < 1e-12
    # loss
    z, t, tau = rng.standard_normal((3, 9)), rng.standard_normal((3, 4)), 1.7
    ids, dloss = np.array([[0, 3, 3, 8], [1, -1, 9, 2], [-1, -1, 12, -5]]), np.array([0.5, 2.0, 1.0])
    t[0, 0] = -np.inf
    z[1, 5] = -np.inf
    loss, _, grad, _, _ = P.distill(z, ids, t, tau, dloss)
    assert loss[2] == 0 and not grad[2].any() and (loss[:2] > 0).all()
    for n in range(3):
        for v in range(9):
            if np.isinf(z[n, v]):
                assert grad[n, v] == 0
                continue
            up, down = z.copy(), z.copy()
            up[n, v] += h
            down[n, v] -= h
            diff = ((P.distill(up, ids, t, tau, dloss)[0] - P.distill(down, ids, t, tau, dloss)[0]) * dloss).sum() / (2 * h)
            assert abs(diff - grad[n, v]) < 1e-7
