"""Layer operators on tensors so large that they are read and written past the caches: rows and elements do not depend on each other, so
they have to come out as in smaller calls, bit for bit; sums over rows within the bounds of the plain implementation."""
import pytest
import torch

import layer_plain as P
from paper_2311_16883_amd import binding as B

pytestmark = pytest.mark.gpu


def randn(seed, *size, dtype):
    return torch.randn(*size, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda", dtype=torch.float32).to(dtype)


@pytest.mark.parametrize("dtype,M,D", [(torch.bfloat16, 40009, 1024), (torch.bfloat16, 9001, 4096), (torch.float32, 20011, 1024),
                                       (torch.float32, 70001, 256)])
@pytest.mark.parametrize("in_place", [False, True])
def test_norm(dtype, M, D, in_place):
    x, dy = randn(1, M, D, dtype=dtype), randn(2, M, D, dtype=dtype)
    gamma, beta = randn(3, D, dtype=torch.float32), randn(4, D, dtype=torch.float32)
    parts = list(zip(x.clone().split(M // 9), dy.clone().split(M // 9)))
    y, stats = B.bsr_layer_norm(x.clone() if in_place else x, gamma, beta, want_stats=True)
    if in_place:
        z = x.clone()
        B.bsr_layer_norm(z, gamma, beta, Y=z)
        assert torch.equal(y, z)
        dx, dgamma, dbeta = B.bsr_layer_norm_grad(x, gamma, stats, dy, dX=dy)
    else:
        dx, dgamma, dbeta = B.bsr_layer_norm_grad(x, gamma, stats, dy)
    row = 0
    sums = torch.zeros(4, D, dtype=torch.float64, device="cuda")
    for px, py in parts:
        at = slice(row, row + px.shape[0])
        y1, stats1 = B.bsr_layer_norm(px, gamma, beta, want_stats=True)
        assert torch.equal(y[at], y1) and torch.equal(stats[at], stats1)
        assert torch.equal(dx[at], B.bsr_layer_norm_grad(px, gamma, stats1, py)[0])
        g = py.double() * ((px.double() - stats1[:, :1].double()) * stats1[:, 1:].double())
        sums += torch.stack((g.sum(dim=0), py.double().sum(dim=0), g.abs().sum(dim=0), py.double().abs().sum(dim=0)))
        row += px.shape[0]
    # as in layer_plain.layer_norm_grad
    K = M // 512 + 94
    assert ((dgamma - sums[0]).abs() <= K * P.U * sums[2]).all()
    assert ((dbeta - sums[1]).abs() <= K * P.U * sums[3]).all()


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype,M,F", [(torch.bfloat16, 20011, 1024), (torch.float32, 9001, 1024)])
@pytest.mark.parametrize("in_place", [False, True])
def test_slopes(act, dtype, M, F, in_place):
    gu, dh = randn(5, M, 2 * F, dtype=dtype), randn(6, M, F, dtype=dtype)
    parts = list(zip(gu.clone().split(M // 7), dh.split(M // 7)))
    dgu = B.bsr_gated_ff_grad(gu, dh, None, act=act, want_dX=False, dGU=gu if in_place else None)
    assert (dgu.data_ptr() == gu.data_ptr()) == in_place
    row = 0
    for pg, ph in parts:
        assert torch.equal(dgu[row:row + pg.shape[0]], B.bsr_gated_ff_grad(pg, ph, None, act=act, want_dX=False))
        row += pg.shape[0]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param,grad", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.float32, torch.bfloat16)])
def test_optimizer(bits, param, grad):
    """One large tensor, tensors that are no whole vectors, and copies; the first elements alone get the same numbers, at another
    alignment too."""
    n = [(16 << 20) + 77, 1, 3 * 128 + 5]
    few = 100 * 128

    def run(sizes, offset=0):
        def place(seed, i, s, dtype):
            buf = torch.zeros(offset + s, dtype=dtype, device="cuda")
            buf[offset:] = randn(seed + i, n[i], dtype=dtype)[:s]
            return buf[offset:]
        p = [place(10, i, s, param) for i, s in enumerate(sizes)]
        g = [place(20, i, s, grad) for i, s in enumerate(sizes)]
        copies = [torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in sizes]
        batch = B.AdamWBatch(p, g, bits=bits, copies=copies, weight_decay=0.1)
        for step in (1, 2, 3):
            B.bsr_adamw_batched(batch, lr=1e-2, step=step, seed=9)
        return p, copies, batch.states
    large, small = run(n), run([few])
    for kind in range(2):
        assert torch.equal(large[kind][0][:few], small[kind][0])
    for a, b in zip(large[2][0], small[2][0]):
        assert torch.equal(a[:few] if a.dim() == 1 else a[:, :few // 128], b)
    p, copies, states = run(n, 1)
    for a, b in zip(large[0] + large[1] + [t for s in large[2] for t in s], p + copies + [t for s in states for t in s]):
        assert torch.equal(a, b)
    if bits == 32:
        for i in (1, 2):                                           # the tensors behind it, alone
            p1, g1 = [randn(10 + i, n[i], dtype=param)], [randn(20 + i, n[i], dtype=grad)]
            batch = B.AdamWBatch(p1, g1, weight_decay=0.1)
            for step in (1, 2, 3):
                B.bsr_adamw_batched(batch, lr=1e-2, step=step)
            assert torch.equal(p1[0], large[0][i])
            for a, b in zip(large[2][i], batch.states[0]):
                assert torch.equal(a, b)
    else:
        for which, row in (("m", 0), ("r", 1)):
            codes, scales = large[2][0][row], large[2][0][2][row]
            v = B.bsr_adamw_state_values(codes, scales, which)
            assert torch.equal(v[:few], B.bsr_adamw_state_values(codes[:few], scales[:B.bsr_adamw_blocks(few)], which))
            assert torch.equal(v[-77:], B.bsr_adamw_state_values(codes[-77:], scales[-1:], which))
            assert torch.isfinite(v).all() and (v != 0).any()
