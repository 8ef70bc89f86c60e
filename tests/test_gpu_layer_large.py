"""Layer operators where offsets pass 32 bits: rows far into large matrices against the same rows alone, elements far into a large
tensor against the plain implementation."""
import numpy as np
import pytest
import torch

import layer_plain as P
from layer_plain import f64
from paper_2311_16883_amd import binding as B

pytestmark = pytest.mark.gpu


def part_of(M, D, rows, dtype=torch.bfloat16, scale=1.0):
    """A large matrix of cheap numbers, and the rows `rows` of it alone."""
    x = torch.empty(M, D, dtype=dtype, device="cuda")
    step = max(1, (1 << 28) // D)
    for a in range(0, M, step):
        g = torch.Generator(device="cuda").manual_seed(a + D)
        x[a:a + step] = torch.randn(min(step, M - a), D, generator=g, device="cuda", dtype=dtype) * scale
    return x, x[rows].clone()


def test_norm_of_more_than_four_billion_elements():
    M, D = 70001, 65000
    rows = slice(M - 3, M)
    x, few = part_of(M, D, rows)
    y, stats = B.bsr_layer_norm(x, want_stats=True)
    y1, s1 = B.bsr_layer_norm(few, want_stats=True)
    assert torch.equal(y[rows], y1) and torch.equal(stats[rows], s1)
    dx, dg, db = B.bsr_layer_norm_grad(x, None, stats, y, dX=y)            # (the norm itself as the gradient, in its place)
    dx1 = B.bsr_layer_norm_grad(few, None, s1, y1, want_params=False)
    assert torch.equal(dx[rows], dx1)
    # dY = xh: every column's sum of squares is about M, and the sum about 0; a sixteenth of the columns summed in binary64
    del y, dx
    cols = torch.arange(0, D, 16, device="cuda")
    total, square = torch.zeros(len(cols), dtype=torch.float64, device="cuda"), torch.zeros(len(cols), dtype=torch.float64, device="cuda")
    size = torch.zeros_like(total)
    for a in range(0, M, 7000):
        xh = (x[a:a + 7000][:, cols].double() - stats[a:a + 7000, :1].double()) * stats[a:a + 7000, 1:].double()
        yy = ((x[a:a + 7000][:, cols].float() - stats[a:a + 7000, :1]) * stats[a:a + 7000, 1:]).bfloat16().double()
        total += yy.sum(dim=0)
        square += (yy * xh).sum(dim=0)
        size += yy.abs().sum(dim=0)
    # (M additions of terms of the columns' sizes; a few of the recomputed dY may be one bfloat16 step off where binary32 rounded otherwise)
    assert float((dg[cols].double() - square).abs().max()) <= M * P.U * float(square.max()) + 20 * 2.0 ** -6 * 6
    assert float((db[cols].double() - total).abs().max()) <= M * P.U * float(size.max()) + 20 * 2.0 ** -6


def test_gated_block_of_more_than_four_billion_elements():
    M, D, F = 2200001, 1960, 72                        # X: 4.3e9 elements
    rows = slice(M - 5, M)
    x, few = part_of(M, D, rows, scale=0.05)
    w = torch.randn(D, 2 * F, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").bfloat16()
    h, gu = B.bsr_gated_ff(x, w, want_GU=True)
    # (the same rows in a smaller product: other tiles, other orders of additions)
    want, e_h, wgu, e_gu = P.gated(f64(few), f64(w), "silu", "bf16")
    P.check(gu[rows], wgu, e_gu, "bf16")
    P.check(h[rows], want, e_h, "bf16")
    dx, dgu = B.bsr_gated_ff_grad(gu, h, w, dGU=gu, dX=x)
    d = f64(dgu[rows])
    P.check(dx[rows], d @ f64(w).T, (2 * F + 1) * P.U * (np.abs(d) @ np.abs(f64(w)).T), "bf16")


def test_weights_of_more_than_four_gigabytes():
    M, D, F = 3, 60000, 20000                          # W: 2.4e9 elements, 4.8 GB
    w, _ = part_of(D, 2 * F, slice(0, 1), scale=0.01)
    x = torch.randn(40, D, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda").bfloat16()
    cols = [0, 1, F // 2, F - 1]
    wc = torch.cat((w[:, cols], w[:, [F + c for c in cols]]), dim=1)
    for m in (1, 2, 3, 40):
        h, gu = B.bsr_gated_ff(x[:m], w, want_GU=True)
        want, e_h, wgu, e_gu = P.gated(f64(x[:m]), f64(wc), "silu", "bf16")
        P.check(gu[:, cols + [F + c for c in cols]], wgu, e_gu, "bf16")
        P.check(h[:, cols], want, e_h, "bf16")
    dx, dgu = B.bsr_gated_ff_grad(gu, h, w, dGU=gu)
    some = [0, 7, D // 2, D - 1]
    d = f64(dgu)
    P.check(dx[:, some], d @ f64(w[some]).T, (2 * F + 1) * P.U * (np.abs(d) @ np.abs(f64(w[some])).T), "bf16")


@pytest.mark.parametrize("bits", [8, 32])
def test_optimizer_step_of_more_than_four_billion_elements(bits):
    n = (1 << 32) + 5003
    p = torch.empty(n, dtype=torch.bfloat16, device="cuda")
    g = torch.empty(n, dtype=torch.bfloat16, device="cuda")
    for a in range(0, n, 1 << 29):
        e = min(n, a + (1 << 29))
        p[a:e], g[a:e] = 0.5, 1e-3
    ends = [(0, 1000), ((1 << 32) - 1000, (1 << 32) + 1000), (n - 1003, n)]
    for a, b in ends:
        p[a:b] = torch.randn(b - a, device="cuda").bfloat16()
        g[a:b] = torch.randn(b - a, device="cuda").bfloat16()
    before = [(f64(p[a:b]), f64(g[a:b])) for a, b in ends]
    batch = B.AdamWBatch([p], [g], bits=bits, weight_decay=0.1)
    o = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, grad_scale=1.0, step=1)
    B.bsr_adamw_batched(batch, **o, seed=3)
    o = {k: float(np.float32(v)) if k in ("lr", "eps") else v for k, v in o.items()}
    for (a, b), (p0, g0) in zip(ends, before):
        want, bound, m, e_m, r, e_r = P.adamw(p0, g0, 0 * p0, 0 * p0, a, o, float(np.float32(0.1)))
        P.check(p[a:b], want, bound, "bf16")
        s = batch.states[0]
        if bits == 32:
            P.check(s[0][a:b], m, e_m)
            continue
        # whole blocks: scale and codes of what was there, by the numbers of these very elements
        first, last = -(-a // 128) * 128, b // 128 * 128
        u, v = P.uniform(first, last - first, 3, 1)
        for row, code, bits_, x, e, z in ((0, s[0], 3, m, e_m, u), (1, s[1], 4, r, e_r, v)):
            x, e = np.abs(x[first - a:last - a]), e[first - a:last - a]
            scales, step = P.steps_of(x, bits_)
            got = np.abs(P.decode(code[first:last].cpu().numpy(), s[2][row, first // 128:last // 128].cpu().numpy(), bits_))
            lo, hi = np.floor((x - e) / step + z - 1e-6) * step, np.floor((x + e) / step + z + 1e-6) * step
            if bits_ == 4:
                lo, hi = np.maximum(lo, step), np.maximum(hi, step)
            off = ~((got >= lo) & (got <= hi))
            assert off.mean() < 0.002 and (np.abs(got - x) <= 2 * step).all()      # (those beside a power of two, as in check_codes)
