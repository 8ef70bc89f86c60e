"""Layer operators on the GPU against the plain binary64 implementation (layer_plain.py), at the sizes, strides, alignments and
values where they can go wrong, within the bounds that layer_plain derives."""
import numpy as np
import pytest
import torch

import layer_plain as P
from layer_plain import DT, check, f64, randn, strided, around_is_untouched
from paper_2311_16883_amd import binding as B

pytestmark = pytest.mark.gpu

NORM_SIZES = [(1, 1, 0, 0), (1, 64, 0, 0), (3, 3, 2, 1), (5, 7, 1, 3), (2, 8, 0, 0), (33, 65, 6, 1), (70, 130, 0, 0), (9, 257, 3, 1),
              (200, 411, 0, 0), (13, 1000, 8, 0), (8, 1536, 0, 0), (6, 2047, 1, 1), (5, 2048, 0, 0), (4, 4099, 5, 2), (3, 8192, 0, 0),
              (3, 8193, 0, 1), (2, 16390, 0, 0), (2, 33001, 3, 1), (1500, 96, 32, 0)]


@pytest.mark.parametrize("dtype,params", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("M,D,pad,offset", NORM_SIZES)
def test_layer_norm(dtype, params, M, D, pad, offset):
    x = randn(1, M, D, dtype=dtype, scale=2.0) + 0.5
    gamma, beta = randn(2, D, dtype=params) + 1, randn(3, D, dtype=params)
    src, out = strided(x, pad, offset), strided(torch.zeros(M, D, dtype=DT[dtype]), pad, offset, fill=7.0)
    Y, stats = B.bsr_layer_norm(src, gamma.cuda(), beta.cuda(), eps=1e-5, Y=out, want_stats=True)
    assert Y is out and around_is_untouched(out, pad, offset, 7.0)
    y, bound, s, e_s = P.layer_norm(f64(x), f64(gamma), f64(beta), float(np.float32(1e-5)))
    check(stats, s, e_s, what="stats")
    check(Y, y, bound, dtype, "Y")
    again = B.bsr_layer_norm(src, gamma.cuda(), beta.cuda(), eps=1e-5)
    assert torch.equal(again, Y)
    inplace = src.clone()
    assert B.bsr_layer_norm(inplace, gamma.cuda(), beta.cuda(), eps=1e-5, Y=inplace) is inplace and torch.equal(inplace, Y)


@pytest.mark.parametrize("dtype,params", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("M,D,pad,offset", NORM_SIZES + [(5000, 24, 0, 0), (2500, 131, 0, 0), (700, 1024, 0, 0), (24, 1024, 0, 0), (61, 337, 3, 1), (300, 80, 0, 0), (2, 9920, 0, 0)])
def test_layer_norm_grad(dtype, params, M, D, pad, offset):
    x, dy = randn(1, M, D, dtype=dtype, scale=2.0) + 0.5, randn(4, M, D, dtype=dtype)
    gamma = randn(2, D, dtype=params) + 1
    src, grad = strided(x, pad, offset), strided(dy, pad + 1, offset)
    _, stats = B.bsr_layer_norm(src, want_stats=True)
    out = strided(torch.zeros(M, D, dtype=DT[dtype]), pad, offset, fill=7.0)
    dX, dgamma, dbeta = B.bsr_layer_norm_grad(src, gamma.cuda(), stats, grad, dX=out)
    assert dX is out and around_is_untouched(out, pad, offset, 7.0)
    dx, e_x, dg, e_g, db, e_b = P.layer_norm_grad(f64(x), f64(gamma), f64(stats), f64(dy))
    check(dX, dx, e_x, dtype, "dX")
    check(dgamma, dg, e_g, what="dgamma")
    check(dbeta, db, e_b, what="dbeta")
    # in the place of dY, weights' gradients added to what is there, and none at all
    same, g1, b1 = grad.clone(), dgamma.clone(), dbeta.clone()
    B.bsr_layer_norm_grad(src, gamma.cuda(), stats, same, dX=same, dgamma=g1, dbeta=b1, accumulate=True)
    assert torch.equal(same, dX) and torch.equal(g1, dgamma + dgamma) and torch.equal(b1, dbeta + dbeta)
    alone = B.bsr_layer_norm_grad(src, gamma.cuda(), stats, grad, want_params=False)
    check(alone, dx, e_x, dtype, "dX alone")
    over = src.clone()
    B.bsr_layer_norm_grad(over, gamma.cuda(), stats, grad, dX=over)
    assert torch.equal(over, dX)


def test_layer_norm_without_weights_and_far_from_zero():
    x = (randn(5, 40, 300) * 0.01 + 4096.0)
    Y, stats = B.bsr_layer_norm(x.cuda(), want_stats=True)
    y, bound, s, e_s = P.layer_norm(f64(x), None, None, float(np.float32(1e-5)))
    check(stats, s, e_s)
    check(Y, y, bound)
    dy = randn(6, 40, 300)
    dX, dg, db = B.bsr_layer_norm_grad(x.cuda(), None, stats, dy.cuda())
    dx, e_x, wg, e_g, wb, e_b = P.layer_norm_grad(f64(x), None, f64(stats), f64(dy))
    check(dX, dx, e_x)
    check(dg, wg, e_g)
    check(db, wb, e_b)


def test_layer_norm_rows_of_one_value_of_nan_and_of_infinities_stay_by_themselves():
    x = randn(7, 9, 100)
    x[2] = 3.25
    x[4, 50] = float("nan")
    x[6, 3] = float("inf")
    Y, stats = B.bsr_layer_norm(x.cuda(), want_stats=True)
    assert torch.equal(Y[2].cpu(), torch.zeros(100)) and float(stats[2, 0]) == 3.25
    assert bool(Y[4].isnan().all()) and bool(Y[6].isnan().any())
    others = [0, 1, 3, 5, 7, 8]
    y, bound, _, _ = P.layer_norm(f64(x[others]), None, None, float(np.float32(1e-5)))
    check(Y[others], y, bound)


def test_layer_norm_of_nothing():
    for M, D in ((0, 5), (4, 0), (0, 0)):
        x = torch.zeros(M, D, device="cuda")
        Y, stats = B.bsr_layer_norm(x, want_stats=True)
        assert Y.shape == (M, D) and stats.shape == (M, 2)
        dX, dg, db = B.bsr_layer_norm_grad(x, None, torch.zeros(M, 2, device="cuda"), x)
        assert dX.shape == (M, D) and torch.equal(dg, torch.zeros(D, device="cuda")) and torch.equal(db, dg)
    ones = torch.ones(5, device="cuda")
    _, dg, db = B.bsr_layer_norm_grad(torch.zeros(0, 5, device="cuda"), None, torch.zeros(0, 2, device="cuda"),
                                      torch.zeros(0, 5, device="cuda"), dgamma=ones, dbeta=ones.clone(), accumulate=True)
    assert torch.equal(dg, torch.ones(5, device="cuda"))


# ---- gated block ----

GATED_SIZES = [(1, 1, 1), (1, 64, 64), (1, 2048, 320), (2, 9, 3), (7, 33, 20), (16, 128, 64), (17, 65, 33), (31, 256, 100), (64, 96, 128), (65, 100, 129),
               (100, 411, 77), (128, 384, 256), (130, 264, 200), (257, 136, 130), (300, 520, 257), (513, 72, 300), (3, 5000, 48),
               (90, 130, 66), (70, 38, 34), (150, 250, 130), (200, 1030, 62), (33, 66, 1002), (4, 70, 2200), (2, 33, 4100), (4, 7, 9), (20, 1000, 136), (40, 2500, 72)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,D,F", GATED_SIZES)
def test_gated_ff(dtype, M, D, F):
    name = ("silu", "gelu", "gelu_tanh", "relu")[(M + D + F) % 4]
    x, w = randn(1, M, D, dtype=dtype), randn(2, D, 2 * F, dtype=dtype, scale=D ** -0.5)
    H, GU = B.bsr_gated_ff(x.cuda(), w.cuda(), act=name, want_GU=True)
    h, e_h, gu, e_gu = P.gated(f64(x), f64(w), name, dtype)
    check(GU, gu, e_gu, dtype, "GU")
    check(H, h, e_h, dtype, "H")
    # rows of wider matrices, away from 16 bytes, around which nothing is read that counts or written
    for pad, offset in ((8, 0), (3, 1)):
        src, wide = strided(x, pad, offset), strided(w, pad, offset)
        out, both = strided(torch.zeros(M, F, dtype=DT[dtype]), pad, offset, 7.0), strided(torch.zeros(M, 2 * F, dtype=DT[dtype]), pad, offset, 7.0)
        B.bsr_gated_ff(src, wide, act=name, H=out, GU=both)
        assert around_is_untouched(out, pad, offset, 7.0) and around_is_untouched(both, pad, offset, 7.0)
        check(both, gu, e_gu, dtype, "GU")
        check(out, h, e_h, dtype, "H")
        assert torch.equal(B.bsr_gated_ff(src, wide, act=name), out)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,D,F", GATED_SIZES)
def test_gated_ff_grad(dtype, M, D, F):
    name = ("silu", "gelu", "gelu_tanh", "relu")[(M + D + F + 1) % 4]
    gu, dh = randn(1, M, 2 * F, dtype=dtype, scale=2.0), randn(2, M, F, dtype=dtype)
    w = randn(3, D, 2 * F, dtype=dtype, scale=D ** -0.5)
    for pad, offset in ((0, 0), (8, 0), (3, 1)):
        src, grad, wide = strided(gu, pad, offset), strided(dh, pad, offset), strided(w, pad, offset)
        out, x = strided(torch.zeros(M, 2 * F, dtype=DT[dtype]), pad, offset, 7.0), strided(torch.zeros(M, D, dtype=DT[dtype]), pad, offset, 7.0)
        dX, dGU = B.bsr_gated_ff_grad(src, grad, wide, act=name, dGU=out, dX=x)
        assert dX is x and dGU is out and around_is_untouched(out, pad, offset, 7.0) and around_is_untouched(x, pad, offset, 7.0)
        want, bound = P.gated_slopes(f64(gu), f64(dh), name)
        check(dGU, want, bound, dtype, "dGU")
        d = f64(dGU)
        size = np.abs(d) @ np.abs(f64(w)).T
        check(dX, d @ f64(w).T, (2 * F + 1) * P.U * size, dtype, "dX")
        same = src.clone()
        dX2, dGU2 = B.bsr_gated_ff_grad(same, grad, wide, act=name, dGU=same)
        assert dGU2 is same and torch.equal(dGU2, dGU)
        check(dX2, f64(dX), 2 * (2 * F + 1) * P.U * size, dtype, "dX in place")
        assert torch.equal(B.bsr_gated_ff_grad(src, grad, None, act=name, want_dX=False), dGU)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gated_many_tiles(dtype):
    """More tiles than compute units, ragged in both directions."""
    M, D, F = 3077, 72, 2120
    x, w = randn(1, M, D, dtype=dtype), randn(2, D, 2 * F, dtype=dtype, scale=D ** -0.5)
    H, GU = B.bsr_gated_ff(x.cuda(), w.cuda(), act="silu", want_GU=True)
    h, e_h, gu, e_gu = P.gated(f64(x), f64(w), "silu", dtype)
    check(GU, gu, e_gu, dtype, "GU")
    check(H, h, e_h, dtype, "H")
    M, D, F = 3077, 4200, 36
    gu, dh, w = randn(1, M, 2 * F, dtype=dtype), randn(2, M, F, dtype=dtype), randn(3, D, 2 * F, dtype=dtype)
    dX, dGU = B.bsr_gated_ff_grad(gu.cuda(), dh.cuda(), w.cuda(), act="silu")
    d = f64(dGU)
    size = np.abs(d) @ np.abs(f64(w)).T
    check(dX, d @ f64(w).T, (2 * F + 1) * P.U * size, dtype, "dX")


# Sizes that every tile takes, each with its contraction whole and split where that occurs, and with whole vectors or not.
TILE_SIZES = [(13260, 1144, 264), (609, 1143, 6534), (84, 105, 8932), (65, 104, 9048), (1, 8, 10), (1, 2168, 16), (1, 2385, 10), (2, 8, 8), (2, 13, 12), (2, 16, 16), (3, 168, 16), (4, 187, 8), (33, 1990, 12), (35, 9, 8),
              (36, 16, 16), (39, 348, 8), (41, 8, 10), (45, 16, 16), (65, 1048, 8), (66, 280, 9), (624, 9, 6982), (798, 8, 5217), (3099, 8, 413),
              (3342, 4608, 8), (3918, 8, 948), (4140, 11042, 14), (4261, 2664, 16), (4793, 3594, 9), (6341, 8, 325), (6552, 1406, 10),
              (6661, 9, 312), (7059, 9, 399), (8203, 4872, 16), (8291, 22, 433), (10347, 8, 68), (11432, 16, 304), (65, 4616, 2082),
              (66, 5048, 2080), (80, 10448, 1040), (20, 9000, 40), (9, 9001, 33), (5, 70, 8300), (32, 64, 8256)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,D,F", TILE_SIZES)
def test_gated_ff_in_every_tile(dtype, M, D, F):
    x, w = randn(1, M, D, dtype=dtype), randn(2, D, 2 * F, dtype=dtype, scale=D ** -0.5)
    H, GU = B.bsr_gated_ff(x.cuda(), w.cuda(), act="gelu_tanh", want_GU=True)
    h, e_h, gu, e_gu = P.gated(f64(x), f64(w), "gelu_tanh", dtype)
    check(GU, gu, e_gu, dtype, "GU")
    check(H, h, e_h, dtype, "H")
    assert torch.equal(B.bsr_gated_ff(x.cuda(), w.cuda(), act="gelu_tanh"), H)


@pytest.mark.parametrize("act", ["silu", "relu"])
@pytest.mark.parametrize("M,D,F,pad,offset", [(1, 130, 3, 0, 0), (3, 128, 32, 0, 0), (4, 1024, 40, 8, 0), (5, 1025, 37, 3, 1), (16, 1040, 96, 0, 0), (17, 2047, 65, 0, 0),
                                              (31, 2100, 31, 1, 3), (32, 3000, 64, 16, 8), (32, 1500, 7, 0, 0), (7, 77, 33, 5, 0), (29, 400, 8190, 0, 0)])
def test_up_to_32_rows(act, M, D, F, pad, offset):
    """Slices and vectors that the contraction or the columns end in, rows behind the last one, NaN around the operands."""
    x, w = randn(1, M, D, dtype="bf16"), randn(2, D, 2 * F, dtype="bf16", scale=D ** -0.5)
    H, GU = strided(torch.zeros(M, F, dtype=torch.bfloat16), pad, offset, 7.0), strided(torch.zeros(M, 2 * F, dtype=torch.bfloat16), pad, offset, 7.0)
    B.bsr_gated_ff(strided(x, pad, offset), strided(w, pad, offset), act=act, H=H, GU=GU)
    assert around_is_untouched(H, pad, offset, 7.0) and around_is_untouched(GU, pad, offset, 7.0)
    h, e_h, gu, e_gu = P.gated(f64(x), f64(w), act, "bf16")
    check(GU, gu, e_gu, "bf16", "GU")
    check(H, h, e_h, "bf16", "H")
    # a row does not depend on the others
    again = B.bsr_gated_ff(strided(torch.cat((x, x))[:min(32, 2 * M)], pad, offset), strided(w, pad, offset), act=act)
    if M > 2:
        assert torch.equal(again[:M], H)


TILE_GRAD_SIZES = [(1, 8, 14), (1, 9, 91), (1, 10, 8), (1, 10, 94), (1, 10, 558), (1, 11, 9), (1, 15, 8), (1, 16, 424), (33, 9, 623), (34, 8, 13),
                   (36, 11, 19), (36, 13, 8), (44, 10, 126), (44, 11, 8), (59, 11, 113), (62, 8, 616), (141, 13218, 11), (1046, 10033, 8),
                   (1482, 6300, 11), (1556, 3880, 8), (1961, 3371, 8), (2177, 11, 1971), (2584, 2573, 11), (3080, 652, 8), (3642, 12, 2136),
                   (4200, 759, 8), (4238, 10, 884), (4507, 10, 4071), (5155, 16, 3384), (6191, 8, 677), (7959, 778, 9), (8402, 298, 10)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,D,F", TILE_GRAD_SIZES)
def test_gated_ff_grad_in_every_tile(dtype, M, D, F):
    gu, dh, w = randn(1, M, 2 * F, dtype=dtype), randn(2, M, F, dtype=dtype), randn(3, D, 2 * F, dtype=dtype)
    dX, dGU = B.bsr_gated_ff_grad(gu.cuda(), dh.cuda(), w.cuda(), act="silu")
    d = f64(dGU)
    size = np.abs(d) @ np.abs(f64(w)).T
    check(dX, d @ f64(w).T, (2 * F + 1) * P.U * size, dtype, "dX")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", ["silu", "gelu", "gelu_tanh", "relu"])
def test_activations_over_their_range(dtype, name):
    g = torch.cat((torch.linspace(-12, 12, 4001), torch.tensor([0.0, -0.0, 1e-30, -1e-30, 50.0, -50.0, 200.0, -200.0, 1e4, -1e4]))).to(DT[dtype])
    n = len(g)
    gu = torch.cat((g[None], torch.full((1, n), 1.0).to(DT[dtype])), dim=1)
    dh = torch.ones(1, n, dtype=DT[dtype])
    d = B.bsr_gated_ff_grad(gu.cuda(), dh.cuda(), None, act=name, want_dX=False)
    want, bound = P.gated_slopes(f64(gu), f64(dh), name)
    check(d, want, bound, dtype)
    # forward: G = g and U = 1 from a product of one column
    w = torch.cat((g, torch.ones(n).to(DT[dtype])))[None]
    H = B.bsr_gated_ff(torch.ones(1, 1, dtype=DT[dtype]).cuda(), w.cuda(), act=name)
    h, e_h, _, _ = P.gated(np.ones((1, 1)), f64(w), name, dtype)
    check(H, h, e_h, dtype)


def test_gated_rows_of_nan_and_infinities_stay_by_themselves():
    for dtype in ("f32", "bf16"):
        M, D, F = 70, 100, 40
        x, w = randn(1, M, D, dtype=dtype), randn(2, D, 2 * F, dtype=dtype, scale=0.1)
        x[3, 7], x[50, 99] = float("nan"), float("inf")
        H, GU = B.bsr_gated_ff(x.cuda(), w.cuda(), want_GU=True)
        assert bool(GU[3].isnan().all()) and not bool(GU[50].isfinite().any())
        rows = [i for i in range(M) if i not in (3, 50)]
        h, e_h, gu, e_gu = P.gated(f64(x[rows]), f64(w), "silu", dtype)
        check(GU[rows], gu, e_gu, dtype)
        check(H[rows], h, e_h, dtype)


def test_gated_of_nothing():
    for M, D, F in ((0, 4, 4), (4, 0, 4), (4, 4, 0)):
        x, w = torch.ones(M, D, device="cuda"), torch.ones(D, 2 * F, device="cuda")
        H, GU = B.bsr_gated_ff(x, w, want_GU=True)
        assert torch.equal(H, torch.zeros(M, F, device="cuda")) and torch.equal(GU, torch.zeros(M, 2 * F, device="cuda"))
        dX, dGU = B.bsr_gated_ff_grad(GU, H, w)
        assert torch.equal(dX, torch.zeros(M, D, device="cuda")) and dGU.shape == (M, 2 * F)


# ---- AdamW ----

SIZES = [1, 3, 127, 128, 129, 1000, 4096, 4097, 12345, 0, 40001]


def moments(seed, n):
    return randn(seed, n, scale=3e-4), (randn(seed + 1, n, scale=1e-3)).abs()


def make(sizes, dtype, grad, bits, copy, offset=0):
    """Tensors at `offset` elements into buffers; -> batch, and the numbers before the step in binary64"""
    def put(x):
        buf = torch.zeros(len(x) + offset + 8, dtype=x.dtype, device="cuda")
        buf[offset:offset + len(x)] = x.cuda()
        return buf[offset:offset + len(x)]
    params, grads, states, before = [], [], [], []
    for i, n in enumerate(sizes):
        p, g = randn(10 * i, n, dtype=dtype, scale=0.02), randn(10 * i + 1, n, dtype=grad, scale=1e-3)
        if n > 5:
            g[1], g[2] = 0.0, 30.0
        m, r = moments(10 * i + 2, n)
        params.append(put(p))
        grads.append(put(g))
        if bits == 32:
            states.append((put(m), put(r * r)))
            before.append((f64(p), f64(g), f64(m), np.sqrt(f64(r * r))))
        else:
            blocks = B.bsr_adamw_blocks(n)
            codes = [torch.randint(0, 256, (n,), generator=torch.Generator().manual_seed(i + k), dtype=torch.uint8) for k in range(2)]
            scales = torch.randint(100, 120, (2, blocks), generator=torch.Generator().manual_seed(i), dtype=torch.uint8)
            if blocks > 3:
                scales[:, 2] = 0                     # zero moments
                codes[0][256:384] = codes[1][256:384] = 0
            before.append((f64(p), f64(g), P.decode(codes[0].numpy(), scales[0].numpy(), 3), P.decode(codes[1].numpy(), scales[1].numpy(), 4)))
            states.append((put(codes[0]), put(codes[1]), scales.cuda()))
    copies = [put(torch.zeros(n, dtype=torch.bfloat16)) if i % 3 else None for i, n in enumerate(sizes)] if copy else None
    decays = [0.1 * (i % 2) for i in range(len(sizes))]
    return B.AdamWBatch(params, grads, bits=bits, states=states, copies=copies, weight_decay=decays), before, decays


OPTIONS = dict(lr=3e-4, beta1=0.9, beta2=0.999, eps=1e-8, grad_scale=0.5, step=17)


def rounded(options):
    """The numbers as binary32 holds them (the betas enter as they are)."""
    return {k: float(np.float32(v)) if k in ("lr", "eps", "grad_scale") else v for k, v in options.items()}


def check_codes(codes, scales, x, e, bits, u):
    """Codes of values x, known to e, after rounding by u."""
    a = np.abs(x)
    byte, step = P.steps_of(a, bits)
    near = P.steps_of(a * (1 + 1e-5), bits)[0] != P.steps_of(a * (1 - 1e-5), bits)[0]       # a block whose largest is beside a border
    scales = np.asarray(scales).astype(int)
    assert (near | (scales == byte)).all(), (scales[:4], byte[:4])
    sure = ~np.repeat(near, 128)[:len(x)]
    value = P.decode(codes, scales, bits)
    lo, hi = np.floor((a - e) / step + u - 1e-6) * step, np.floor((a + e) / step + u + 1e-6) * step
    if bits == 4:
        lo, hi = np.where(a > 0, np.maximum(lo, step), lo), np.where(a > 0, np.maximum(hi, step), hi)
    gone = np.repeat(byte == 0, 128)[:len(x)]
    lo, hi = np.where(gone, 0.0, lo), np.where(gone, 0.0, hi)
    # a magnitude whose exponent its error may change has a neighbour at half or twice the distance
    edge = np.floor(np.log2(np.maximum(a - e, 1e-300))) != np.floor(np.log2(np.maximum(a + e, 1e-300)))
    ok = (np.abs(value) >= lo) & (np.abs(value) <= hi) | edge & (np.abs(np.abs(value) - a) <= 2 * step) | ~sure & (np.abs(np.abs(value) - a) <= 2 * step)
    assert ok.all(), (np.argwhere(~ok)[:4].ravel(), value[~ok][:4], a[~ok][:4], step[~ok][:4])
    assert (np.sign(value) * x >= 0).all()
    assert sure.sum() == 0 or edge.mean() < 0.01


@pytest.mark.parametrize("dtype,grad,bits,copy", [("f32", "f32", 32, False), ("f32", "bf16", 32, True), ("bf16", "bf16", 32, False), ("bf16", "f32", 8, False),
                                                  ("f32", "f32", 8, True), ("f32", "bf16", 8, False), ("bf16", "bf16", 8, True)])
@pytest.mark.parametrize("offset", [0, 3])
def test_adamw_step(dtype, grad, bits, copy, offset):
    batch, before, decays = make(SIZES, dtype, grad, bits, copy, offset)
    seed = (5 << 32) + 77
    B.bsr_adamw_batched(batch, **OPTIONS, seed=seed)
    o, first = rounded(OPTIONS), 0
    for i, n in enumerate(SIZES):
        if n == 0:
            continue
        p, e_p, m, e_m, r, e_r = P.adamw(*before[i], first, o, float(np.float32(decays[i])))
        check(batch.params[i], p, e_p, dtype, f"param {i}")
        if batch.copies[i] is not None:
            check(batch.copies[i], p, e_p, "bf16", f"copy {i}")
        s = batch.states[i]
        if bits == 32:
            check(s[0], m, e_m)
            check(s[1], r * r, 3 * r * e_r)
        else:
            um, ur = P.uniform(first, n, seed, o["step"])
            codes, roots, scales = s[0].cpu().numpy(), s[1].cpu().numpy(), s[2].cpu().numpy()
            check_codes(codes, scales[0], m, e_m, 3, um)
            check_codes(roots, scales[1], r, e_r, 4, ur)
            for which, c, bitsk, row in (("m", s[0], 3, 0), ("r", s[1], 4, 1)):
                for out in ("f32", "bf16"):
                    got = B.bsr_adamw_state_values(c, s[2][row].contiguous(), which, dtype=DT[out])
                    assert np.array_equal(f64(got), P.decode(c.cpu().numpy(), scales[row], bitsk))
        first += -(-n // 128) * 128
