"""The optimizer's moments where their numbers come to an end: roots of second moments below and above binary32's range, codes beside
their borders, gradients of any NaN."""
import math

import numpy as np
import pytest
import torch

import layer_plain as P
import test_gpu_layer_ops as ops
from layer_plain import U, check, f64
from paper_2311_16883_amd import binding as B

pytestmark = pytest.mark.gpu

BETA2 = 0.999


def first_step(g, bits, eps, lr=1e-3):
    """From zeros; -> what the parameters became, the state, the numbers as the kernels take them"""
    batch = B.AdamWBatch([torch.zeros(len(g), device="cuda")], [g.cuda()], bits=bits)
    B.bsr_adamw_batched(batch, lr=lr, step=1, eps=eps, seed=3)
    return batch.params[0], batch.states[0], dict(ops.rounded(dict(lr=lr, eps=eps, grad_scale=1.0)), beta1=0.9, beta2=BETA2, step=1)


def spread(size, n=300):
    """Magnitudes from size / 2 to 2 * size, of both signs"""
    x = torch.exp2(torch.rand(n, generator=torch.Generator().manual_seed(11)) * 2 - 1) * size
    return torch.where(torch.arange(n) % 2 == 0, x, -x)


SMALL = [(1e-17, 1e-20), (2e-18, 1e-20), (1e-19, 1e-23), (1e-21, 1e-25), (1e-23, 1e-27), (1e-25, 1e-30)]


@pytest.mark.parametrize("size,eps", SMALL)
def test_small_second_moments_in_8_bits_keep_their_roots(size, eps):
    """Roots down to 2^-95 have codes; their squares do not fit binary32."""
    g = spread(size)
    n = len(g)
    p, state, o = first_step(g, 8, eps)
    zero = np.zeros(n)
    want, bound, m, e_m, r, e_r = P.adamw(zero, f64(g), zero, zero, 0, o, 0.0)
    check(p, want, bound, what="param")
    um, ur = P.uniform(0, n, 3, 1)
    scales = state[2].cpu().numpy()
    ops.check_codes(state[0].cpu().numpy(), scales[0], m, e_m, 3, um)
    ops.check_codes(state[1].cpu().numpy(), scales[1], r, e_r, 4, ur)


@pytest.mark.parametrize("size", [1e20, 1e25, 1e30, 1e35])
def test_large_second_moments_in_8_bits_keep_their_roots(size):
    """... nor do those of roots above 2^64."""
    test_small_second_moments_in_8_bits_keep_their_roots(size, 1e-8)


@pytest.mark.parametrize("size,eps", SMALL)
def test_small_second_moments_in_binary32_have_the_roots_of_what_is_held(size, eps):
    """Below 2^-126 v has fewer bits, below 2^-150 none: then the update is m over eps."""
    g = spread(size)
    p, (m, v), o = first_step(g, 32, eps)
    # two products and a sum, each within half a step of its own: of 2^-149 among the subnormals
    want_v = (1 - BETA2) * f64(g) ** 2
    assert (np.abs(f64(v) - want_v) <= 4 * U * want_v + 1.5 * 2.0 ** -149).all()
    denominator = np.sqrt(f64(v)) / math.sqrt(1 - BETA2) + o["eps"]
    want = -o["lr"] / (1 - 0.9) * f64(m) / denominator
    check(p, want, 16 * U * np.abs(want), what="param")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bits", [3, 4])
def test_codes_are_cut_off_just_below_their_borders(bits, dtype):
    """Without an exponent codes are a fixed distance apart: one rounding step below the border, to which u would carry it, a number has the code below."""
    n, seed, step = 128 * 40, 21, 1
    u = P.uniform(0, n, seed, step)[0 if bits == 3 else 1]
    unit = 2.0 ** (0 - 14 - bits)                    # of blocks whose largest number is 1
    k = np.arange(n) % (1 << bits)
    border = ((k + 1 - u) * unit).astype(np.float32)             # (exact: at most 4 + 16 bits)
    x = np.nextafter(border, np.float32(0))
    x[::128] = 1.0
    batch = B.AdamWBatch([torch.zeros(n, dtype=dtype, device="cuda")], [torch.from_numpy(x).cuda()], bits=8)
    # without a past: m is the gradient, and v its square, exactly
    B.bsr_adamw_batched(batch, lr=1e-3, step=step, beta1=0.0, beta2=0.0, seed=seed)
    codes, scales = batch.states[0][0 if bits == 3 else 1].cpu().numpy(), batch.states[0][2].cpu().numpy()[0 if bits == 3 else 1]
    assert (scales == 127).all()
    value = P.decode(codes, scales, bits)
    own = np.floor(np.log2(x.astype(float))) - bits
    distance = 2.0 ** np.maximum(own, -14 - bits)
    want = np.floor(x.astype(float) / distance + u) * distance
    want = np.maximum(want, unit) if bits == 4 else want
    assert np.array_equal(value, want), (int((value != want).sum()), np.argwhere(value != want)[:4].ravel())


@pytest.mark.parametrize("dtype,word", [(torch.float32, -1), (torch.float32, 0x7FFFFFFF), (torch.float32, 0x7F800001), (torch.bfloat16, -1), (torch.bfloat16, 0x7FFF)])
def test_a_nan_of_any_bits_makes_both_moments_of_its_block_nan(dtype, word):
    g = torch.full((300,), 1e-3, dtype=dtype)
    g.view(torch.int32 if dtype == torch.float32 else torch.int16)[130] = word
    assert bool(g[130].isnan())
    batch = B.AdamWBatch([torch.zeros(300, device="cuda")], [g.cuda()], bits=8)
    B.bsr_adamw_batched(batch, lr=1e-3, step=1)
    m, r, scales = batch.states[0]
    assert (scales[:, 1] == 255).all() and not (scales[:, (0, 2)] == 255).any()
    for codes, row, which in ((m, 0, "m"), (r, 1, "r")):
        values = B.bsr_adamw_state_values(codes, scales[row].contiguous(), which)
        assert bool(values[128:256].isnan().all()) and not bool(values[:128].isnan().any()) and not bool(values[256:].isnan().any())
    assert bool(batch.params[0][130].isnan()) and int(batch.params[0].isnan().sum()) == 1
