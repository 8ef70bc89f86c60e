"""The layer operators from their definitions, in binary64 (numpy), and bounds on what binary32 arithmetic may differ from them.
Written apart from the library; only tests import it.

U is the rounding error of one binary32 operation, H of one rounding to bfloat16, both relative.  A sum of n terms in which no term
goes through more than K additions is off by at most K * U * (sum of the terms' magnitudes), whatever the order.
"""
import math

import numpy as np
import torch
from scipy.special import erf

U = 2.0 ** -24
H = 2.0 ** -8
TINY = 1e-37                          # results near the subnormals

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def f64(x):
    return x.detach().cpu().double().numpy()


def randn(seed, *size, dtype="f32", scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*size, generator=g) * scale).to(DT[dtype])


def strided(x, pad=0, offset=0, fill=float("nan")):
    """The same matrix on the GPU with `pad` more elements per row and `offset` elements into its buffer, `fill` around it."""
    rows, cols = x.shape
    ld = cols + pad
    buf = torch.full((offset + rows * ld + 8,), fill, dtype=x.dtype, device="cuda")
    view = buf[offset:offset + rows * ld].view(rows, ld)[:, :cols]
    view.copy_(x)
    return view


def around_is_untouched(view, pad, offset, fill):
    """Everything of strided()'s buffer but the matrix still holds `fill`."""
    rows, cols = view.shape
    ld = cols + pad
    buf = torch.as_strided(view, (offset + rows * ld + 8,), (1,), 0).clone()
    if rows:
        buf[offset:offset + rows * ld].view(rows, ld)[:, :cols] = fill
    return bool((buf == fill).all())


def check(got, want, bound, dtype="f32", what=""):
    """|got - want| within the binary32 bound and the one rounding to dtype."""
    got, want = f64(got), np.asarray(want)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    tol = np.broadcast_to(bound, want.shape) + TINY + (H * (np.abs(want) + bound) if dtype == "bf16" else 0.0)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:3].tolist(), got[bad][:3], want[bad][:3], np.asarray(tol)[bad][:3])


# ---- layer norm ----

def additions(D):
    """Additions that an element of a row goes through: those of its lane (32 at most where rows stay in registers; one for every 1024 * 4 of
    the longest), 6 between lanes, 16 between waves."""
    return min(D, 64 + D // 1024)


def layer_norm(x, gamma, beta, eps):
    """-> y, its bound, stats, their bound"""
    D = x.shape[1]
    K = additions(D)
    gamma, beta = np.ones(D) if gamma is None else gamma, np.zeros(D) if beta is None else beta
    mean = x.mean(axis=1, keepdims=True)
    d = x - mean
    var = (d * d).mean(axis=1, keepdims=True)
    rstd = 1.0 / np.sqrt(var + eps)
    xh = d * rstd
    y = xh * gamma + beta
    first = (K + 2) * U * np.abs(x).mean(axis=1, keepdims=True)                    # what the first mean is off
    size = np.abs(d).mean(axis=1, keepdims=True) + first
    e_d = 2 * U * (np.abs(d) + first) + (K + 3) * U * size
    e_var = 2 * (K + 4) * U * (var + first ** 2) / (var + eps)                     # relative
    e_rstd = 0.5 * e_var + 4 * U
    bound = np.abs(gamma) * (np.abs(xh) * (e_rstd + 4 * U) + e_d * rstd) * 1.01 + 2 * U * (np.abs(y) + np.abs(beta))
    e_stats = np.concatenate((U * np.abs(mean) + (K + 3) * U * size, e_rstd * rstd * 1.01), axis=1)
    return y, bound, np.concatenate((mean, rstd), axis=1), e_stats


def layer_norm_grad(x, gamma, stats, dy):
    """-> dx, bound, dgamma, bound, dbeta, bound (from the statistics as they are)"""
    M, D = x.shape
    K, KM = additions(D), min(M, M // 512 + 90) + 4
    gamma = np.ones(D) if gamma is None else gamma
    mean, rstd = stats[:, :1], stats[:, 1:]
    xh = (x - mean) * rstd
    g = dy * gamma
    a, b = g.mean(axis=1, keepdims=True), (g * xh).mean(axis=1, keepdims=True)
    dx = rstd * (g - a - xh * b)
    e_a = (K + 3) * U * np.abs(g).mean(axis=1, keepdims=True)
    e_b = (K + 6) * U * np.abs(g * xh).mean(axis=1, keepdims=True)
    bound = rstd * (4 * U * (np.abs(g) + np.abs(a)) + e_a + np.abs(xh) * (e_b + 6 * U * np.abs(b))) * 1.01 + 2 * U * np.abs(dx)
    dgamma, dbeta = (dy * xh).sum(axis=0), dy.sum(axis=0)
    return dx, bound, dgamma, KM * U * np.abs(dy * xh).sum(axis=0), dbeta, KM * U * np.abs(dy).sum(axis=0)


# ---- gated block ----

def act(g, name):
    """act(g), act'(g), and bounds on what binary32 evaluations of them are off"""
    size = np.abs(g)
    if name == "relu":
        return np.maximum(g, 0.0), (g > 0) * 1.0, 0.0 * g, 0.0 * g
    if name == "silu":
        with np.errstate(over="ignore"):
            p = 1.0 / (1.0 + np.exp(-g))
        return g * p, p * (1.0 + g * (1.0 - p)), 8 * U * size, 16 * U * (1.0 + size)
    if name == "gelu":
        p, q = 0.5 * (1.0 + erf(g / math.sqrt(2.0))), np.exp(-0.5 * g * g) / math.sqrt(2.0 * math.pi)
        # (the exponent's own rounding counts g^2 times)
        return g * p, p + g * q, 8 * U * size, 8 * U + size * q * U * (8 + g * g)
    c, b = math.sqrt(2.0 / math.pi), 0.044715
    z = c * (g + b * g ** 3)
    t = np.tanh(z)
    w = 0.5 * size * c * (1.0 + 3.0 * b * g * g)
    near = 1.0 - t * t
    # tanh off by 4 U of itself and by 4 U of its argument's size times its slope
    e_t = 4 * U * np.abs(t) + 4 * U * np.abs(z) * near
    return 0.5 * g * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * g * near * c * (1.0 + 3.0 * b * g * g), size * e_t + 4 * U * size, \
        e_t + 2 * w * e_t * (np.abs(z) < 12) + 4 * U + 8 * U * w * near


def gated(x, w, name, dtype):
    """-> h, bound, gu, bound"""
    D, F = w.shape[0], w.shape[1] // 2
    gu, size = x @ w, np.abs(x) @ np.abs(w)
    # products (exact in binary32 where they are bfloat16's) and D additions
    e = (D + 1) * U * size
    g, u, eg, eu = gu[:, :F], gu[:, F:], e[:, :F], e[:, F:]
    a, _, ea, _ = act(g, name)
    ea = ea + 1.13 * eg + 16 * U * eg                                            # |act'| <= 1.13
    return a * u, ea * np.abs(u) + np.abs(a) * eu + ea * eu + 2 * U * np.abs(a * u), gu, e


def gated_slopes(gu, dh, name):
    """-> dgu, bound"""
    F = dh.shape[1]
    g, u = gu[:, :F], gu[:, F:]
    a, s, ea, es = act(g, name)
    dgu = np.concatenate((dh * u * s, dh * a), axis=1)
    return dgu, np.concatenate((np.abs(dh * u) * es, np.abs(dh) * ea), axis=1) + 3 * U * np.abs(dgu)


# ---- AdamW ----

def mix(x):
    x = ((x ^ (x >> 16)) * 0x85A308D3) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0xA4093823) & 0xFFFFFFFF
    return x ^ (x >> 16)


def uniform(first, n, seed, step):
    """The two numbers in [0, 1) of each element."""
    key = mix(mix(((seed & 0xFFFFFFFF) + 0x9E3779B1 * (step & 0xFFFFFFFF)) & 0xFFFFFFFF) ^ (seed >> 32))
    i = np.arange(first, first + n, dtype=np.uint64)
    h = (i & np.uint64(0xFFFFFFFF)) * np.uint64(0x9E3779B1) + (i >> np.uint64(32)) * np.uint64(0x7F4A7C15) + np.uint64(key)
    h &= np.uint64(0xFFFFFFFF)
    for shift, factor in ((16, 0x85A308D3), (15, 0xA4093823)):
        h = ((h ^ (h >> np.uint64(shift))) * np.uint64(factor)) & np.uint64(0xFFFFFFFF)
    h ^= h >> np.uint64(16)
    return (h & np.uint64(0xFFFF)).astype(float) / 65536, (h >> np.uint64(16)).astype(float) / 65536


def magnitude(c, bits):
    """k(c, bits) of the header"""
    e, r = c >> bits, c % (1 << bits)
    return float(r) if e == 0 else float(r + (1 << bits)) * 2.0 ** (e - 1)


def decode(codes, scales, bits):
    """What codes [n] with scale bytes [blocks] stand for."""
    table = np.array([magnitude(c & 127 if bits == 3 else c, bits) * (-1 if bits == 3 and c > 127 else 1) for c in range(256)])
    s = np.repeat(np.asarray(scales).astype(float), 128)[:len(codes)]
    return np.where(s == 255, np.nan, table[np.asarray(codes)] * 2.0 ** (s - 127 - 14 - bits))


def steps_of(x, bits):
    """For magnitudes x [n] >= 0 of a tensor: scale byte of every block, and the distance of each element's neighbours."""
    scales, step = [], np.empty_like(x)
    for at in range(0, len(x), 128):
        part = x[at:at + 128]
        most = part.max()
        e = math.floor(math.log2(most)) if most > 0 else -200
        byte = e + 127 + (most > (2.0 - 2.0 ** -bits) * 2.0 ** e)
        byte = 0 if byte < 32 else byte
        scales.append(byte)
        own = np.floor(np.log2(np.maximum(part, 1e-300))) - bits
        step[at:at + 128] = 2.0 ** np.maximum(own, byte - 127 - 14 - bits)
    return np.array(scales), step


def adamw(p, g, m, r, first, o, decay):
    """One step from moments m and r = sqrt(v) -> p, bound, m, bound, r, bound (before moments are rounded)"""
    g = g * o["grad_scale"]
    m1 = o["beta1"] * m + (1 - o["beta1"]) * g
    e_m = 4 * U * (np.abs(o["beta1"] * m) + np.abs((1 - o["beta1"]) * g))
    r1 = np.sqrt(o["beta2"] * r * r + (1 - o["beta2"]) * g * g)
    e_r = 5 * U * r1
    denominator = r1 / math.sqrt(1 - o["beta2"] ** o["step"]) + o["eps"]
    rate = o["lr"] / (1 - o["beta1"] ** o["step"])
    update = rate * m1 / denominator
    out = p * (1 - o["lr"] * decay) - update
    bound = 3 * U * np.abs(p) + 16 * U * np.abs(update) + rate / denominator * e_m + 2 * U * np.abs(out)
    return out, bound, m1, e_m, r1, e_r
