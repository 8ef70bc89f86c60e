"""Performance cases of the layer operators: norm, gated feed-forward block and optimizer step of a training step.

Around the pruned linear layers of such a step stand a layer norm in front of each block (kinds "norm", "norm_grad": the
backward pass gives the input's gradient and those of weight and bias, which are sums over all rows), the gated
feed-forward block ("gated": H = act(X Wg) * (X Wu) with W = [Wg | Wu] of one allocation, and [G | U] where it is kept for
the way back; "gated_grad": the gradients of [G | U], which is the dY of the weights' block-sparse gradient, and of X),
and at the end the optimizer ("adamw": one AdamW step over all of a model's tensors, moments in binary32 or in 8 bits).

Inputs are synthetic: activations are normal with a few columns of larger values, gradients normal and small, weights
normal with the usual scale.  Optimizer states are those of a run under way.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
BLOCK = 128                        # elements that share a scale where moments are held in 8 bits


def listed():
    return [
        # the smallest call: a few tokens of a toy model's width; launches and host work count
        dict(name="norm_few_rows", kind="norm", dtype="bf16", M=8, D=384, pad=0, stats=False),
        # the norm of a batch of 128 images of 196 patches, hidden width 1536, statistics kept for the way back
        dict(name="norm_batch", kind="norm", dtype="bf16", M=25088, D=1536, pad=0, stats=True),
        # backward in binary32, sizes that fit nothing, rows of a wider matrix: a short last batch
        dict(name="norm_grad_ragged_f32", kind="norm_grad", dtype="f32", M=2999, D=805, pad=3),
        # backward of a large batch: the sums over 65536 rows beside the rows' own gradients
        dict(name="norm_grad_batch", kind="norm_grad", dtype="bf16", M=65536, D=2048, pad=0),
        # one token of a model being served: the weights are read once, nothing else counts
        dict(name="gated_one_token", kind="gated", dtype="bf16", act="silu", M=1, D=2048, F=5504, pad=0, save=False),
        # forward in binary32, odd sizes throughout
        dict(name="gated_ragged_f32", kind="gated", dtype="f32", act="gelu", M=997, D=411, F=1003, pad=0, save=True),
        # forward of a training batch: the largest product
        dict(name="gated_batch", kind="gated", dtype="bf16", act="silu", M=8192, D=2048, F=5504, pad=0, save=True),
        # backward, odd sizes, rows of wider matrices
        dict(name="gated_grad_ragged", kind="gated_grad", dtype="bf16", act="gelu_tanh", M=2999, D=805, F=1537, pad=5),
        # backward of 128 images of 196 patches, width 384, hidden width two thirds of an ungated block's 1536
        dict(name="gated_grad_batch", kind="gated_grad", dtype="bf16", act="gelu", M=25088, D=384, F=1024, pad=0),
        # a toy model with odd widths, weights in bfloat16 and their gradients too, 8 bits of state
        dict(name="adamw_toy_8bit", kind="adamw", dtype="bf16", grad="bf16", bits=8, copy=False, layers=4, D=77, F=131, V=1009),
        # binary32 weights with their bfloat16 copy, moments in binary32: 49 million elements in 74 tensors
        dict(name="adamw_model_f32", kind="adamw", dtype="f32", grad="f32", bits=32, copy=True, layers=12, D=512, F=1408, V=32768),
        # the same kind of model, larger, moments in 8 bits: 180 million elements in 146 tensors
        dict(name="adamw_model_8bit", kind="adamw", dtype="f32", grad="bf16", bits=8, copy=True, layers=24, D=768, F=2048, V=50000),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A row length: a third of them whole 64s, a third whole 8s, a third anything."""
    n = _log_int(rng, lo, hi)
    unit = rng.choice((64, 8, 1))
    return max(unit, n // unit * unit)


def draw(rng):
    """One more case; its work is bounded by the largest listed case of its kind."""
    kind = rng.choice(("norm", "norm_grad", "gated", "gated_grad", "adamw"))
    while True:
        case = dict(kind=kind, dtype=rng.choice(("bf16", "bf16", "f32")))
        if kind in ("norm", "norm_grad"):
            case.update(M=_log_int(rng, 1, 65536), D=_width(rng, 64, 16384), pad=rng.choice((0, 0, 8, 3)))
            if kind == "norm":
                case["stats"] = rng.random() < 0.5
            fits = work(case)["bytes"] <= 800e6
        elif kind in ("gated", "gated_grad"):
            case.update(act=rng.choice(("silu", "gelu", "gelu_tanh", "relu")), M=_log_int(rng, 1, 16384), D=_width(rng, 64, 4096),
                        F=_width(rng, 64, 8192), pad=rng.choice((0, 0, 0, 8, 5)))
            if kind == "gated":
                case["save"] = rng.random() < 0.5
            fits = work(case)["flops"] <= (360e9 if case["dtype"] == "bf16" else 90e9)
        else:
            case.update(grad="bf16" if case["dtype"] == "bf16" else rng.choice(("f32", "bf16")), bits=rng.choice((8, 32)),
                        copy=case["dtype"] == "f32" and rng.random() < 0.5, layers=rng.randint(1, 32), D=_width(rng, 64, 1024),
                        F=_width(rng, 64, 4000), V=_log_int(rng, 500, 60000))
            fits = work(case)["bytes"] <= 2.5e9
        if fits:
            return case


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _randn(gen, *size):
    return torch.randn(*size, generator=gen, device="cuda")


def _rows(x, pad, dtype):
    """The matrix with `pad` more elements between its rows."""
    wide = torch.zeros(x.shape[0], x.shape[1] + pad, dtype=dtype, device="cuda")
    wide[:, :x.shape[1]] = x
    return wide[:, :x.shape[1]]


def _activations(gen, M, D):
    return _randn(gen, M, D) * (1.0 + 6.0 * (torch.rand(D, generator=gen, device="cuda") < 0.02)) + 0.3 * _randn(gen, D)


def _sizes(case):
    """(elements, weight decay) of a model's tensors: token table, then per layer two norms, two blocks of weights, two
    that mix the width."""
    D, F = case["D"], case["F"]
    layer = [(D, 0.0), (D, 0.0), (D * 2 * F, 0.1), (F * D, 0.1), (D * D, 0.1), (D * D, 0.1)]
    return [(case["V"] * D, 0.01)] + layer * case["layers"] + [(D, 0.0)]


def _segments(case):
    """First element, elements, weight decay of each tensor in buffers that hold them all, each from a whole block on."""
    at, found = 0, []
    for n, decay in _sizes(case):
        found.append((at, n, decay))
        at += -(-n // BLOCK) * BLOCK
    return found, at


def prepare(case, seed):
    gen, kind, s = _generator(seed), case["kind"], dict(case)
    dtype = DTYPES[case["dtype"]]
    if kind in ("norm", "norm_grad"):
        M, D = case["M"], case["D"]
        s["X"] = _rows(_activations(gen, M, D), case["pad"], dtype)
        s["gamma"], s["beta"] = (1.0 + 0.2 * _randn(gen, D)).to(dtype), (0.1 * _randn(gen, D)).to(dtype)
        s["eps"] = 1e-5
        if kind == "norm_grad":
            s["dY"] = _rows(1e-3 * _randn(gen, M, D), case["pad"], dtype)
            s["stats"] = _stats(s["X"], s["eps"])
    elif kind in ("gated", "gated_grad"):
        M, D, F = case["M"], case["D"], case["F"]
        s["W"] = (_randn(gen, D, 2 * F) * D ** -0.5).to(dtype)
        if kind == "gated":
            s["X"] = _rows(_activations(gen, M, D), case["pad"], dtype)
        else:
            s["GU"] = _rows(_randn(gen, M, 2 * F) * 1.5, case["pad"], dtype)
            s["dH"] = _rows(1e-3 * _randn(gen, M, F), case["pad"], dtype)
    else:
        segments, total = _segments(case)
        there = torch.zeros(total, device="cuda")
        s["decay"] = torch.zeros(total // BLOCK, device="cuda")
        for at, n, decay in segments:
            there[at:at + n] = 1.0
            s["decay"][at // BLOCK:(at + n + BLOCK - 1) // BLOCK] = decay
        size = torch.exp(0.7 * _randn(gen, total // BLOCK)).repeat_interleave(BLOCK) * there
        s["param"] = (0.02 * _randn(gen, total) * there).to(dtype)
        s["grad_flat"] = (1e-3 * _randn(gen, total) * size).to(DTYPES[case["grad"]])
        s["copy_flat"] = s["param"].bfloat16() if case["copy"] else None
        m = 3e-4 * _randn(gen, total) * size
        r = 1e-3 * torch.exp(0.5 * _randn(gen, total)) * size
        s.update(segments=segments, lr=3e-4, beta1=0.9, beta2=0.999, eps=1e-8, step=1000, grad_scale=0.7, seed=int(seed) % (1 << 31))
        if case["bits"] == 32:
            s["m"], s["v"] = m, r * r
        else:
            half = torch.full((total,), 0.5, device="cuda")
            s["m"], ms = _encode(m, half, 3)
            s["r"], rs = _encode(r, half, 4)
            s["scales"] = torch.stack((ms, rs))
    return s


# ---------------------------------------------------------------------------
# the operators in their plain form
# ---------------------------------------------------------------------------

def _stats(X, eps):
    """[M, 2]: mean, 1 / sqrt(variance + eps)."""
    x = X.float()
    mean = x.mean(dim=1, keepdim=True)
    d = x - mean
    return torch.cat((mean, 1.0 / torch.sqrt((d * d).mean(dim=1, keepdim=True) + eps)), dim=1)


def _plain_norm(s):
    stats = _stats(s["X"], s["eps"])
    y = (s["X"].float() - stats[:, :1]) * stats[:, 1:] * s["gamma"].float() + s["beta"].float()
    return (y.to(s["X"].dtype), stats) if s["stats"] else y.to(s["X"].dtype)


def _plain_norm_grad(s):
    dy, rstd = s["dY"].float(), s["stats"][:, 1:]
    xh = (s["X"].float() - s["stats"][:, :1]) * rstd
    g = dy * s["gamma"].float()
    dx = rstd * (g - g.mean(dim=1, keepdim=True) - xh * (g * xh).mean(dim=1, keepdim=True))
    return dx.to(s["X"].dtype), (dy * xh).sum(dim=0), dy.sum(dim=0)


def _act(g, act):
    """act(g) and its derivative."""
    if act == "relu":
        return torch.clamp_min(g, 0.0), (g > 0).float()
    if act == "silu":
        p = 1.0 / (1.0 + torch.exp(-g))
        return g * p, p * (1.0 + g * (1.0 - p))
    if act == "gelu":
        p = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
        return g * p, p + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))
    c, b = math.sqrt(2.0 / math.pi), 0.044715
    t = torch.tanh(c * (g + b * g * g * g))
    return 0.5 * g * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * g * (1.0 - t * t) * c * (1.0 + 3.0 * b * g * g)


def _plain_gated(s):
    F, dtype = s["F"], s["X"].dtype
    gu = s["X"].float() @ s["W"].float()
    h = (_act(gu[:, :F], s["act"])[0] * gu[:, F:]).to(dtype)
    return (h, gu.to(dtype)) if s["save"] else h


def _plain_gated_grad(s):
    F, dtype = s["F"], s["GU"].dtype
    g, u, dh = s["GU"][:, :F].float(), s["GU"][:, F:].float(), s["dH"].float()
    a, slope = _act(g, s["act"])
    dgu = torch.cat((dh * u * slope, dh * a), dim=1)
    return (dgu @ s["W"].float().t()).to(dtype), dgu.to(dtype)


# Moments in 8 bits: a magnitude of 4 bits of exponent and `bits` of fraction (m: 3 and a sign, r = sqrt(v): 4 and none), in
# units of a power of two that a block of 128 shares: 2^(scale byte - 127 - 14 - bits).  Rounded to one of the two neighbours by
# a number u in [0, 1): floor(x / step + u).  A positive r is never rounded to 0.

def _decode(codes, scales, bits):
    c = codes.long()
    magnitude = c & 127 if bits == 3 else c
    e, f = magnitude >> bits, magnitude & ((1 << bits) - 1)
    n = torch.where(e > 0, (f + (1 << bits)) << (e - 1).clamp_min(0), f).float()
    x = n.view(-1, BLOCK) * torch.exp2(scales.float() - (127.0 + 14.0 + bits))[:, None]
    x = torch.where((scales == 255)[:, None], float("nan"), x).view(-1)
    return torch.where(c > 127, -x, x) if bits == 3 else x


def _encode(x, u, bits):
    """-> codes, scale bytes"""
    a = torch.abs(x)
    most = a.view(-1, BLOCK).amax(dim=1)
    part, e = torch.frexp(most)                       # most = part * 2^e, part in [1/2, 1)
    scale = e.long() + 126 + (part > 1.0 - 0.5 ** (bits + 1)).long()
    scale = torch.where((most == 0) | (scale < 32), 0, torch.where(torch.isfinite(most), scale.clamp_max(255), 255))
    least = (scale - (127 + 14 + bits)).repeat_interleave(BLOCK)          # exponent of the block's unit
    ex = torch.maximum(torch.frexp(a)[1].long() - (1 + bits), least)      # exponent of this element's step
    n = torch.floor(a * torch.exp2(-ex.to(a.dtype)) + u).long()
    if bits == 4:
        n = torch.where(a > 0, n.clamp_min(1), n)
    code = n + ((ex - least) << bits)
    code = torch.where(scale.repeat_interleave(BLOCK) % 255 == 0, 0, code.clamp(0, 127 if bits == 3 else 255))
    if bits == 3:
        code = torch.where((x < 0) & (code > 0), code + 128, code)
    return code.to(torch.uint8), scale.to(torch.uint8)


def _mix(x):
    """A 32-bit number's bits spread over 32 bits."""
    x = (x ^ (x >> 16)) * 0x85A308D3 & 0xFFFFFFFF
    x = (x ^ (x >> 15)) * 0xA4093823 & 0xFFFFFFFF
    return x ^ (x >> 16)


def _uniform(first, count, seed, step):
    """Two numbers in [0, 1), multiples of 2^-16, for each element of the whole list of tensors."""
    key = _mix(_mix((seed & 0xFFFFFFFF) + 0x9E3779B1 * step & 0xFFFFFFFF) ^ (seed >> 32))
    i = torch.arange(first, first + count, device="cuda")
    h = _mix(((i & 0xFFFFFFFF) * 0x9E3779B1 + (i >> 32) * 0x7F4A7C15 + key) & 0xFFFFFFFF)
    return (h & 0xFFFF).float() * 2.0 ** -16, (h >> 16).float() * 2.0 ** -16


def _plain_adamw(s):
    b1, b2, t, lr = s["beta1"], s["beta2"], s["step"], s["lr"]
    g = s["grad_flat"].float() * s["grad_scale"]
    if s["bits"] == 32:
        m, v = b1 * s["m"] + (1.0 - b1) * g, b2 * s["v"] + (1.0 - b2) * g * g
        r = torch.sqrt(v)
    else:
        old = _decode(s["r"], s["scales"][1], 4)
        m = b1 * _decode(s["m"], s["scales"][0], 3) + (1.0 - b1) * g
        r = torch.sqrt(b2 * old * old + (1.0 - b2) * g * g)
    p = s["param"].float()
    keep = (1.0 - lr * s["decay"]).repeat_interleave(BLOCK)
    p = p * keep - (lr / (1.0 - b1 ** t)) * m / (r * (1.0 / math.sqrt(1.0 - b2 ** t)) + s["eps"])
    s["param"].copy_(p)
    out = [s["param"]]
    if s["copy_flat"] is not None:
        out.append(s["copy_flat"].copy_(p))
    if s["bits"] == 32:
        return out + [s["m"].copy_(m), s["v"].copy_(v)]
    um, ur = _uniform(0, p.numel(), s["seed"], t)
    s["m"], ms = _encode(m, um, 3)
    s["r"], rs = _encode(r, ur, 4)
    s["scales"] = torch.stack((ms, rs))
    # the values that the codes stand for; bfloat16 holds them exactly
    return out + [_decode(s["m"], ms, 3).bfloat16(), _decode(s["r"], rs, 4).bfloat16()]


def _own_adamw(B, s):
    if "batch" not in s:                              # a program's tensors stay where they are, and so does the list of them
        # (whole blocks: what fills a buffer up to the next tensor is stepped with the tensor before it, as the plain form does)
        ends = [at + -(-n // BLOCK) * BLOCK for at, n, _ in s["segments"]]
        parts = [slice(at, end) for (at, _, _), end in zip(s["segments"], ends)]

        def part(flat):
            return [flat[x] for x in parts]
        if s["bits"] == 32:
            states = list(zip(part(s["m"]), part(s["v"])))
        else:
            states = [(s["m"][x], s["r"][x], s["scales"][:, x.start // BLOCK:x.stop // BLOCK]) for x in parts]
        s["batch"] = B.AdamWBatch(part(s["param"]), part(s["grad_flat"]), bits=s["bits"], states=states,
                                  copies=part(s["copy_flat"]) if s["copy_flat"] is not None else None,
                                  weight_decay=[d for _, _, d in s["segments"]])
    B.bsr_adamw_batched(s["batch"], lr=s["lr"], step=s["step"], beta1=s["beta1"], beta2=s["beta2"], eps=s["eps"],
                        grad_scale=s["grad_scale"], seed=s["seed"])
    out = [s["param"]] + ([s["copy_flat"]] if s["copy_flat"] is not None else [])
    if s["bits"] == 32:
        return out + [s["m"], s["v"]]
    return out + [B.bsr_adamw_state_values(s["m"], s["scales"][0], "m", dtype=torch.bfloat16),
                  B.bsr_adamw_state_values(s["r"], s["scales"][1], "r", dtype=torch.bfloat16)]


def run(s):
    kind = s["kind"]
    if own:
        from paper_2311_16883_amd import binding as B
        if kind == "norm":
            return B.bsr_layer_norm(s["X"], s["gamma"], s["beta"], eps=s["eps"], want_stats=s["stats"])
        if kind == "norm_grad":
            return B.bsr_layer_norm_grad(s["X"], s["gamma"], s["stats"], s["dY"])
        if kind == "gated":
            return B.bsr_gated_ff(s["X"], s["W"], act=s["act"], want_GU=s["save"])
        if kind == "gated_grad":
            return B.bsr_gated_ff_grad(s["GU"], s["dH"], s["W"], act=s["act"])
        return _own_adamw(B, s)
    if kind == "norm":
        return _plain_norm(s)
    if kind == "norm_grad":
        return _plain_norm_grad(s)
    if kind == "gated":
        return _plain_gated(s)
    if kind == "gated_grad":
        return _plain_gated_grad(s)
    return _plain_adamw(s)


# ---------------------------------------------------------------------------
# the work of a pass
# ---------------------------------------------------------------------------

def work(case):
    kind, e = case["kind"], SIZE[case["dtype"]]
    if kind in ("norm", "norm_grad"):
        M, D = case["M"], case["D"]
        if kind == "norm":
            return {"bytes": 2 * M * D * e + 2 * D * e + (8 * M if case["stats"] else 0), "flops": 7 * M * D}
        return {"bytes": 3 * M * D * e + D * e + 8 * M + 8 * D, "flops": 13 * M * D}
    if kind in ("gated", "gated_grad"):
        M, D, F = case["M"], case["D"], case["F"]
        weights = 2 * D * F * e
        if kind == "gated":
            return {"bytes": weights + M * D * e + M * F * e * (3 if case["save"] else 1), "flops": 4 * M * D * F}
        return {"bytes": weights + 5 * M * F * e + M * D * e, "flops": 4 * M * D * F}
    n = sum(k for k, _ in _sizes(case))
    moments = 16.0 if case["bits"] == 32 else 4.0 + 4.0 / BLOCK + 6.0      # 8 bits: read, written, and read once more as values
    return {"bytes": n * (2 * e + SIZE[case["grad"]] + (2 if case["copy"] else 0) + moments), "flops": 15 * n}


# ---------------------------------------------------------------------------
# the operators from their definitions, in 64 bits
# ---------------------------------------------------------------------------

def _exact_act(g, act):
    f = torch.nn.functional
    return {"relu": f.relu, "silu": f.silu, "gelu": f.gelu, "gelu_tanh": lambda x: f.gelu(x, approximate="tanh")}[act](g)


def _exact_code(x, u, bits):
    """The value that an 8-bit moment stands for after rounding, a block per row."""
    most = x.abs().amax(dim=1, keepdim=True)
    top = torch.floor(torch.log2(most.clamp_min(1e-300)))
    top = top + (most > (2.0 - 2.0 ** -bits) * torch.exp2(top))
    unit = torch.exp2(top - 14 - bits)
    size = torch.exp2(torch.floor(torch.log2(x.abs().clamp_min(1e-300))) - bits)
    step = torch.maximum(size, unit)
    n = torch.floor(x.abs() / step + u)
    if bits == 4:
        n = torch.where(x > 0, n.clamp_min(1.0), n)
    return torch.where(top < 32 - 127, 0.0, n * step * torch.sign(x))


def _exact_moments(s):
    """The moments that the codes stand for, by a table of all 256 codes."""
    def values(bits):
        v = []
        for c in range(256):
            k = c % 128 if bits == 3 else c
            e, f = k >> bits, k % (1 << bits)
            v.append((f if e == 0 else (f + (1 << bits)) * 2.0 ** (e - 1)) * (-1.0 if bits == 3 and c > 127 else 1.0) * 2.0 ** -(14 + bits))
        return torch.tensor(v, dtype=torch.float64, device="cuda")
    unit = torch.exp2(s["scales"].double() - 127.0)
    return tuple((values(bits)[s[name].int()].view(-1, BLOCK) * unit[row][:, None]) for name, bits, row in (("m", 3, 0), ("r", 4, 1)))


def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind == "norm":
        x = s["X"].double()
        y = torch.nn.functional.layer_norm(x, (s["D"],), s["gamma"].double(), s["beta"].double(), s["eps"])
        var, mean = torch.var_mean(x, dim=1, unbiased=False)
        return (y, torch.stack((mean, (var + s["eps"]) ** -0.5), dim=1)) if s["stats"] else y
    if kind == "norm_grad":
        x, gamma = s["X"].double().requires_grad_(), s["gamma"].double().requires_grad_()
        beta = torch.zeros_like(gamma).requires_grad_()
        torch.nn.functional.layer_norm(x, (s["D"],), gamma, beta, s["eps"]).backward(s["dY"].double())
        return x.grad, gamma.grad, beta.grad
    if kind == "gated":
        g, u = (s["X"].double() @ s["W"].double()).split(s["F"], dim=1)
        h = _exact_act(g, s["act"]) * u
        return (h, torch.cat((g, u), dim=1)) if s["save"] else h
    if kind == "gated_grad":
        gu = s["GU"].double().requires_grad_()
        g, u = gu.split(s["F"], dim=1)
        (_exact_act(g, s["act"]) * u).backward(s["dH"].double())
        return gu.grad @ s["W"].double().t(), gu.grad
    g = s["grad_flat"].double().view(-1, BLOCK) * s["grad_scale"]
    m, r = _exact_moments(s) if s["bits"] == 8 else (s["m"].double().view(-1, BLOCK), s["v"].double().view(-1, BLOCK).sqrt())
    m = m + (1.0 - s["beta1"]) * (g - m)
    v = r * r + (1.0 - s["beta2"]) * (g * g - r * r)
    t = s["step"]
    p = s["param"].double().view(-1, BLOCK)
    p = p - s["lr"] * s["decay"].double()[:, None] * p
    p = p - s["lr"] * (m / (1.0 - s["beta1"] ** t)) / (torch.sqrt(v / (1.0 - s["beta2"] ** t)) + s["eps"])
    out = [p.view(-1)] + ([p.view(-1)] if s["copy_flat"] is not None else [])
    if s["bits"] == 32:
        return out + [m.view(-1), v.view(-1)]
    um, ur = _uniform(0, p.numel(), s["seed"], t)
    return out + [_exact_code(m, um.double().view(-1, BLOCK), 3).view(-1), _exact_code(v.sqrt(), ur.double().view(-1, BLOCK), 4).view(-1)]
