"""Token operators at the sizes from which rows pass by the caches, with whole-line accesses in place of those at any alignment: just
above and just below each size, and above it with a pitch or an address that rules it out.  And the table gradient's sorts of more than
half a million positions, and the longest rows of logits with the most entries.  Compared on the device, in binary64."""
import numpy as np
import pytest
import torch

import token_plain as P
from paper_2311_16883_amd import binding as B
from test_gpu_token_ops import DT, IX, check, f64, student

pytestmark = pytest.mark.gpu

MIB = 1 << 20
LINE = {"f32": 32, "bf16": 64}                       # elements of 128 bytes


def randn(seed, *size, dtype):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*size, generator=g, device="cuda").to(DT[dtype])


def placed(x, how):
    """The same matrix in rows of whole lines ("lines"), with a pitch of 16 bytes more, or 16 bytes into its buffer; NaN around it."""
    extra = 16 // x.element_size()
    rows, cols = x.shape
    ld, offset = cols + (extra if how == "pitch" else 0), extra if how == "address" else 0
    buf = torch.full((rows * ld + offset,), float("nan"), dtype=x.dtype, device="cuda")
    view = buf[offset:].view(rows, ld)[:, :cols]
    view.copy_(x)
    assert (view.data_ptr() % 128 == 0) == (how != "address")
    return view


def nothing_else_written(view, how):
    rows, cols = view.shape
    return how != "pitch" or bool(torch.isnan(torch.as_strided(view, (rows - 1, view.stride(0) - cols), view.stride(), view.storage_offset() + cols)).all())


def close(got, want, bound, dtype):
    """As check(), on the device."""
    got = got.double()
    tol = bound + (P.BF16 * (want.abs() + bound) + 1e-40 if dtype == "bf16" else 0.0)
    bad = ~((got - want).abs() <= tol)
    assert not bool(bad.any()), (int(bad.sum()), torch.nonzero(bad)[:3].tolist(), got[bad][:3].tolist(), want[bad][:3].tolist())


def rows_of(mib, D, dtype):
    return mib * MIB // (D * (4 if dtype == "f32" else 2))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lines,less,how", [(16, 0, "lines"), (16, 1, "lines"), (1, 0, "lines"), (33, -7, "lines"), (16, 0, "pitch"),
                                            (16, 0, "address")])
def test_lookup_of_32_mib(dtype, lines, less, how):
    D, V = lines * LINE[dtype], 3000
    T = rows_of(32, D, dtype) - less + (1 if 32 * MIB % (lines * 128) else 0)
    table = randn(1, V, D, dtype=dtype)
    tokens = torch.randint(-1, V + 1, (T,), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    out = placed(torch.zeros(T, D, dtype=DT[dtype], device="cuda"), how)
    assert B.bsr_embedding_lookup(table, tokens, scale=1.7, out=out) is out and nothing_else_written(out, how)
    want = (table[tokens.clamp(0, V - 1)].float() * torch.tensor(1.7, device="cuda")).to(DT[dtype])
    want[(tokens < 0) | (tokens >= V)] = 0
    assert torch.equal(out, want)


def experts(T, k, E, align):
    """Choices, some dropped, sorted on the host's word (torch's stable sort)."""
    g = torch.Generator(device="cuda").manual_seed(T + k)
    ids = torch.randint(0, E, (T, k), generator=g, device="cuda")
    ids[torch.rand(T, k, generator=g, device="cuda") < 0.02] = -1
    flat = torch.where(ids < 0, E, ids).reshape(-1)
    counts = torch.bincount(flat, minlength=E + 1)[:E]
    ends = torch.cumsum((counts + align - 1) // align * align, 0)
    starts, before = ends - (counts + align - 1) // align * align, torch.cumsum(counts, 0) - counts
    entries = torch.argsort(flat, stable=True)[:int(counts.sum())]
    e = flat[entries]
    place = starts[e] + torch.arange(len(entries), device="cuda") - before[e]
    rows = P.capacity(T * k, E, align)
    order = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    order[place] = entries.int()
    slots = torch.full((T * k,), -1, dtype=torch.int32, device="cuda")
    slots[entries] = place.int()
    return order, slots.view(T, k)


def trimmed(T, k, rows, E=8):
    """The same with exactly `rows` rows in the sorted matrix: as many of padding at its end, or the last rows' entries dropped."""
    order, slots = experts(T, k, E, 16)
    if rows <= len(order):
        order = order[:rows].clone()
        slots = torch.where(slots < rows, slots, -1)
    else:
        order = torch.cat((order, torch.full((rows - len(order),), -1, dtype=torch.int32, device="cuda")))
    return order, slots


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lines,k,less,how", [(16, 2, 0, "lines"), (16, 2, 1, "lines"), (1, 1, 0, "lines"), (32, 4, -9, "lines"),
                                              (16, 2, 0, "pitch"), (16, 2, 0, "address")])
def test_gather_of_32_mib(dtype, lines, k, less, how):
    D = lines * LINE[dtype]
    rows = rows_of(32, D, dtype) - less
    T = rows // k - 40
    order, slots = trimmed(T, k, rows)
    X = randn(3, T, D, dtype=dtype)
    Xs = placed(torch.ones(rows, D, dtype=DT[dtype], device="cuda"), how)
    assert B.bsr_expert_gather(X, slots, order, out=Xs) is Xs and nothing_else_written(Xs, how)
    want = X[order.long().clamp_min(0) // k]
    want[order < 0] = 0
    assert torch.equal(Xs, want)


def returned(Ys, slots, weights):
    out = torch.zeros(slots.shape[0], Ys.shape[1], dtype=torch.float64, device="cuda")
    size = torch.zeros_like(out)
    for j in range(slots.shape[1]):
        t = torch.nonzero(slots[:, j] >= 0)[:, 0]
        term = Ys[slots[t, j].long()].double() * (1.0 if weights is None else weights[t, j].double()[:, None])
        out[t] += term
        size[t] += term.abs()
    return out, (slots.shape[1] + 1) * P.U * size + 1e-44


# MiB of the rows that are read and of those that are written, of 64 and 32: both above, one, none
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T_mib,k,rows_mib,more,how", [
    (32, 3, 64, 0, "lines"), (33, 2, 64, 0, "lines"), (32, 5, 65, 0, "lines"), (31, 3, 64, 0, "lines"), (16, 5, 64, 0, "lines"),
    (20, 2, 64, 0, "lines"), (32, 1, 63, 0, "lines"), (32, 1, 64, -1, "lines"), (34, 2, 63, 0, "lines"), (34, 4, 63, 0, "lines"),
    (35, 7, 62, 0, "lines"), (31, 1, 63, 0, "lines"), (33, 2, 65, 0, "pitch"), (33, 4, 65, 0, "address"), (33, 8, 65, 0, "pitch")])
def test_return_of_64_mib(dtype, T_mib, k, rows_mib, more, how):
    D = 16 * LINE[dtype]
    T, rows = rows_of(T_mib, D, dtype), rows_of(rows_mib, D, dtype) + more
    order, slots = trimmed(T, k, rows)
    Ys = randn(4, rows, D, dtype=dtype)
    Ys[order < 0] = float("nan")
    weights = torch.rand(T, k, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda")
    for w in (weights, None):
        want, bound = returned(Ys, slots, w)
        out = placed(torch.ones(T, D, dtype=DT[dtype], device="cuda"), how)
        assert B.bsr_expert_combine(placed(Ys, how), slots, w, out=out) is out and nothing_else_written(out, how)
        close(out, want, bound, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("k,rows_mib,more,ys_how,how", [
    (2, 64, 0, "lines", "lines"), (3, 64, 0, "lines", "lines"), (6, 65, 0, "lines", "lines"), (2, 64, -1, "lines", "lines"),
    (2, 32, 0, "lines", "lines"), (4, 33, 0, "lines", "lines"), (8, 33, 0, "lines", "lines"), (2, 32, -1, "lines", "lines"),
    (2, 65, 0, "pitch", "lines"), (4, 65, 0, "lines", "pitch"), (8, 65, 0, "address", "address"), (2, 65, 0, "lines", "address")])
def test_gradient_of_the_return_of_64_mib(dtype, k, rows_mib, more, ys_how, how):
    D = 16 * LINE[dtype]
    rows = rows_of(rows_mib, D, dtype) + more
    T = rows // k - 30
    order, slots = trimmed(T, k, rows)
    Ys, dOut = randn(6, rows, D, dtype=dtype), randn(7, T, D, dtype=dtype)
    Ys[order < 0] = float("nan")
    w = torch.rand(T, k, generator=torch.Generator(device="cuda").manual_seed(8), device="cuda")
    dYs = placed(torch.ones(rows, D, dtype=DT[dtype], device="cuda"), how)
    got, dw = B.bsr_expert_combine_grad(placed(Ys, ys_how), slots, order, w, dOut, dYs=dYs)
    assert got is dYs and nothing_else_written(dYs, how)
    entry = order.long().clamp_min(0)
    want = w.reshape(-1)[entry].double()[:, None] * dOut[entry // k].double()
    want[order < 0] = 0
    close(dYs, want, P.U * want.abs() + 1e-44, dtype)
    for j in range(k):
        t = torch.nonzero(slots[:, j] >= 0)[:, 0]
        terms = Ys[slots[t, j].long()].double() * dOut[t].double()
        close(dw[t, j], terms.sum(dim=1), (D + 1) * P.U * terms.abs().sum(dim=1) + 1e-44, "f32")
    assert not dw[slots < 0].any()


def table_gradient(tokens, dY, V, scale):
    keep = torch.nonzero((tokens >= 0) & (tokens < V))[:, 0]
    at, rows = tokens[keep].long(), dY[keep].double() * scale
    dE = torch.zeros(V, dY.shape[1], dtype=torch.float64, device="cuda").index_add_(0, at, rows)
    size = torch.zeros_like(dE).index_add_(0, at, rows.abs())
    return dE, (torch.bincount(at, minlength=V)[:, None] + 1) * P.U * size + 1e-44


def text(T, V, index, seed):
    """Tokens as frequent as in text, some positions without one."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = (torch.exp(torch.rand(T, generator=g, device="cuda").double() * np.log(V + 1.0)).long() - 1).clamp(0, V - 1)
    t[torch.rand(T, generator=g, device="cuda") < 0.03] = -1
    t[torch.rand(T, generator=g, device="cuda") < 0.01] = V
    return t.to(IX[index])


@pytest.mark.parametrize("dtype,index", [("f32", "i32"), ("bf16", "i64")])
@pytest.mark.parametrize("lines,V,less,how", [(16, 5000, 0, "lines"), (16, 5000, 1, "lines"), (16, 400000, 0, "lines"), (3, 70000, -5, "lines"),
                                              (64, 20000, 0, "lines"), (16, 5000, 0, "pitch"), (16, 5000, 0, "address")])
def test_table_gradient_of_96_mib(dtype, index, lines, V, less, how):
    D = lines * LINE[dtype]
    T = rows_of(96, D, dtype) - less
    tokens, dY = text(T, V, index, T), randn(9, T, D, dtype=dtype)
    dY[(tokens < 0) | (tokens >= V)] = float("nan")
    got = B.bsr_embedding_grad(tokens, placed(dY, how), V, scale=0.75)
    want, bound = table_gradient(tokens, dY, V, 0.75)
    close(got, want, bound, "f32")


@pytest.mark.parametrize("index", ["i32", "i64"])
@pytest.mark.parametrize("T", [524288, 524289, 700001])
@pytest.mark.parametrize("V", [900, 50000, 2000003])
def test_table_gradient_of_more_than_half_a_million_positions(index, T, V):
    """One, two and three digits, each from the tokens or from the pairs that the digit before left."""
    tokens, dY = text(T, V, index, V), randn(10, T, 8, dtype="f32")
    got = B.bsr_embedding_grad(tokens, dY, V)
    want, bound = table_gradient(tokens, dY, V, 1.0)
    close(got, want, bound, "f32")
    # one position per token: a permutation, exact
    order = torch.randperm(T, generator=torch.Generator().manual_seed(T)).cuda().to(IX[index])
    got = B.bsr_embedding_grad(order, dY, T + 3)
    exact = torch.zeros(T + 3, 8, device="cuda")
    exact[order.long()] = dY
    assert torch.equal(got, exact)


@pytest.mark.parametrize("dtype,V", [("bf16", 262144), ("f32", 131071), ("bf16", 130001)])
def test_the_longest_rows_of_logits_with_the_most_entries(dtype, V):
    """Rows that a compute unit has one of: registers, shared memory for their last quarter, and for 1024 entries."""
    N, K = 98, 1024
    z, ids, t, dloss = student(N, V, K, V, dtype, "f32")
    part = torch.tensor([0, 1, 2, 3, 4, 50, N - 1])
    args = z.cuda(), ids.cuda(), t.cuda(), dloss.cuda()
    loss, grad = B.bsr_distill_loss_grad(*args, 0.9)
    want, _, g, el, eg = P.distill(f64(z[part]), ids[part].numpy(), f64(t[part]), float(np.float32(0.9)), f64(dloss[part]))
    check(loss[part], want, el)
    check(grad[part], g, eg, dtype)


def test_table_gradient_of_more_than_a_billion_positions():
    """Windows of the longest kind: a few tokens at either end and around 2^30, nothing in between."""
    T, V, D = (1 << 30) + 777, 50, 2
    tokens = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    dY = torch.full((T, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    at = torch.cat([torch.arange(a, a + 3000) for a in (0, (1 << 29) - 1500, (1 << 30) - 2300)]).cuda()
    tokens[at] = text(len(at), V, "i32", 1).clamp_min(0).clamp_max(V - 1)
    dY[at] = torch.randint(-8, 9, (len(at), D), generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).cuda()
    got = B.bsr_embedding_grad(tokens, dY, V, scale=0.5)
    want = torch.zeros(V, D, dtype=torch.float64, device="cuda").index_add_(0, tokens[at].long(), dY[at].double() * 0.5)
    assert torch.equal(got.double(), want)                 # small whole numbers: exact in any order
    del tokens, dY
    torch.cuda.empty_cache()
