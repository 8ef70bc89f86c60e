"""Token operators on the GPU against the plain binary64 implementation (token_plain.py), at the sizes, strides, alignments and
masks where they can go wrong.  Copies, scaled rows and index arrays are compared exactly, sums within the bounds that
token_plain derives from the number and size of their terms."""
import numpy as np
import pytest
import torch

import token_plain as P
from paper_2311_16883_amd import binding as B

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
IX = {"i32": torch.int32, "i64": torch.int64}


def randn(seed, *size, dtype="f32", scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*size, generator=g) * scale).to(DT[dtype])


def f64(x):
    return x.detach().cpu().double().numpy()


def strided(x, pad=0, offset=0, fill=float("nan")):
    """The same matrix on the GPU with `pad` more elements per row and `offset` elements into its buffer, NaN around it."""
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
    inside = buf[offset:offset + rows * ld].view(rows, ld)
    if rows:
        inside[:, :cols] = fill
    return bool((buf == fill).all())


def check(got, want, bound, dtype="f32"):
    """|got - want| within the binary32 bound, and the one rounding to bfloat16."""
    got, want = f64(got), np.asarray(want)
    assert got.shape == want.shape
    tol = np.broadcast_to(bound, want.shape) + (P.BF16 * (np.abs(want) + bound) + 1e-40 if dtype == "bf16" else 0.0)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:3].tolist(), got[bad][:3], want[bad][:3], np.asarray(tol)[bad][:3])


# ---- token table ----

@pytest.mark.parametrize("dtype,index", [("f32", "i32"), ("bf16", "i64"), ("bf16", "i32"), ("f32", "i64")])
@pytest.mark.parametrize("T,V,D,pad,offset", [
    (1, 1, 1, 0, 0), (1, 50, 64, 0, 0), (5, 3, 3, 2, 1), (7, 100, 7, 1, 3), (64, 1000, 8, 0, 0), (33, 20, 130, 6, 1),
    (200, 5000, 411, 0, 0), (16, 300, 1024, 0, 0), (3, 11, 5001, 7, 5), (1000, 64, 96, 32, 0)])
def test_lookup(dtype, index, T, V, D, pad, offset):
    table = randn(1, V, D, dtype=dtype)
    g = torch.Generator().manual_seed(2)
    tokens = torch.randint(-1, V + 1, (T,), generator=g).to(IX[index])       # some outside: -1 and V
    scale = 1.7
    src = strided(table, pad, offset)
    out = strided(torch.zeros(T, D, dtype=DT[dtype]), pad, offset, fill=7.0)
    got = B.bsr_embedding_lookup(src, tokens.cuda(), scale=scale, out=out)
    assert got is out and around_is_untouched(out, pad, offset, 7.0)
    there = (tokens >= 0) & (tokens < V)
    want = table[tokens.long().clamp(0, V - 1)].float() * torch.tensor(scale, dtype=torch.float32)
    want = torch.where(there[:, None], want, torch.zeros(())).to(DT[dtype])
    assert torch.equal(got.cpu(), want)
    check(got, P.lookup(f64(table), tokens.numpy(), float(np.float32(scale))), P.U * np.abs(f64(want)), dtype)


def test_more_rows_than_a_launch_has_lanes_for():
    """2^26 tokens and more, at 16 lanes a row: more than 2^30 lanes, and 2^32 for rows of 64 lanes."""
    T = (1 << 26) + 5
    tokens = torch.arange(T, dtype=torch.int32, device="cuda") % 1000
    table = torch.arange(1000, dtype=torch.float32, device="cuda")[:, None].expand(1000, 2).bfloat16().contiguous()
    out = B.bsr_embedding_lookup(table, tokens)
    for part in (slice(0, 3000), slice((1 << 26) - 2000, T)):
        assert torch.equal(out[part], table[tokens[part].long()])
    assert torch.equal(out[:, 0].float().sum(dtype=torch.float64), table[:, 0].double()[tokens.long()].sum())
    del out, tokens
    T = (1 << 26) + 5                                    # 33 vectors of 16 bytes a row would be 70 GB: one row, read by every token
    slots = torch.zeros(T, 1, dtype=torch.int32, device="cuda")
    row = torch.arange(264, dtype=torch.float32, device="cuda").bfloat16()[None]
    got = B.bsr_expert_combine(row, slots)
    for part in (slice(0, 100), slice((1 << 26) - 50, T)):
        assert torch.equal(got[part], row.expand(got[part].shape[0], -1))
    del got, slots
    torch.cuda.empty_cache()


def test_lookup_of_special_values_and_far_tokens():
    table = torch.tensor([[float("nan"), 1.0], [float("inf"), -0.0], [3.0, 4.0]]).cuda()
    tokens = torch.tensor([2, 2 ** 40, -(2 ** 40), 1, 2 ** 32 + 1, 3]).cuda()        # low words 0 and 1 must not be taken
    got = B.bsr_embedding_lookup(table, tokens)
    want = torch.tensor([[3.0, 4.0], [0, 0], [0, 0], [float("inf"), -0.0], [0, 0], [0, 0]])
    assert torch.equal(got.cpu(), want) and torch.signbit(got[3, 1])
    assert B.bsr_embedding_lookup(table, tokens[:0]).shape == (0, 2)
    assert not B.bsr_embedding_lookup(table[:0], tokens).any()


def token_mix(kind, T, V, seed):
    g = torch.Generator().manual_seed(seed)
    if kind == "uniform":
        return torch.randint(0, V, (T,), generator=g)
    if kind == "one":
        return torch.full((T,), V - 1)
    if kind == "none":
        return torch.where(torch.rand(T, generator=g) < 0.5, -1, V)
    if kind == "ascending":
        return torch.arange(T) % V
    t = torch.exp(torch.rand(T, generator=g).double() * np.log(V + 1.0)).long().clamp(1, V) - 1       # "text"
    return torch.where(torch.rand(T, generator=g) < 0.3, torch.where(torch.rand(T, generator=g) < 0.5, -1, 0), t)


@pytest.mark.parametrize("dtype,index", [("f32", "i64"), ("bf16", "i32")])
@pytest.mark.parametrize("kind", ["uniform", "one", "none", "ascending", "text"])
@pytest.mark.parametrize("T,V,D,pad,offset", [
    (1, 1, 1, 0, 0), (2, 5, 64, 0, 0), (31, 9, 3, 1, 1), (32, 7, 8, 0, 0), (33, 1000, 65, 3, 1), (64, 2, 520, 0, 0),
    (65, 1023, 130, 0, 0), (257, 1024, 72, 5, 3), (2048, 1025, 24, 0, 0), (2049, 70000, 9, 0, 0), (5000, 300, 411, 1, 0),
    (20000, 131071, 16, 0, 0)])
def test_table_grad(dtype, index, kind, T, V, D, pad, offset):
    if V * D > (1 << 21) and kind not in ("text", "one"):
        pytest.skip("large tables: two mixes only")
    tokens = token_mix(kind, T, V, T + V).to(IX[index])
    dY = randn(3, T, D, dtype=dtype)
    scale = 0.75
    want, bound = P.table_grad(tokens.numpy(), f64(dY), V, scale)
    dE = strided(torch.full((V, D), 5.0), pad, offset, fill=9.0)
    got = B.bsr_embedding_grad(tokens.cuda(), strided(dY, pad, offset), V, scale=scale, dE=dE)
    assert got is dE and around_is_untouched(dE, pad, offset, 9.0)
    check(got, want, bound)
    again = B.bsr_embedding_grad(tokens.cuda(), strided(dY, pad, offset), V, scale=scale)
    assert torch.equal(again, got)
    # added to what is there; rows of tokens that do not occur keep their bits
    old = torch.full((V, D), 5.0, device="cuda")
    old[:, 0] = float("nan")
    got = B.bsr_embedding_grad(tokens.cuda(), dY.cuda(), V, scale=scale, dE=old, accumulate=True)
    assert bool(torch.isnan(got[:, 0]).all())
    check(got[:, 1:], want[:, 1:] + 5.0, bound[:, 1:] + 2 * P.U * (5.0 + np.abs(want[:, 1:])))
    untouched = np.ones(V, bool)
    untouched[tokens.numpy()[(tokens.numpy() >= 0) & (tokens.numpy() < V)]] = False
    assert bool((got[:, 1:].cpu()[untouched] == 5.0).all())


@pytest.mark.parametrize("T,V,D", [(70000, 40000, 64), (150000, 300, 40), (140000, 1500000, 8)])
def test_table_grad_of_many_positions(T, V, D):
    """Several entries per lane of the sort, three digits, tokens with thousands of positions: against binary64 sums."""
    tokens = token_mix("text", T, V, 5)
    dY = randn(6, T, D)
    got = B.bsr_embedding_grad(tokens.cuda(), dY.cuda(), V)
    keep = (tokens >= 0) & (tokens < V)
    want = torch.zeros(V, D, dtype=torch.float64).index_add_(0, tokens[keep], dY[keep].double())
    size = torch.zeros(V, D, dtype=torch.float64).index_add_(0, tokens[keep], dY[keep].double().abs())
    n = torch.bincount(tokens[keep], minlength=V)
    check(got, want.numpy(), ((n[:, None] + 1) * P.U * size).numpy() + 1e-44)


@pytest.mark.parametrize("pad", [0, 3])
@pytest.mark.parametrize("T,V,D", [(9001, 2003, 33), (9001, 281, 600), (9001, 282, 600), (16390, 2, 520), (12000, 60000, 31)])
def test_table_grad_clears_in_parts(T, V, D, pad):
    """Sorts in several launches, which clear dE between them: nothing of what was there stays.  Windows of either rule."""
    tokens = token_mix("uniform", T, V, 8)
    dY = randn(9, T, D, dtype="bf16")
    dE = strided(torch.full((V, D), float("nan")), pad, 0, fill=9.0)
    got = B.bsr_embedding_grad(tokens.cuda(), dY.cuda(), V, dE=dE)
    assert got is dE and around_is_untouched(dE, pad, 0, 9.0)
    rows = dY.double()
    want = torch.zeros(V, D, dtype=torch.float64).index_add_(0, tokens, rows)
    size = torch.zeros(V, D, dtype=torch.float64).index_add_(0, tokens, rows.abs())
    n = torch.bincount(tokens, minlength=V)
    check(got, want.numpy(), ((n[:, None] + 1) * P.U * size).numpy() + 1e-44)


@pytest.mark.parametrize("index", ["i32", "i64"])
@pytest.mark.parametrize("T", [511, 512, 513, 2047, 8160, 8161, 8191, 8192, 8193])
def test_table_grad_at_the_sizes_of_the_sorts(index, T):
    """Around the sizes at which the sort changes: sums of equal tokens, and a permutation, which is exact."""
    V = 97
    tokens = token_mix("text", T, V, T).to(IX[index])
    dY = randn(4, T, 8)
    got = B.bsr_embedding_grad(tokens.cuda(), dY.cuda(), V)
    want, bound = P.table_grad(tokens.numpy(), f64(dY), V, 1.0)
    check(got, want, bound)
    # one position per token: a permutation, exact
    order = torch.randperm(T, generator=torch.Generator().manual_seed(T)).to(IX[index])
    got = B.bsr_embedding_grad(order.cuda(), dY.cuda(), T + 3)
    exact = torch.zeros(T + 3, 8)
    exact[order.long()] = dY
    assert torch.equal(got.cpu(), exact)


def test_table_grad_does_not_read_rows_without_a_token():
    tokens = torch.tensor([4, -1, 4, 9, 0]).cuda()
    dY = torch.ones(5, 12, device="cuda")
    dY[1], dY[3] = float("nan"), float("inf")
    dE = B.bsr_embedding_grad(tokens, dY, 9)
    assert torch.equal(dE.sum(dim=1).cpu(), torch.tensor([12.0, 0, 0, 0, 24, 0, 0, 0, 0]))
    assert not B.bsr_embedding_grad(tokens[:0], dY[:0], 9).any()
    assert B.bsr_embedding_grad(tokens, dY, 0).shape == (0, 12)


def test_table_grad_is_the_gradient_of_the_lookup():
    """Differences of <lookup(table), dY> along random directions (the lookup is linear, so the step may be large)."""
    V, D, T = 40, 48, 200
    table, dY, tokens = randn(1, V, D).cuda(), randn(2, T, D).cuda(), token_mix("text", T, V, 3).cuda()
    dE = B.bsr_embedding_grad(tokens, dY, V, scale=2.0)
    for seed in range(3):
        u = randn(10 + seed, V, D).cuda()
        up, down = (B.bsr_embedding_lookup(table + s * u, tokens, scale=2.0) for s in (1.0, -1.0))
        diff = float(((up.double() - down.double()) * dY.double()).sum() / 2)
        size = float((up.double().abs() * dY.double().abs()).sum())
        assert abs(diff - float((dE.double() * u.double()).sum())) <= 8 * P.U * size


# ---- experts ----

def routing(T, k, E, seed, drop=0.1, index="i64", skew=True):
    g = torch.Generator().manual_seed(seed)
    ids = torch.stack([torch.randperm(max(E, k), generator=g)[:k] % E for _ in range(T)]) if T and k else torch.zeros(T, k).long()
    if skew:
        ids = torch.where(torch.rand(ids.shape, generator=g) < 0.3, 0, ids)
    ids = torch.where(torch.rand(ids.shape, generator=g) < drop, torch.where(torch.rand(ids.shape, generator=g) < 0.5, -1, E), ids)
    return ids.to(IX[index])


@pytest.mark.parametrize("index", ["i32", "i64"])
@pytest.mark.parametrize("T,k,E,align,drop", [
    (1, 1, 1, 1, 0.0), (1, 2, 8, 32, 0.0), (3, 1, 5, 14, 0.5), (33, 2, 8, 16, 0.1), (64, 1, 2, 1, 0.0), (200, 4, 64, 32, 0.1),
    (1000, 2, 300, 7, 0.2), (513, 4, 1023, 64, 0.0), (1025, 2, 16, 32, 1.0), (700, 8, 1024, 3, 0.05), (3000, 6, 12, 64, 0.02),
    (0, 2, 4, 32, 0.0), (5, 0, 4, 32, 0.0)])
def test_expert_sort(index, T, k, E, align, drop):
    ids = routing(T, k, E, T + E, drop, index)
    want = P.sort_by_expert(ids.numpy(), E, align)
    outs = [torch.full(a.shape, 77, dtype=torch.int32, device="cuda") for a in want]
    got = B.bsr_expert_sort(ids.cuda(), E, align=align, offsets=outs[0], counts=outs[1], order=outs[2], slots=outs[3])
    for g, o, w in zip(got, outs, want):
        assert g is o and np.array_equal(g.cpu().numpy(), w)
    flat = B.bsr_expert_sort(ids.reshape(-1).cuda(), E, align=align)
    assert torch.equal(flat[3], got[3].reshape(-1)) and torch.equal(flat[2], got[2])


def test_expert_sort_of_many_entries():
    g = torch.Generator().manual_seed(0)
    for n, E, align in ((300000, 129, 32), (1 << 20, 8, 16)):
        ids = torch.randint(-1, E + 1, (n,), generator=g)
        ids[: n // 3] = 5                                             # a long run of one expert
        offsets, counts, order, slots = (a.cpu().long() for a in B.bsr_expert_sort(ids.cuda(), E, align=align))
        assert torch.equal(counts, torch.bincount(ids[(ids >= 0) & (ids < E)], minlength=E))
        assert torch.equal(offsets[1:] - offsets[:-1], (counts + align - 1) // align * align)
        want = torch.full_like(order, -1)
        for e in range(E):
            members = torch.nonzero(ids == e)[:, 0]
            want[offsets[e]:offsets[e] + len(members)] = members
        assert torch.equal(order, want)
        place = torch.full((n,), -1, dtype=torch.int64)
        there = torch.nonzero(want >= 0)[:, 0]
        place[want[there]] = there
        assert torch.equal(slots, place)


def test_expert_sort_takes_far_ids_for_none():
    ids = torch.tensor([2 ** 32 + 1, 1, -(2 ** 40), 0, 2 ** 33]).cuda()
    _, counts, order, slots = B.bsr_expert_sort(ids, 3)
    assert counts.tolist() == [1, 1, 0] and order.tolist() == [3, 1, -1, -1, -1] and slots.tolist() == [-1, 1, -1, 0, -1]


EXPERT_SHAPES = [(1, 1, 1, 64, 1, 0, 0), (1, 2, 4, 8, 32, 0, 0), (5, 2, 3, 1, 4, 1, 1), (33, 2, 8, 384, 16, 0, 0),
                 (40, 3, 20, 805, 32, 0, 0), (100, 4, 6, 7, 14, 3, 1), (64, 1, 16, 130, 1, 6, 3), (17, 8, 9, 96, 32, 0, 0),
                 (9, 11, 30, 200, 8, 1, 1), (300, 6, 256, 72, 2, 0, 0), (12, 17, 40, 5, 1, 0, 0), (7, 2, 4, 4100, 16, 0, 0)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,k,E,D,align,pad,offset", EXPERT_SHAPES)
def test_gather_and_combine(dtype, T, k, E, D, align, pad, offset):
    ids = routing(T, k, E, 3)
    _, _, order, slots = P.sort_by_expert(ids.numpy(), E, align)
    d_order, d_slots = torch.from_numpy(order).cuda(), torch.from_numpy(slots).cuda()
    X = randn(4, T, D, dtype=dtype)
    Xs = strided(torch.zeros(len(order), D, dtype=DT[dtype]), pad, offset, fill=7.0)
    got = B.bsr_expert_gather(strided(X, pad, offset), d_slots, d_order, out=Xs)
    assert got is Xs and around_is_untouched(Xs, pad, offset, 7.0)
    assert np.array_equal(f64(got), P.gather(f64(X), order, k))
    # back, with NaN in the rows that hold nothing
    Ys = randn(5, len(order), D, dtype=dtype)
    Ys[torch.from_numpy(order) < 0] = float("nan")
    w = torch.rand(T, k, generator=torch.Generator().manual_seed(6))
    for weights in (w, None):
        out = strided(torch.zeros(T, D, dtype=DT[dtype]), pad, offset, fill=7.0)
        got = B.bsr_expert_combine(strided(Ys, pad, offset), d_slots, None if weights is None else weights.cuda(), out=out)
        assert got is out and around_is_untouched(out, pad, offset, 7.0)
        want, bound = P.combine(f64(Ys), slots, None if weights is None else weights.numpy())
        check(got, want, bound, dtype)
        assert torch.equal(got, B.bsr_expert_combine(Ys.cuda(), d_slots, None if weights is None else weights.cuda()))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,k,E,D,align,pad,offset", EXPERT_SHAPES)
def test_combine_grad(dtype, T, k, E, D, align, pad, offset):
    ids = routing(T, k, E, 8)
    _, _, order, slots = P.sort_by_expert(ids.numpy(), E, align)
    d_order, d_slots = torch.from_numpy(order).cuda(), torch.from_numpy(slots).cuda()
    Ys, dOut = randn(9, len(order), D, dtype=dtype), randn(10, T, D, dtype=dtype)
    Ys[torch.from_numpy(order) < 0] = float("nan")
    w = torch.rand(T, k, generator=torch.Generator().manual_seed(6))
    dYs = strided(torch.full((len(order), D), 3.0, dtype=DT[dtype]), pad, offset, fill=7.0)
    dw = torch.full((T, k), 3.0, device="cuda")
    got = B.bsr_expert_combine_grad(strided(Ys, pad, offset), d_slots, d_order, w.cuda(), strided(dOut, pad, offset), dYs=dYs,
                                    dweights=dw)
    assert got[0] is dYs and got[1] is dw and around_is_untouched(dYs, pad, offset, 7.0)
    want, want_w, bound = P.combine_grad(f64(Ys), slots, order, w.double().numpy(), f64(dOut))
    check(dYs, want, P.U * np.abs(want) + 1e-44, dtype)
    check(dw, want_w, bound)
    again = B.bsr_expert_combine_grad(Ys.cuda(), d_slots, d_order, w.cuda(), dOut.cuda())
    assert torch.equal(again[0], dYs) and torch.equal(again[1], dw)


def test_gather_and_combine_against_differences():
    T, k, E, D = 50, 2, 4, 64
    _, _, order, slots = B.bsr_expert_sort(routing(T, k, E, 1).cuda(), E, align=16)
    X, w, dOut = randn(1, T, D).cuda(), torch.rand(T, k).cuda(), randn(2, T, D).cuda()
    dXs, u = randn(3, len(order), D).cuda(), randn(4, T, D).cuda()
    dX = B.bsr_expert_combine(dXs, slots)
    up, down = (B.bsr_expert_gather(X + s * u, slots, order).double() for s in (1.0, -1.0))
    size = float((up.abs() * dXs.double().abs()).sum())
    assert abs(float(((up - down) * dXs.double()).sum() / 2) - float((dX.double() * u.double()).sum())) <= 8 * P.U * size
    Ys, uy, uw = randn(5, len(order), D).cuda(), randn(6, len(order), D).cuda(), randn(7, T, k).cuda()
    dYs, dw = B.bsr_expert_combine_grad(Ys, slots, order, w, dOut)
    up, down = (B.bsr_expert_combine(Ys + s * uy, slots, w).double() for s in (1.0, -1.0))
    size = float((up.abs() * dOut.double().abs()).sum())
    assert abs(float(((up - down) * dOut.double()).sum() / 2) - float((dYs.double() * uy.double()).sum())) <= 16 * P.U * size
    up, down = (B.bsr_expert_combine(Ys, slots, w + s * uw).double() for s in (1.0, -1.0))
    size = float((up.abs() * dOut.double().abs()).sum())
    assert abs(float(((up - down) * dOut.double()).sum() / 2) - float((dw.double() * uw.double()).sum())) <= 16 * P.U * size


# ---- distillation ----

def student(N, V, K, seed, dtype="f32", tdtype="f32", index="i64", masks=True):
    g = torch.Generator().manual_seed(seed)
    z = (torch.randn(N, V, generator=g) * 2).to(DT[dtype])
    ids = torch.randint(0, max(V, 1), (N, K), generator=g)                      # some columns twice
    t = (torch.randn(N, K, generator=g) * 2 + 3).to(DT[tdtype])
    if masks and N > 2 and K > 0:
        ids = torch.where(torch.rand(N, K, generator=g) < 0.1, torch.where(torch.rand(N, K, generator=g) < 0.5, -1, V), ids)
        ids[1] = -1                                                             # a row without entries
        t[2] = float("-inf")                                                    # one whose entries weigh nothing
        t[0, K // 2] = float("-inf")
        if V > 3 and N > 4:
            z[3, V // 2:] = float("-inf")                                       # masked columns
            ids[3] = torch.where(ids[3] >= V // 2, 0, ids[3])
            z[4, 1::2] = torch.finfo(DT[dtype]).min
            ids[4] = torch.where(ids[4] % 2 == 1, 0, ids[4])
    dloss = torch.rand(N, generator=g) + 0.1
    return z, ids.to(IX[index]), t, dloss


DISTILL_SHAPES = [(1, 1, 1), (1, 2, 3), (3, 5, 2), (5, 8, 0), (6, 63, 7), (7, 64, 64), (9, 1000, 20), (40, 411, 5), (5, 8191, 50),
                  (6, 8192, 1), (5, 8193, 33), (7, 20011, 100), (300, 1031, 8), (5, 131075, 64), (2, 262144, 1024), (700, 4099, 12),
                  (5, 40000, 300)]


@pytest.mark.parametrize("dtype,tdtype,index", [("f32", "f32", "i64"), ("bf16", "bf16", "i32"), ("bf16", "f32", "i64")])
@pytest.mark.parametrize("N,V,K", DISTILL_SHAPES)
def test_distill(dtype, tdtype, index, N, V, K):
    tau = (1.0, 2.0, 0.7)[(N + V) % 3]
    z, ids, t, dloss = student(N, V, K, N + V, dtype, tdtype, index)
    tau32 = float(np.float32(tau))
    want, stats, grad, e_loss, e_grad = P.distill(f64(z), ids.numpy(), f64(t), tau32, f64(dloss))
    for pad, offset in ((0, 0), (3, 1)):
        zd = strided(z, pad, offset)
        args = (zd, ids.cuda(), t.cuda())
        loss, got_stats = B.bsr_distill_loss(*args, tau)
        check(loss, want, e_loss)
        assert np.array_equal(f64(got_stats)[:, 0], stats[:, 0])
        check(got_stats[:, 1], stats[:, 1], (V / 256 + 200) * P.U * (1 + np.abs(stats[:, 1])))
        out = strided(torch.zeros(N, V, dtype=DT[dtype]), pad, offset, fill=7.0)
        got = B.bsr_distill_grad(*args, got_stats, dloss.cuda(), tau, dlogits=out)
        assert got is out and around_is_untouched(out, pad, offset, 7.0)
        check(got, grad, e_grad, dtype)
        loss2, got2 = B.bsr_distill_loss_grad(*args, dloss.cuda(), tau)
        check(loss2, want, e_loss)
        check(got2, grad, e_grad, dtype)
        again = B.bsr_distill_loss_grad(*args, dloss.cuda(), tau)
        assert torch.equal(again[0], loss2) and torch.equal(again[1], got2)
        # in place
        fresh = strided(z, pad, offset, fill=7.0)
        got3 = B.bsr_distill_grad(fresh, ids.cuda(), t.cuda(), got_stats, dloss.cuda(), tau, dlogits=fresh)
        assert torch.equal(got3, got) and around_is_untouched(fresh, pad, offset, 7.0)
        fresh = strided(z, pad, offset, fill=7.0)
        loss4, got4 = B.bsr_distill_loss_grad(fresh, ids.cuda(), t.cuda(), dloss.cuda(), tau, dlogits=fresh)
        assert torch.equal(got4, got2) and torch.equal(loss4, loss2) and around_is_untouched(fresh, pad, offset, 7.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vecs", [1, 2, 511, 512, 513, 1024, 1025, 2048, 2049, 4096, 4097, 8192, 8193, 16384, 16385, 24576, 24577, 32767,
                                  32768, 32769])
def test_distill_at_the_edges_of_row_lengths(dtype, vecs):
    """Rows of so many 16-byte vectors and a few columns more or less, enough rows for a workgroup each, at any alignment."""
    per = 128 // torch.finfo(DT[dtype]).bits
    N, K = 130, 7
    for V, pad, offset in ((vecs * per, 0, 0), (vecs * per + per - 1, 1, 3)):
        z, ids, t, dloss = student(N, V, K, V, dtype, "f32")
        ids[7] = V - 1                                                          # the last column, by every entry
        part = torch.tensor([0, 1, 2, 3, 4, 7, 64, N - 1])
        zd = strided(z, pad, offset)
        loss, grad = B.bsr_distill_loss_grad(zd, ids.cuda(), t.cuda(), dloss.cuda(), 0.9)
        want, _, g, el, eg = P.distill(f64(z[part]), ids[part].numpy(), f64(t[part]), float(np.float32(0.9)), f64(dloss[part]))
        check(loss[part], want, el)
        check(grad[part], g, eg, dtype)
        one, stats = B.bsr_distill_loss(zd, ids.cuda(), t.cuda(), 0.9)
        other = B.bsr_distill_grad(zd, ids.cuda(), t.cuda(), stats, dloss.cuda(), 0.9)
        check(one[part], want, el)
        check(other[part], g, eg, dtype)
        # every row, against the other way round (two roundings of either)
        close = (grad.float() - other.float()).abs() <= 2.0 ** -7 * other.float().abs() + 1e-6
        assert bool(close.all())
        fresh = strided(z, pad, offset, fill=7.0)
        loss2, grad2 = B.bsr_distill_loss_grad(fresh, ids.cuda(), t.cuda(), dloss.cuda(), 0.9, dlogits=fresh)
        assert torch.equal(loss2, loss) and torch.equal(grad2, grad) and around_is_untouched(fresh, pad, offset, 7.0)


@pytest.mark.parametrize("dtype,V", [("bf16", 70001), ("f32", 32771)])
def test_distill_of_long_rows_in_a_last_round_of_few(dtype, V):
    """More long rows than compute units: whole rounds a workgroup per row, the last few rows by chunks; in place and apart."""
    N, K = 256 + 11, 6
    z, ids, t, dloss = student(N, V, K, 9, dtype, "f32", "i32")
    ids[260] = -1
    part = torch.tensor([0, 1, 2, 3, 4, 255, 256, 257, 260, N - 1])
    loss, grad = B.bsr_distill_loss_grad(z.cuda(), ids.cuda(), t.cuda(), dloss.cuda(), 1.3)
    want, _, g, el, eg = P.distill(f64(z[part]), ids[part].numpy(), f64(t[part]), float(np.float32(1.3)), f64(dloss[part]))
    check(loss[part], want, el)
    check(grad[part], g, eg, dtype)
    fresh = z.cuda()
    loss2, grad2 = B.bsr_distill_loss_grad(fresh, ids.cuda(), t.cuda(), dloss.cuda(), 1.3, dlogits=fresh)
    assert torch.equal(loss2, loss) and torch.equal(grad2, grad)


def test_distill_of_more_rows_than_a_grid_dimension():
    N, V, K = 70001, 40, 3
    z, ids, t, dloss = student(N, V, K, 1)
    loss, grad = B.bsr_distill_loss_grad(z.cuda(), ids.cuda(), t.cuda(), dloss.cuda())
    loss1, stats = B.bsr_distill_loss(z.cuda(), ids.cuda(), t.cuda())
    grad1 = B.bsr_distill_grad(z.cuda(), ids.cuda(), t.cuda(), stats, dloss.cuda())
    for part in (slice(0, 40), slice(65500, 65580), slice(69990, 70001)):
        want, st, g, el, eg = P.distill(f64(z[part]), ids[part].numpy(), f64(t[part]), 1.0, f64(dloss[part]))
        for l, d in ((loss, grad), (loss1, grad1)):
            check(l[part], want, el)
            check(d[part], g, eg)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [40, 9000, 300001])
def test_distill_rows_without_a_distribution_or_entries(dtype, V):
    """NaN, +inf and all -inf rows are NaN and do not spread; a row without entries is 0 whatever its logits; a row of the type's
    lowest value is a uniform distribution; q > 0 where p = 0 is an infinite loss and a finite gradient."""
    z, ids, t, dloss = student(8, V, 4, 3, dtype, masks=False)
    low = torch.finfo(DT[dtype]).min
    z[0, 5], z[1, 7], z[2] = float("nan"), float("inf"), float("-inf")
    z[3] = float("nan")
    ids[3] = -1
    z[4] = low
    z[5, ids[5, 0]] = float("-inf")
    ids[5, 1:] = (ids[5, 0] + 1) % V
    for tau in (1.0, 0.5):
        loss, grad = B.bsr_distill_loss_grad(z.cuda(), ids.cuda(), t.cuda(), dloss.cuda(), tau)
        loss1, stats = B.bsr_distill_loss(z.cuda(), ids.cuda(), t.cuda(), tau)
        grad1 = B.bsr_distill_grad(z.cuda(), ids.cuda(), t.cuda(), stats, dloss.cuda(), tau)
        for l, d in ((loss, grad), (loss1, grad1)):
            assert bool(torch.isnan(l[:3]).all()) and bool(torch.isnan(d[:3]).all())
            assert float(l[3]) == 0 and not d[3].any()
            assert float(l[5]) == float("inf") and bool(torch.isfinite(d[5]).all())
        zf, tf = f64(z[4:]), f64(t[4:])
        want, _, g, el, eg = P.distill(zf, ids[4:].numpy(), tf, tau, f64(dloss[4:]))
        for l, d in ((loss, grad), (loss1, grad1)):
            check(d[4:], g, eg, dtype)
            check(l[torch.tensor([4, 6, 7])], want[[0, 2, 3]], el[[0, 2, 3]])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,V", [(6, 700), (6, 20003), (5, 131075), (130, 70001)])
@pytest.mark.parametrize("scale,tau", [(1e6, 1.0), (3e37, 0.5), (5.0, 1e-4), (1.0, 2.0 ** -60), (1.0, 2.0 ** 60), (3e30, 1e-10),
                                       (2e4, 0.05), (1e-30, 1.0)])
def test_distill_of_far_logits_and_temperatures(dtype, N, V, scale, tau):
    """Exponents from far below the spacing of the logits to far above the range of the type."""
    z, ids, t, dloss = student(N, V, 5, N + V, masks=False)
    z, t = (z * scale).to(DT[dtype]), (t * scale).to(DT[dtype])
    z[0, 3] = z[0, 11] = z[0].max()                                             # two logits on top
    part = torch.tensor([0, 1, 2, 3, N - 1])
    tau32 = float(np.float32(tau))
    want, _, g, el, eg = P.distill(f64(z[part]), ids[part].numpy(), f64(t[part]), tau32, f64(dloss[part]))
    loss, grad = B.bsr_distill_loss_grad(z.cuda(), ids.cuda(), t.cuda(), dloss.cuda(), tau)
    loss1, stats = B.bsr_distill_loss(z.cuda(), ids.cuda(), t.cuda(), tau)
    grad1 = B.bsr_distill_grad(z.cuda(), ids.cuda(), t.cuda(), stats, dloss.cuda(), tau)
    for l, d in ((loss, grad), (loss1, grad1)):
        finite = np.abs(want) < 3e38                                            # (beyond that binary32 has no loss)
        check(l[part][torch.from_numpy(finite)], want[finite], el[finite])
        check(d[part], g, eg, dtype)
    fresh = z.cuda()
    loss2, grad2 = B.bsr_distill_loss_grad(fresh, ids.cuda(), t.cuda(), dloss.cuda(), tau, dlogits=fresh)
    assert torch.equal(grad2, grad)


def test_distill_gradient_against_differences():
    """The loss along a random direction: central differences of the kernel's own loss against its gradient."""
    N, V, K, tau, h = 6, 500, 9, 1.5, 2.0 ** -6
    z, ids, t, dloss = student(N, V, K, 5, masks=False)
    u = randn(6, N, V)
    args = (ids.cuda(), t.cuda())
    _, grad = B.bsr_distill_loss_grad(z.cuda(), *args, dloss.cuda(), tau)
    up, down = (B.bsr_distill_loss((z + s * h * u).cuda(), *args, tau)[0].double() for s in (1.0, -1.0))
    diff = (up - down) / (2 * h) * dloss.cuda().double()
    slope = (grad.double() * u.cuda().double()).sum(dim=1)
    # h^2 / 6 times the third derivative of log-sum-exp (at most |u|^3 max / tau) and the loss's rounding over h
    bound = (h * h / 6 * 8 * float(u.abs().max()) ** 3 / tau + 2 * 60 * P.U * tau * tau * 20 / h) * f64(dloss)
    assert bool((np.abs(f64(diff - slope)) <= bound).all())


def test_one_class_is_the_cross_entropy():
    N, V = 50, 1003
    z = randn(1, N, V)
    label = torch.randint(0, V, (N, 1), generator=torch.Generator().manual_seed(2))
    loss, _ = B.bsr_distill_loss(z.cuda(), label.cuda(), torch.zeros(N, 1).cuda())
    want = torch.nn.functional.cross_entropy(z.double(), label[:, 0], reduction="none")
    check(loss, want.numpy(), 60 * P.U * (1 + want.numpy()))


# ---- streams, graphs, devices' memory ----

def test_calls_on_a_stream_of_their_own():
    """Outputs and workspaces of a call on another stream belong to that stream: memory given back right after the call is not
    handed to the current stream while the call still runs."""
    T, V, D = 20000, 5000, 256
    tokens, dY = token_mix("text", T, V, 3).cuda(), randn(4, T, D).cuda()
    z, ids, t, dloss = (a.cuda() for a in student(64, 50000, 16, 5))
    want = B.bsr_embedding_grad(tokens, dY, V), B.bsr_distill_loss_grad(z, ids, t, dloss)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for stream in (side, side.cuda_stream):
        for _ in range(5):
            a = B.bsr_embedding_grad(tokens, dY, V, stream=stream)
            b = B.bsr_distill_loss_grad(z, ids, t, dloss, stream=stream)
            trash = [torch.full((1 << 18,), 3.0e38, device="cuda") for _ in range(8)]     # on the current stream
            assert torch.cuda.current_stream().cuda_stream != side.cuda_stream
            side.synchronize()
            assert torch.equal(a, want[0]) and torch.equal(b[0], want[1][0]) and torch.equal(b[1], want[1][1])
            del trash


def test_graph_replays():
    T, V, D, k, E = 300, 2000, 96, 2, 8
    tokens, dY, table = token_mix("text", T, V, 3).cuda(), randn(4, T, D, dtype="bf16").cuda(), randn(5, V, D, dtype="bf16").cuda()
    ids, w = routing(T, k, E, 6).cuda(), torch.rand(T, k).cuda()
    z, tid, t, dloss = (a.cuda() for a in student(30, 9000, 16, 7, dtype="bf16", tdtype="bf16"))

    def step():
        x = B.bsr_embedding_lookup(table, tokens, scale=2.0)
        offsets, counts, order, slots = B.bsr_expert_sort(ids, E, align=32)
        xs = B.bsr_expert_gather(x, slots, order)
        y = B.bsr_expert_combine(xs, slots, w)
        dys, dw = B.bsr_expert_combine_grad(xs, slots, order, w, dY)
        dx = B.bsr_expert_combine(dys, slots)
        dE = B.bsr_embedding_grad(tokens, dx, V)
        loss, stats = B.bsr_distill_loss(z, tid, t, 2.0)
        return (x, offsets, counts, order, slots, xs, y, dys, dw, dx, dE, loss, stats,
                B.bsr_distill_grad(z, tid, t, stats, dloss, 2.0), *B.bsr_distill_loss_grad(z, tid, t, dloss, 2.0))

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for replay in range(4):
        for x, seed in ((dY, 20), (table, 30)):
            x.copy_(randn(seed + replay, *x.shape, dtype="bf16"))
        tokens.copy_(token_mix("text", T, V, 40 + replay))
        ids.copy_(routing(T, k, E, 50 + replay))
        z.copy_(student(30, 9000, 16, 60 + replay, dtype="bf16")[0])
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        for g, e in zip(got, step()):
            assert torch.equal(g, e) or (bool(torch.isnan(g).any()) and torch.equal(torch.nan_to_num(g), torch.nan_to_num(e)))


def test_refusals_of_the_python_calls():
    x, ids = torch.zeros(4, 8, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    s2, order = torch.zeros(4, 2, dtype=torch.int32, device="cuda"), torch.zeros(8, dtype=torch.int32, device="cuda")
    w, st = torch.zeros(4, 2, device="cuda"), torch.zeros(4, 2, device="cuda")
    e2 = torch.zeros(4, 2, dtype=torch.int64, device="cuda")
    for call in (lambda: B.bsr_embedding_lookup(x, ids[:, None]), lambda: B.bsr_embedding_lookup(x, e2[:, 0]),
                 lambda: B.bsr_embedding_lookup(x, ids, out=torch.zeros(3, 8, device="cuda")),
                 lambda: B.bsr_embedding_lookup(x, ids, out=x.bfloat16()), lambda: B.bsr_embedding_lookup(x, ids.cpu()),
                 lambda: B.bsr_embedding_lookup(x.t(), ids), lambda: B.bsr_embedding_grad(ids[:3], x, 9),
                 lambda: B.bsr_embedding_grad(ids, x, -1), lambda: B.bsr_embedding_grad(ids, x, 9, accumulate=True),
                 lambda: B.bsr_embedding_grad(ids, x, 9, dE=torch.zeros(8, 8, device="cuda")),
                 lambda: B.bsr_expert_sort(e2, 4, slots=order), lambda: B.bsr_expert_sort(e2, 4, counts=order),
                 lambda: B.bsr_expert_gather(x, s2[:3], order), lambda: B.bsr_expert_gather(x, s2.long(), order),
                 lambda: B.bsr_expert_gather(x, s2, order.long()), lambda: B.bsr_expert_combine(x, s2, w[:, :1]),
                 lambda: B.bsr_expert_combine(x, s2, w.double()), lambda: B.bsr_expert_combine_grad(x, s2, order, w, x),
                 lambda: B.bsr_expert_combine_grad(x, s2, order[:4], w, x.bfloat16()),
                 lambda: B.bsr_distill_loss(x, ids, w), lambda: B.bsr_distill_loss(x, e2, w[:3]),
                 lambda: B.bsr_distill_grad(x, e2, w, st[:3], ids.float()), lambda: B.bsr_distill_grad(x, e2, w, st, ids),
                 lambda: B.bsr_distill_loss_grad(x, e2, w, ids.float()[:3]),
                 lambda: B.bsr_distill_loss_grad(x, e2, w, ids.float(), dlogits=x.bfloat16())):
        with pytest.raises(ValueError):
            call()
    for call, code in ((lambda: B.bsr_embedding_lookup(x.half(), ids), B.BSR_ERR_DTYPE),
                       (lambda: B.bsr_embedding_lookup(x, ids.short()), B.BSR_ERR_DTYPE),
                       (lambda: B.bsr_embedding_lookup(x, ids, scale=float("nan")), B.BSR_ERR_VALUE),
                       (lambda: B.bsr_expert_sort(e2.float(), 4), B.BSR_ERR_DTYPE),
                       (lambda: B.bsr_expert_sort(e2, 0), B.BSR_ERR_SHAPE), (lambda: B.bsr_expert_sort(e2, 2000), B.BSR_ERR_LIMIT),
                       (lambda: B.bsr_distill_loss(x, e2, w, 0.0), B.BSR_ERR_VALUE),
                       (lambda: B.bsr_distill_loss(x, e2, w.half()), B.BSR_ERR_DTYPE),
                       (lambda: B.bsr_distill_loss(x, e2, w, ws=torch.zeros(4, dtype=torch.uint8, device="cuda")),
                        B.BSR_ERR_WORKSPACE)):
        with pytest.raises(B.BsrError) as e:
            call()
        assert e.value.code == code
