"""Token operators of nothing: no rows, no columns, no entries, in every dimension that may be empty."""
import pytest
import torch

from paper_2311_16883_amd import binding as B
from test_gpu_token_step import example

pytestmark = pytest.mark.gpu

NAN = float("nan")


def new(*size, dtype=torch.float32):
    return torch.full(size, NAN if dtype.is_floating_point else 77, dtype=dtype, device="cuda")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_table_of_nothing(dtype):
    tokens = torch.tensor([0, 3, -1], device="cuda")
    for T, V, D in ((0, 5, 8), (3, 0, 8), (3, 5, 0), (0, 0, 0)):
        table, rows = new(V, D, dtype=dtype), new(T, D, dtype=dtype)
        out = B.bsr_embedding_lookup(table, tokens[:T])
        assert out.shape == (T, D) and (V > 0 or not out.any())
        dE = new(V, D)
        assert B.bsr_embedding_grad(tokens[:T], rows, V, dE=dE) is dE and (T > 0 or not dE.any())
        old = torch.ones(V, D, device="cuda")
        B.bsr_embedding_grad(tokens[:T], rows, V, dE=old, accumulate=True)
        assert T > 0 or bool((old == 1).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,k,D", [(0, 2, 8), (4, 0, 8), (4, 2, 0), (0, 0, 0)])
def test_experts_of_nothing(dtype, T, k, D):
    ids = torch.zeros(T, k, dtype=torch.int64, device="cuda")
    offsets, counts, order, slots = B.bsr_expert_sort(ids, 3, align=4)
    n = T * k
    assert counts.tolist() == [n, 0, 0] and offsets.tolist() == [0] + 3 * [-(-n // 4) * 4] and order.numel() == B.bsr_expert_capacity(n, 3, 4)
    X = torch.ones(T, D, dtype=dtype, device="cuda")
    xs = B.bsr_expert_gather(X, slots, order)
    assert xs.shape == (order.numel(), D) and int((xs != 0).sum()) == n * D
    w = torch.ones(T, k, device="cuda")
    out = B.bsr_expert_combine(xs, slots, w, out=new(T, D, dtype=dtype))
    assert bool((out == k).all())
    dYs, dw = B.bsr_expert_combine_grad(xs, slots, order, w, X, dYs=new(order.numel(), D, dtype=dtype), dweights=new(T, k))
    assert int((dYs != 0).sum()) == n * D and not torch.isnan(dYs).any() and bool((dw == D).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows", [0, 5])
def test_padding_alone(dtype, rows):
    """Rows of the sorted matrix without a token to fill them."""
    order = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    slots = torch.full((3, 2), -1, dtype=torch.int32, device="cuda")
    Ys, X, w = new(rows, 8, dtype=dtype), new(3, 8, dtype=dtype), new(3, 2)
    for s, x, ww in ((slots, X, w), (slots[:0], X[:0], w[:0])):
        xs = B.bsr_expert_gather(x, s, order, out=new(rows, 8, dtype=dtype))
        assert not xs.any()
        assert not B.bsr_expert_combine(Ys, s, ww, out=new(len(s), 8, dtype=dtype)).any()
        dYs, dw = B.bsr_expert_combine_grad(Ys, s, order, ww, x, dYs=new(rows, 8, dtype=dtype), dweights=new(len(s), 2))
        assert not dYs.any() and not dw.any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,V,K", [(0, 9, 3), (4, 0, 3), (4, 9, 0), (4, 0, 0), (0, 0, 0)])
def test_logits_of_nothing(dtype, N, V, K):
    z, dloss = torch.ones(N, V, dtype=dtype, device="cuda"), torch.ones(N, device="cuda")
    ids, t = torch.zeros(N, K, dtype=torch.int64, device="cuda"), torch.ones(N, K, device="cuda")
    loss, stats = B.bsr_distill_loss(z, ids, t, loss=new(N), stats=new(N, 2))
    loss2, grad = B.bsr_distill_loss_grad(z, ids, t, dloss, loss=new(N), dlogits=new(N, V, dtype=dtype))
    assert not loss.any() and not loss2.any() and not grad.any() and grad.shape == (N, V)       # rows without an entry
    if V == 0:
        assert bool((stats[:, 0] == -float("inf")).all()) and bool(torch.isnan(stats[:, 1]).all())
    else:
        assert bool((stats[:, 0] == 1).all()) and bool(((stats[:, 1] - 2.1972246).abs() < 1e-6).all())
    assert not B.bsr_distill_grad(z, ids, t, stats, dloss, dlogits=new(N, V, dtype=dtype)).any()


@pytest.mark.parametrize("there", [0, 1])
def test_training_step_of_hardly_any_token(there):
    """The example's step where all positions are padding, or all but one: no expert, or two, have rows."""
    ex = example()
    model, batch = ex.make_model(300, 64, 4, torch.float32, seed=1), ex.make_batch(40, 300, 8, seed=2)
    for name, none in (("tokens", -1), ("teacher_ids", -1), ("dloss", 0)):
        batch[name][there:] = none
    batch["tokens"][:there] = 7
    batch["dloss"][:there] = 1.0
    batch["teacher_ids"][:there] = torch.arange(8, device="cuda")
    loss, grads = ex.step(model, batch, keep=0.5)
    assert bool(torch.isfinite(loss)) and (float(loss) > 0) == (there > 0)
    for n in ("table", "router", "out"):
        assert bool(torch.isfinite(grads[n]).all()) and bool(grads[n].any()) == (there > 0)
    assert sum(bool(g.any()) for g in grads["experts"]) == 2 * there
    rows = torch.nonzero(grads["table"].abs().sum(dim=1))[:, 0].tolist()
    assert rows == [7] * there
