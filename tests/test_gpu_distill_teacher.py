"""Distillation where the teacher's logits, or the student's at the teacher's entries, are no ordinary numbers: NaN and +inf must reach
the loss and the gradient at the entries, in every form of the kernels."""
import numpy as np
import pytest
import torch

import token_plain as P
from paper_2311_16883_amd import binding as B
from test_gpu_token_ops import DT, check, f64, randn

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


def three_calls(z, ids, t, dloss, tau):
    """Loss and gradient of both in one call, of one after the other, and of the latter in place of the logits."""
    args = z.cuda(), ids.cuda(), t.cuda()
    yield B.bsr_distill_loss_grad(*args, dloss.cuda(), tau)
    loss, stats = B.bsr_distill_loss(*args, tau)
    yield loss, B.bsr_distill_grad(*args, stats, dloss.cuda(), tau)
    fresh = z.cuda()
    yield loss, B.bsr_distill_grad(fresh, ids.cuda(), t.cuda(), stats, dloss.cuda(), tau, dlogits=fresh)
    fresh = z.cuda()
    yield B.bsr_distill_loss_grad(fresh, ids.cuda(), t.cuda(), dloss.cuda(), tau, dlogits=fresh)


# rows in one wave, in workgroups of every size, by chunks in two passes, and (130 rows) in workgroups that a compute unit has one of
SHAPES = [("f32", 10, 40), ("bf16", 10, 40), ("bf16", 10, 5000), ("f32", 10, 9000), ("bf16", 10, 60000), ("f32", 10, 300001),
          ("bf16", 130, 70001), ("f32", 130, 131000)]


@pytest.mark.parametrize("dtype,N,V", SHAPES)
@pytest.mark.parametrize("K", [1, 6, 100])
def test_a_teachers_nan_and_infinity_reach_the_loss_and_the_gradient(dtype, N, V, K):
    g = torch.Generator().manual_seed(V + K)
    z = (torch.randn(N, V, generator=g) * 2).to(DT[dtype])
    ids = torch.randint(0, V, (N, K), generator=g)
    t = torch.randn(N, K, generator=g) * 2
    dloss = torch.rand(N, generator=g) + 0.1
    last = K - 1
    t[0] = NAN                                          # nothing but NaN
    t[1], t[1, last] = -INF, NAN                        # NaN beside entries that weigh nothing
    t[2, last] = NAN                                    # NaN beside finite ones
    t[3, last] = INF
    t[4] = INF
    t[5], ids[5, :last] = NAN, -1                       # NaN at the only entry
    bad = [0, 1, 2, 3, 4, 5]
    t[6], ids[6] = NAN, -1                              # NaN where there is no entry: a row without entries
    t[7], t[7, last] = -INF, -INF
    if K > 1:
        t[8, 0], ids[8, 0] = NAN, V                     # ... and one beside entries
    tau = 1.5
    clean = torch.where(torch.isfinite(t), t, 0.0)      # elsewhere than at the entries the teacher's logits have no part in the gradient
    rows = list(range(10))
    _, _, grad, _, e_grad = P.distill(f64(z[rows]), ids[rows].numpy(), f64(clean[rows]), tau, f64(dloss[rows]))
    want, _, whole, e_loss, e_whole = P.distill(f64(z[8:10]), ids[8:10].numpy(), f64(t[8:10]), tau, f64(dloss[8:10]))
    at_entry = np.zeros((10, V), bool)
    for n in range(10):
        at_entry[n, [v for v in ids[n].tolist() if 0 <= v < V]] = True
    for loss, got in three_calls(z, ids, t, dloss, tau):
        loss, got = loss[:10], got[:10]
        nan = torch.isnan(got).cpu().numpy()
        for n in bad:
            assert bool(torch.isnan(loss[n])), n
            assert np.array_equal(nan[n], at_entry[n]), n
            other = ~at_entry[n]
            check(got[n].cpu()[torch.from_numpy(other)], grad[n][other], e_grad[n][other], dtype)
        for n in (6, 7):
            assert float(loss[n]) == 0 and not got[n].any()
        check(loss[8:10], want, e_loss)
        check(got[8:10], whole, e_whole, dtype)


@pytest.mark.parametrize("dtype,N,V", SHAPES)
def test_an_entry_at_a_masked_column_costs_infinitely_much_whatever_its_share(dtype, N, V):
    """Down to shares and temperatures whose product is less than any binary32 number."""
    z, dloss = randn(1, N, V, dtype=dtype), torch.ones(N)
    ids = torch.arange(3)[None].repeat(N, 1)
    z[:, 2] = -INF
    for tau, t in ((2.0 ** -60, [0.0, -1.0 * 2.0 ** -61, -70.0 * 2.0 ** -60]), (2.0 ** -40, [0.0, 0.0, -80.0 * 2.0 ** -40]),
                   (1.0, [3.0, 2.0, -50.0])):
        teacher = torch.tensor(t)[None].repeat(N, 1)
        for loss, grad in three_calls(z, ids, teacher, dloss, tau):
            assert bool((loss == INF).all()) and bool(torch.isfinite(grad).all())


@pytest.mark.parametrize("dtype,N,V", SHAPES)
def test_an_entry_at_a_column_of_the_types_lowest_value_costs_what_the_formula_says(dtype, N, V):
    """tau * q * (m - z) is a binary32 number where tau * q is small enough, and +inf elsewhere."""
    z, dloss = randn(2, N, V, dtype=dtype), torch.ones(N)
    ids = torch.arange(2)[None].repeat(N, 1)
    z[:, 1] = torch.finfo(DT[dtype]).min
    t = torch.tensor([[0.0, 0.0]]).repeat(N, 1)
    part = list(range(10))
    for tau in (1.0, 0.25, 8.0):
        want, _, grad, e_loss, e_grad = P.distill(f64(z[part]), ids[part].numpy(), f64(t[part]), tau, f64(dloss[part]))
        for loss, got in three_calls(z, ids, t, dloss, tau):
            if tau * 0.5 > 1:
                assert bool((loss == INF).all())
            else:
                check(loss[part], want, e_loss)
            check(got[part], grad, e_grad, dtype)
