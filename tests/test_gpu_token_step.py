"""The example training step against torch's automatic differentiation of the same model in binary64 (nothing pruned), and with
pruned inputs against the masked product."""
import importlib.util
from pathlib import Path

import pytest
import torch

pytestmark = pytest.mark.gpu


def example():
    path = Path(__file__).resolve().parent.parent / "examples" / "token_step.py"
    spec = importlib.util.spec_from_file_location("token_step_example", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def reference(model, batch, k, scale, temperature):
    """The step in binary64 on the CPU, by automatic differentiation, the experts as one dense product each."""
    m = {n: t.double().cpu().requires_grad_() for n, t in model.items()}
    tokens, ids = batch["tokens"].cpu(), batch["teacher_ids"].cpu()
    there = tokens >= 0
    x = torch.where(there[:, None], scale * m["table"][tokens.clamp_min(0)], 0.0)
    top, choice = torch.topk(x @ m["router"], k, dim=1)
    w = torch.softmax(top, dim=1)
    every = torch.einsum("td,edf->tef", x, m["experts"])
    y = (w[:, :, None] * every[torch.arange(len(tokens))[:, None], choice]).sum(dim=1) * there[:, None]
    logp = torch.log_softmax(y @ m["out"] / temperature, dim=1)
    q = torch.softmax(batch["teacher"].double().cpu() / temperature, dim=1)
    row = temperature ** 2 * (q * (torch.log(q) - logp.gather(1, ids.clamp_min(0)))).sum(dim=1)
    loss = (row * there * batch["dloss"].double().cpu()).sum()
    loss.backward()
    return float(loss.detach()), {n: t.grad for n, t in m.items()}, x, choice


def test_step_against_automatic_differentiation():
    ex = example()
    model = ex.make_model(500, 64, 5, torch.float32, seed=3)
    batch = ex.make_batch(300, 500, 8, seed=4)
    loss, grads = ex.step(model, batch, k=2, keep=1.0, scale=4.0, temperature=1.5)
    want, ref, _, _ = reference(model, batch, 2, 4.0, 1.5)
    assert abs(float(loss) - want) <= 1e-5 * abs(want)
    # sums of up to a few hundred binary32 products of either sign, chained four deep: a few hundred roundings of the largest value
    for n in ("table", "router", "out"):
        got, g = grads[n].double().cpu(), ref[n]
        assert float((got - g).abs().max()) <= 500 * 2.0 ** -24 * float(g.abs().max()), n
    got = torch.stack(grads["experts"]).double().cpu()
    assert float((got - ref["experts"]).abs().max()) <= 500 * 2.0 ** -24 * float(ref["experts"].abs().max())


def test_step_with_pruned_inputs_prunes_the_experts_gradients_alone():
    ex = example()
    model = ex.make_model(400, 64, 4, torch.bfloat16, seed=5)
    batch = ex.make_batch(400, 400, 8, seed=6)
    full_loss, full = ex.step(model, batch, keep=1.0)
    loss, grads = ex.step(model, batch, keep=0.5)
    assert float(loss) == float(full_loss)                      # the forward pass is dense
    for n in ("table", "router", "out"):
        assert torch.equal(grads[n], full[n])
    for g, f in zip(grads["experts"], full["experts"]):
        assert not torch.equal(g, f) and 0.2 < float(g.norm() / f.norm()) < 1.0
