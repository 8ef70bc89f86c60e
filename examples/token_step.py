"""One training step of a small token model whose experts save pruned inputs.

    python examples/token_step.py [--tokens 2048] [--vocab 8192] [--dim 256] [--experts 8] [--keep 0.5] [--dtype bf16] [--steps 5]

The model: token table -> router (k experts of all) -> one linear layer per expert -> weighted return -> logits, learning from the
largest logits of a teacher.  What is a plain matrix product is torch's; the rest are calls of this library:

  forward   bsr_embedding_lookup            x = scale * table[tokens]
            bsr_expert_sort, _gather        tokens to the experts, every expert's rows from a whole block-row on
            bsr_score_select_batched,       the experts' inputs, pruned and kept as BSR for the way back
            bsr_compress_batched            (the dense copy could be freed here)
            bsr_expert_combine              the experts' outputs, weighted, back to their tokens
  backward  bsr_distill_loss_grad           loss and the gradient of the logits, in their place
            bsr_expert_combine_grad         gradients of the experts' outputs and of the router's weights
            bsr_t_dense_matmul_batched      the experts' weight gradients from the BSR tensors
            bsr_expert_combine              gradient of the gather
            bsr_embedding_grad              gradient of the token table

One small copy to the host per step: the experts' segments, which size their products.
"""
import argparse
import sys
from pathlib import Path

import torch

sys.path.insert(0, str(Path(__file__).resolve().parent.parent))

from paper_2311_16883_amd import binding as B  # noqa: E402

BLOCK = 32


def make_model(vocab, dim, experts, dtype, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*size, std):
        return (torch.randn(*size, generator=g, device="cuda") * std).to(dtype)
    return dict(table=normal(vocab, dim, std=0.05), router=normal(dim, experts, std=dim ** -0.5),
                experts=normal(experts, dim, dim, std=dim ** -0.5), out=normal(dim, vocab, std=dim ** -0.5))


def make_batch(tokens, vocab, entries, seed=0):
    """Tokens as frequent as in text, some positions padding (-1, no teacher entries), and a teacher's largest logits."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    ids = (torch.exp(torch.rand(tokens, generator=g, device="cuda") * torch.log(torch.tensor(vocab + 1.0))).long() - 1).clamp_(0, vocab - 1)
    pad = torch.rand(tokens, generator=g, device="cuda") < 0.05
    first = torch.randint(0, vocab, (tokens, 1), generator=g, device="cuda")
    teacher_ids = (first + 7 * torch.arange(entries, device="cuda")) % vocab
    teacher = torch.sort(torch.randn(tokens, entries, generator=g, device="cuda") * 2, dim=1, descending=True).values
    minus_one = torch.full_like(ids, -1)
    return dict(tokens=torch.where(pad, minus_one, ids), teacher_ids=torch.where(pad[:, None], minus_one[:, None], teacher_ids),
                teacher=teacher, dloss=torch.where(pad, 0.0, 1.0 / tokens))


def step(model, batch, k=2, keep=0.5, scale=4.0, temperature=2.0):
    """-> loss (mean over the batch), gradients of the model's tensors (float32; the experts' as a list)."""
    table, router, weights, out = model["table"], model["router"], model["experts"], model["out"]
    vocab, dim = table.shape
    experts = router.shape[1]
    # forward
    x = B.bsr_embedding_lookup(table, batch["tokens"], scale=scale)
    top, choice = torch.topk((x @ router).float(), k, dim=1)
    # padding takes no expert's time
    choice = torch.where((batch["tokens"] < 0)[:, None], -1, choice)
    w = torch.softmax(top, dim=1)
    offsets, counts, order, slots = B.bsr_expert_sort(choice, experts, align=BLOCK)
    xs = B.bsr_expert_gather(x, slots, order)
    ends = offsets.tolist()
    part = [(e, slice(a, b)) for e, (a, b) in enumerate(zip(ends, ends[1:])) if b > a]
    ys = torch.zeros_like(xs)
    for e, rows in part:
        torch.matmul(xs[rows], weights[e], out=ys[rows])
    saved = []
    if part:                                            # (a batch of padding alone has no expert's rows)
        masks = B.bsr_score_select_batched(B.SelectBatch([xs[r] for _, r in part], [(BLOCK, BLOCK)] * len(part), [keep] * len(part)))
        kept = [B.bsr_keep_count(m.numel(), keep) for m in masks]
        saved = B.bsr_compress_batched(B.CompressBatch([(xs[r], BLOCK, BLOCK, m, n) for (_, r), m, n in zip(part, masks, kept)]))
    y = B.bsr_expert_combine(ys, slots, w)
    logits = y @ out
    # backward: the gradient takes the logits' place
    loss, dlogits = B.bsr_distill_loss_grad(logits, batch["teacher_ids"], batch["teacher"], batch["dloss"], temperature,
                                            dlogits=logits)
    d_out = y.t() @ dlogits
    dy = dlogits @ out.t()
    dys, dw = B.bsr_expert_combine_grad(ys, slots, order, w, dy)
    grads = B.bsr_t_dense_matmul_batched(B.MatmulBatch(
        [(*bsr, r.stop - r.start, dim, BLOCK, BLOCK, dys[r]) for (_, r), bsr in zip(part, saved)])) if part else []
    d_experts = [torch.zeros(dim, dim, device="cuda") for _ in range(experts)]
    dxs = torch.zeros_like(xs)
    for (e, rows), g in zip(part, grads):
        d_experts[e] = g
        torch.matmul(dys[rows], weights[e].t(), out=dxs[rows])
    dx = B.bsr_expert_combine(dxs, slots)
    # the router: through the softmax over its k choices
    d_top = w * (dw - (w * dw).sum(dim=1, keepdim=True))
    d_scores = torch.zeros(x.shape[0], experts, device="cuda").scatter_(1, choice.clamp_min(0), d_top).to(x.dtype)
    d_router = x.t() @ d_scores
    dx = dx + d_scores @ router.t()
    d_table = B.bsr_embedding_grad(batch["tokens"], dx, vocab, scale=scale)
    return (loss * batch["dloss"]).sum(), dict(table=d_table, router=d_router.float(), experts=d_experts, out=d_out.float())


def main():
    p = argparse.ArgumentParser()
    p.add_argument("--tokens", type=int, default=2048)
    p.add_argument("--vocab", type=int, default=8192)
    p.add_argument("--dim", type=int, default=256)
    p.add_argument("--experts", type=int, default=8)
    p.add_argument("--choices", type=int, default=2)
    p.add_argument("--entries", type=int, default=16)
    p.add_argument("--keep", type=float, default=0.5)
    p.add_argument("--dtype", choices=("f32", "bf16"), default="bf16")
    p.add_argument("--steps", type=int, default=5)
    p.add_argument("--rate", type=float, default=2.0)
    a = p.parse_args()
    dtype = torch.bfloat16 if a.dtype == "bf16" else torch.float32
    model = make_model(a.vocab, a.dim, a.experts, torch.float32)
    batch = make_batch(a.tokens, a.vocab, a.entries)
    for i in range(a.steps):
        cast = {n: t.to(dtype) for n, t in model.items()}
        loss, grads = step(cast, batch, k=a.choices, keep=a.keep)
        for n in ("table", "router", "out"):
            model[n] -= a.rate * grads[n]
        model["experts"] -= a.rate * torch.stack(grads["experts"])
        print(f"step {i}: loss {float(loss):.4f}", flush=True)


if __name__ == "__main__":
    main()
