"""Trains a toy MoE language model whose experts see their own tokens only, with every operator of the library.

One embedding (tied to the output head), one MoE layer with two matrices an expert, and its router. A step is: lookup -> route -> rows by expert -> up
product -> ReLU -> down product -> combined, on top of the embedding -> the head's loss, without its logits; then the same calls' gradients in reverse, the
global norm's clip factor, and the optimizer step on all tiers. Activations are bf16, the router and its logits fp32; PyTorch is left with the router's own small
products, the ReLU and additions. Run: python examples/sparse_moe.py [steps]
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_19058_gb300 import skewadam as S  # noqa: E402

VOCAB, WIDTH, EXPERTS, FFN, TOP_K = 512, 64, 8, 128, 2
BATCH, CONTEXT = 8, 128
LR, DECAY, MAX_NORM, SEED = 3e-3, 0.05, 0.3, 7


class Model:
    def __init__(self, device="cuda", seed=0):
        gen = torch.Generator(device=device).manual_seed(seed)
        make = lambda shape, dtype=torch.bfloat16: torch.randn(shape, generator=gen, device=device).mul_(0.05).to(dtype)  # noqa: E731
        self.table = make((VOCAB, WIDTH))
        self.gate = make((WIDTH, EXPERTS), torch.float32)
        self.up, self.down = make((EXPERTS, WIDTH, FFN)), make((EXPERTS, FFN, WIDTH))
        self.params = [self.table, self.gate, self.up, self.down]
        self.grads = [torch.zeros_like(p) for p in self.params]
        tiers = [S.TIER_BACKBONE, S.TIER_ROUTER, S.TIER_EXPERT, S.TIER_EXPERT]
        self.opt = S.SkewAdam(list(zip(self.params, self.grads, tiers)), S.hparams(weight_decay=DECAY))
        self.clip = S.GradClip(self.grads)
        self.embedding = S.Embedding(VOCAB, WIDTH, scale=WIDTH ** 0.5)
        self.router = S.Router(EXPERTS, TOP_K, score="sigmoid")
        self.dispatch = S.Dispatch(EXPERTS, TOP_K)
        self.ups, self.downs = S.Experts(EXPERTS, WIDTH, FFN), S.Experts(EXPERTS, FFN, WIDTH)
        self.head = S.HeadLoss(VOCAB, WIDTH)

    def gradients(self, ids, targets):
        """The mean loss over the targets that are there, and every gradient, left in ``grads``."""
        h = self.embedding.lookup(self.table, ids)
        logits = h.float() @ self.gate
        chosen, weights, counts = self.router.route(logits)
        order = self.dispatch.order(chosen)
        offsets = order[0]
        rows = self.dispatch.spread(h, order)
        a = self.ups.product(rows, self.up, offsets)
        r = torch.relu(a)
        y = self.downs.product(r, self.down, offsets)
        out = h + self.dispatch.combine(y, weights, order)
        loss, lse = self.head.loss(out, self.table, targets)

        there = (targets >= 0).float()
        dloss = there / there.sum().clamp(min=1)
        dtable, dgate, dup, ddown = self.grads
        dh, _ = self.head.grad(out, self.table, targets, lse, dloss, out=dtable)
        dy, dweights = self.dispatch.combine_grad(dh, y, weights, order)
        self.downs.grad(r, dy, offsets, out=ddown)
        da = torch.where(a > 0, self.downs.grad_rows(dy, self.down, offsets), 0)
        self.ups.grad(rows, da, offsets, out=dup)
        dlogits = self.router.grad(logits, chosen, dweights)
        torch.mm(h.float().t(), dlogits, out=dgate)
        dh = dh.float() + self.dispatch.combine(self.ups.grad_rows(da, self.up, offsets), None, order).float() + dlogits @ self.gate.t()
        self.embedding.grad(ids, dh.bfloat16(), base=dtable, out=dtable)  # the head's, plus the lookup's
        return (loss * dloss).sum(), counts

    def step(self, t, ids, targets):
        loss, counts = self.gradients(ids, targets)
        self.clip.norm(MAX_NORM)
        self.opt.step(t, LR, SEED, grad_scale=self.clip.gamma)
        return loss, counts


def batch(gen, device="cuda"):
    """Tokens with frequencies of about 1 / rank, and their successors: one in eight at random, the others settled; the last of each sequence has none."""
    u = torch.rand(BATCH * CONTEXT, generator=gen, device=device)
    ids = (torch.exp(u * torch.log(torch.tensor(VOCAB + 1.0))) - 1).long().clamp_(0, VOCAB - 1)
    targets = (ids * 37 + 11) % VOCAB
    noise = torch.rand(ids.shape, generator=gen, device=device) < 0.125
    targets = torch.where(noise, torch.randint(0, VOCAB, ids.shape, generator=gen, device=device), targets)
    targets[CONTEXT - 1::CONTEXT] = -1
    return ids, targets


def train(steps, log=None):
    model = Model()
    gen = torch.Generator(device="cuda").manual_seed(1)
    losses = []
    for t in range(1, steps + 1):
        loss, counts = model.step(t, *batch(gen))
        losses.append(loss)
        if log and (t == 1 or t % 20 == 0):
            norm, gamma = model.clip.result.tolist()
            log(f"step {t:4d}  loss {float(loss):.4f}  gradient norm {norm:.3f}  clip factor {gamma:.3f}  tokens per expert {counts.tolist()}")
    model.opt.sync_status()
    S.skew_ops_sync_status(torch.cuda.current_stream().cuda_stream)
    return torch.stack(losses).tolist()


if __name__ == "__main__":
    train(int(sys.argv[1]) if len(sys.argv) > 1 else 200, print)
