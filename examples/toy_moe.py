"""Trains a toy MoE language model with the library's operators around its optimizer step.

One embedding (tied to the output head), one MoE layer and its router, on synthetic text in which a token
mostly settles the next one. A step is: lookup -> router -> experts -> head and loss; the logits' gradient of
the router and the embedding's gradient, added to the one that the head left; the global norm's clip
factor; the optimizer step on all tiers, which takes the factor on the device. What lies between
(the experts' products, the loss) is plain PyTorch. Run: python examples/toy_moe.py [steps]
"""
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_19058_gb300 import skewadam as S  # noqa: E402

VOCAB, WIDTH, EXPERTS, FFN, TOP_K = 512, 64, 8, 128, 2
BATCH, CONTEXT = 8, 128
LR, DECAY, MAX_NORM, SEED = 3e-3, 0.05, 0.3, 7  # (a norm that early steps exceed)
BIAS_RATE = 1e-3  # the balance bias moves by this much a step, towards even loads


class Route(torch.autograd.Function):
    """The router's weights as a differentiable function of its logits."""

    @staticmethod
    def forward(ctx, logits, router, bias):
        chosen, weights, counts = router.route(logits, bias=bias)
        ctx.router = router
        ctx.save_for_backward(logits, chosen)
        ctx.mark_non_differentiable(chosen, counts)
        return weights, chosen, counts

    @staticmethod
    def backward(ctx, dweights, _chosen, _counts):
        logits, chosen = ctx.saved_tensors
        return ctx.router.grad(logits, chosen, dweights.contiguous()), None, None


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
        self.embedding = S.Embedding(VOCAB, WIDTH, act_dtype=torch.float32, scale=WIDTH ** 0.5)
        self.router = S.Router(EXPERTS, TOP_K, score="sigmoid")
        self.bias = torch.zeros(EXPERTS, device=device)

    def loss(self, h, table, gate, up, down, targets):
        weights, chosen, counts = Route.apply(h @ gate, self.router, self.bias)
        # every expert on every token, then the chosen ones': fine for a toy
        y = torch.relu(torch.einsum("td,edf->tef", h, up.float()))
        y = torch.einsum("tef,efd->ted", y, down.float())
        y = torch.gather(y, 1, chosen.long()[:, :, None].expand(-1, -1, WIDTH))
        out = h + (y * weights[:, :, None]).sum(1)
        return F.cross_entropy(out @ table.float().t(), targets), counts

    def step(self, t, ids, targets):
        """One training step; the loss and the experts' loads, on the device."""
        h = self.embedding.lookup(self.table, ids).requires_grad_()
        leaves = [p.detach().requires_grad_() for p in self.params]
        loss, counts = self.loss(h, *leaves, targets)
        dh, *grads = torch.autograd.grad(loss, [h, *leaves])
        for g, new in zip(self.grads, grads):
            g.copy_(new)
        self.embedding.grad(ids, dh, base=self.grads[0], out=self.grads[0])  # the head's, plus the lookup's
        self.clip.norm(MAX_NORM)
        self.opt.step(t, LR, SEED, grad_scale=self.clip.gamma)
        self.bias += BIAS_RATE * torch.sign(counts.float().mean() - counts)
        return loss.detach(), counts


def batch(gen, device="cuda"):
    """Tokens with frequencies of about 1 / rank, and their successors: one in eight at random, the others settled."""
    u = torch.rand(BATCH * CONTEXT, generator=gen, device=device)
    ids = (torch.exp(u * torch.log(torch.tensor(VOCAB + 1.0))) - 1).long().clamp_(0, VOCAB - 1)
    targets = (ids * 37 + 11) % VOCAB
    noise = torch.rand(ids.shape, generator=gen, device=device) < 0.125
    return ids, torch.where(noise, torch.randint(0, VOCAB, ids.shape, generator=gen, device=device), targets)


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
    return torch.stack(losses).tolist()


if __name__ == "__main__":
    train(int(sys.argv[1]) if len(sys.argv) > 1 else 200, print)
