"""A small language model with attention, trained with the optimizer step for its matrices and AdamW for all else, on one GPU.

    python examples/train_attention_lm.py [--steps 120] [--state e4m3]

Embedding lookup, then attention and a feed-forward, each behind the norm before it and followed by its own norm and gate on the way back to the
residual stream (fira_block_norm does all of that between two blocks at once), output head.  Queries and keys lie in one buffer with the values and
are turned by their positions there.  The products, the softmax and the loss are torch's, with autograd; the rest runs in libfira.so:

  forward   fira_embed_lookup, fira_layer_norm, fira_rotary, fira_block_norm
  backward  the gradient of each; those of vectors and of the table are added up in fp32 over the micro-batches
  clipping  GradientList: the norm of all gradients together, and the accumulated fp32 gradients scaled into the ones that the optimizers take
  step      fira_step for the blocks' matrices (low-rank); AdamWList.fira_adamw_step for table, head, norms and gates, their states in fp32 or in 8 bits

The data is that of train_small_lm.py: every token has one successor."""
import argparse
import math
import os
import sys

import torch

sys.path[:0] = [os.path.dirname(os.path.dirname(os.path.abspath(__file__))), os.path.dirname(os.path.abspath(__file__))]
from paper_2410_01623_amd import fira, training  # noqa: E402
from train_small_lm import BF16, DEV, F32, Lookup, Norm, added_to, batches  # noqa: E402


class Turn(torch.autograd.Function):
    """Queries and keys turned by their positions."""

    @staticmethod
    def forward(ctx, q, k, frequencies, scale):
        ctx.save_for_backward(frequencies)
        ctx.scale = scale
        return training.fira_rotary(q, k, None, frequencies, scale=scale)

    @staticmethod
    def backward(ctx, dq, dk):
        return (*training.fira_rotary_gradient(dq, dk, None, ctx.saved_tensors[0], scale=ctx.scale), None, None)


class Between(torch.autograd.Function):
    """The stream after a block, and the next block's norm of it; the gradients of gate, weight and post_weight are added to `totals` (fp32)."""

    @staticmethod
    def forward(ctx, x, block, gate, weight, post_weight, totals):
        r = training.fira_block_norm(x, block, weight, gate=gate, post_weight=post_weight, norm=fira.FIRA_RMS_NORM, post=fira.FIRA_RMS_NORM)
        ctx.save_for_backward(r.residual, block, gate, weight, post_weight, r.rstd, r.post_rstd)
        ctx.totals = totals
        return r.residual, r.y

    @staticmethod
    def backward(ctx, dr, dy):
        residual, block, gate, weight, post_weight, rstd, post_rstd = ctx.saved_tensors
        dgate, dweight, dpost_weight = ctx.totals
        g = training.fira_block_norm_gradient(dr, dy, residual, block, weight, None, rstd, gate=gate, post_weight=post_weight, post_rstd=post_rstd, norm=fira.FIRA_RMS_NORM,
                                              post=fira.FIRA_RMS_NORM, dgate=dgate, dweight=dweight, dpost_weight=dpost_weight, accumulate=True)
        return g.dx, g.dblock, None, None, None, None


class AttentionModel:
    """Parameters, their accumulated gradients, and the two optimizers."""

    def __init__(self, vocab=512, dim=128, heads=4, kv_heads=2, hidden=256, rank=32, max_norm=0.5, state=torch.float32, seed=0):
        gen = torch.Generator(device=DEV)
        gen.manual_seed(seed)
        self.dim, self.heads, self.kv_heads, self.head = dim, heads, kv_heads, dim // heads
        # three quarters of a head are turned, for texts of twice the length
        self.frequencies, self.turn_scale = training.fira_rotary_frequencies(self.head // 8 * 6, context=fira.FIRA_ROTARY_BY_PARTS, factor=2.0, trained=64.0)
        low_rank = {"qkv": (dim, (heads + 2 * kv_heads) * self.head), "out": (dim, dim), "up": (dim, hidden), "down": (hidden, dim)}
        full = {"table": (vocab, dim), "unembed": (dim, vocab)}
        self.p = {k: (0.02 * torch.randn(s, device=DEV, generator=gen)).to(BF16) for k, s in {**low_rank, **full}.items()}
        vectors = {k: 1.0 for k in ("norm0", "norm1", "norm2", "post1", "post2")} | {"gate1": 0.5, "gate2": 0.5}
        self.p.update({k: torch.full((dim,), v, device=DEV) for k, v in vectors.items()})
        self.scale = math.sqrt(dim)
        self.total = {k: torch.zeros(v.shape, dtype=F32, device=DEV) for k, v in self.p.items()}     # gradients of all micro-batches
        self.grad = {k: torch.empty_like(v) for k, v in self.p.items()}                            # ... clipped, as the optimizers take them
        self.clip = training.GradientList(list(self.total.values()), list(self.grad.values()))
        self.max_norm = max_norm
        self.matrices, others = list(low_rank), [k for k in self.p if k not in low_rank]
        self.ctx = fira.FiraContext(list(low_rank.values()), rank, fira.FIRA_BF16, hp=fira.make_hparams(lr=3e-3, beta2=0.99, gamma=1.01), device=DEV)
        self.list = self.ctx.prepare(list(range(len(self.matrices))), [self.p[k] for k in self.matrices], [self.grad[k] for k in self.matrices])
        # (8 bits for what is large, decay for what is a matrix)
        self.adamw = training.AdamWList([self.p[k] for k in others], [self.grad[k] for k in others], weight_decay=[0.01 if k in full else 0.0 for k in others],
                                        state=[state if k in full else torch.float32 for k in others])
        self.workspace, self.steps = None, 0

    def loss(self, ids):
        """Mean loss of predicting ids[:, 1:] from ids[:, :-1]; after .backward() the gradients are in self.total."""
        p, t = self.p, self.total
        leaf = {k: p[k].detach().requires_grad_(True) for k in (*self.matrices, "table", "unembed")}
        for k in (*self.matrices, "unembed"):
            leaf[k].register_hook(added_to(t[k]))
        x = Lookup.apply(leaf["table"], ids[:, :-1], self.scale, t["table"])
        y = Norm.apply(x, p["norm0"], None, True, t["norm0"], None)
        x, y = Between.apply(x, self.attention(y @ leaf["qkv"]) @ leaf["out"], p["gate1"], p["norm1"], p["post1"], (t["gate1"], t["norm1"], t["post1"]))
        _, y = Between.apply(x, torch.nn.functional.silu(y @ leaf["up"]) @ leaf["down"], p["gate2"], p["norm2"], p["post2"], (t["gate2"], t["norm2"], t["post2"]))
        return torch.nn.functional.cross_entropy((y @ leaf["unembed"]).flatten(0, 1).float(), ids[:, 1:].flatten())

    def attention(self, qkv):
        """Causal attention of the heads in one buffer, in fp32."""
        b, n, _ = qkv.shape
        h, k = self.heads, self.kv_heads
        qkv = qkv.view(b, n, h + 2 * k, self.head)
        q, key = Turn.apply(qkv[:, :, :h], qkv[:, :, h:h + k], self.frequencies, self.turn_scale)
        q, key, value = (x.float().transpose(1, 2).contiguous() for x in (q, key.repeat_interleave(h // k, 2), qkv[:, :, h + k:].repeat_interleave(h // k, 2)))
        scores = q @ key.transpose(2, 3) / math.sqrt(self.head)
        later = torch.ones(n, n, dtype=torch.bool, device=DEV).triu(1)
        return (scores.masked_fill(later, -math.inf).softmax(-1) @ value).transpose(1, 2).reshape(b, n, h * self.head).to(BF16)

    def step(self, batches, refresh_every=40):
        """One step of both optimizers over the micro-batches -> (mean loss, norm of the gradients before clipping), on the GPU."""
        for t in self.total.values():
            t.zero_()
        mean = 0.0
        for ids in batches:
            loss = self.loss(ids)
            (loss / len(batches)).backward()
            mean = mean + loss.detach() / len(batches)
        norm = self.clip.fira_clip_gradients(self.max_norm)
        if self.steps % refresh_every == 0:
            self.workspace = self.ctx.fira_refresh_projectors(list(range(len(self.matrices))), [self.grad[k] for k in self.matrices], iters=2, seed=self.steps, workspace=self.workspace)
        self.ctx.fira_step(prepared=self.list)
        self.adamw.fira_adamw_step(3e-3, beta2=0.99)
        self.steps += 1
        return mean, norm


def train(steps=120, state=torch.float32, report=None):
    """-> the model, losses of the steps, norms of their gradients."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1)
    model = AttentionModel(state=state)
    successor = torch.randperm(model.p["table"].shape[0], device=DEV, generator=gen)
    losses, norms = [], []
    for k in range(steps):
        loss, norm = model.step(batches(successor, 2, 32, 32, gen))
        losses.append(loss)
        norms.append(norm)
        if report and (k % 10 == 0 or k == steps - 1):
            report(f"step {k:4d}  loss {float(loss):.4f}  gradient norm {float(norm):.3f}")
    return model, [float(x) for x in losses], [float(x) for x in norms]


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=120)
    ap.add_argument("--state", choices=["f32", "e4m3"], default="f32")
    args = ap.parse_args()
    train(args.steps, torch.float8_e4m3fn if args.state == "e4m3" else torch.float32, report=lambda line: print(line, flush=True))
