"""A decoder block trained with the package's operators and optimizer.

    python examples/train_block.py [--steps 60]

Tokens are looked up in a scaled table (``embed``); the residual is added and normalised in
one pass (``add_norm``); queries and keys are normalised per head and rotated
(``qk_norm_rope``) and go through ``attention`` with grouped heads; the loss comes from
``token_logprob``. Every projection keeps its input in 8 bits for the backward pass
(``act_pack``) and forms its weight gradient from it (``weight_grad``) in the buffer that
``HiMuon`` steps on; the table's gradient comes from the sorted tokens (``embed_grad``). All of
them join autograd by themselves, the projections through the function below.

The task: every token has one successor, and a sequence walks from a random one on.
"""
import argparse
import math
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch
import torch.nn.functional as F

import paper_2606_27216_amd as hm

VOCAB, WIDTH, HEADS, KV_HEADS, HEAD, HIDDEN = 1000, 256, 8, 4, 64, 1024
BATCH, SEQ = 16, 128
EPS = 1e-6


class Linear8(torch.autograd.Function):
    """x W^T whose backward pass holds x in 8 bits (33 bytes for 32 values, not 64)
    and writes W's gradient into ``grad``, the buffer that the optimizer reads."""

    @staticmethod
    def forward(ctx, x, weight, grad):
        flat = x.reshape(-1, x.shape[-1])
        ctx.save_for_backward(weight, grad, *hm.act_pack(flat))
        return (flat @ weight.t()).view(*x.shape[:-1], weight.shape[0])

    @staticmethod
    def backward(ctx, g):
        weight, grad, codes, exps = ctx.saved_tensors
        flat = g.reshape(-1, g.shape[-1])
        hm.weight_grad(flat, codes, exps, out=grad)
        return (flat @ weight).view(*g.shape[:-1], weight.shape[1]), None, None


class Block:
    def __init__(self, seed=0, device="cuda"):
        gen = torch.Generator(device=device).manual_seed(seed)

        def matrix(rows, cols):
            return (torch.randn(rows, cols, generator=gen, device=device) / math.sqrt(cols)).bfloat16()

        self.weights = {"qkv": matrix((HEADS + 2 * KV_HEADS) * HEAD, WIDTH), "o": matrix(WIDTH, HEADS * HEAD),
                        "up": matrix(HIDDEN, WIDTH), "down": matrix(WIDTH, HIDDEN), "head": matrix(VOCAB, WIDTH)}
        self.grads = {n: torch.zeros_like(w) for n, w in self.weights.items()}
        self.table = (0.02 * torch.randn(VOCAB, WIDTH, generator=gen, device=device)).bfloat16().requires_grad_()
        self.gains = [torch.ones(HEAD, device=device, requires_grad=True) for _ in range(2)]
        self.norm_gains = [torch.ones(WIDTH, device=device, requires_grad=True) for _ in range(3)]
        rate = 10000.0 ** (-torch.arange(HEAD // 2, device=device, dtype=torch.float64) / (HEAD // 2))
        angle = torch.arange(SEQ, device=device, dtype=torch.float64)[:, None] * rate
        self.cos, self.sin = angle.cos().float(), angle.sin().float()

    def linear(self, name, x):
        return Linear8.apply(x, self.weights[name], self.grads[name])

    def embed(self, tokens):
        return hm.embed(tokens, self.table, scale=math.sqrt(WIDTH))

    def norm_rope(self, q, k):
        return hm.qk_norm_rope(q, k, *self.gains, self.cos, self.sin, eps=EPS)

    def add_norm(self, x, residual, i):
        return hm.add_norm(x, residual, self.norm_gains[i], eps=EPS)

    def attention(self, q, k, v):
        return hm.attention(q, k, v)[0]

    def logprob(self, logits, tokens):
        return hm.token_logprob(logits, tokens)[0]

    def loss(self, tokens):
        B, S = tokens.shape
        x, y = self.add_norm(self.embed(tokens), None, 0)
        qkv = self.linear("qkv", y).view(B, S, HEADS + 2 * KV_HEADS, HEAD)
        q, k = self.norm_rope(qkv[:, :, :HEADS], qkv[:, :, HEADS:HEADS + KV_HEADS])
        y = self.attention(q, k, qkv[:, :, HEADS + KV_HEADS:]).reshape(B, S, HEADS * HEAD)
        x, y = self.add_norm(self.linear("o", y), x, 1)
        x, y = self.add_norm(self.linear("down", F.silu(self.linear("up", y))), x, 2)
        # (the last token of a sequence has no successor: -1 is no token, and counts for nothing)
        return -self.logprob(self.linear("head", y), F.pad(tokens[:, 1:], (0, 1), value=-1)).sum() / (B * (S - 1))


class Walks:
    """Sequences of tokens that each follow the one before: token order[i] by order[i + 1]."""

    def __init__(self, seed):
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.order = torch.randperm(VOCAB, generator=self.gen, device="cuda")

    def batch(self):
        start = torch.randint(0, VOCAB, (BATCH, 1), generator=self.gen, device="cuda")
        return self.order[(start + torch.arange(SEQ, device="cuda")) % VOCAB]


def train(steps, seed=0, lr=0.02, say=print):
    block = Block(seed)
    optimizer = hm.HiMuon(block.weights.values(), T=128, lr=lr, momentum=0.9)
    rest = torch.optim.Adam([block.table, *block.gains, *block.norm_gains], lr=lr / 10, eps=1e-6)
    data = Walks(seed + 1)
    losses = []
    for step in range(steps):
        loss = block.loss(data.batch())
        rest.zero_grad()
        loss.backward()
        optimizer.step(list(block.grads.values()))
        rest.step()
        losses.append(loss.detach())
        if say and (step % 10 == 0 or step == steps - 1):
            say(f"step {step:4d}  loss {float(losses[-1]):.4f}", flush=True)
    return [float(v) for v in losses]


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    parser.add_argument("--steps", type=int, default=100)
    train(parser.parse_args().steps)
