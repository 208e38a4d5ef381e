"""Trains a small mixture-of-experts language model on synthetic tokens with everything the library has for
a training step: expert routing, MoARa on the projection and expert matrices, AdamW with 8-bit moments on
the embedding, norms, head and routers, clipping by the norm of all gradients.

    python examples/train_moe.py [--steps 40] [--bits 8|32]
"""
import argparse
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2609_15037_amd import moara as M  # noqa: E402
from paper_2609_15037_amd.optim import MoARa, moara_targets, warmup_cosine  # noqa: E402
from paper_2609_15037_amd.route import ExpertRouter  # noqa: E402


class Expert(torch.nn.Module):
    def __init__(self, d, ffn):
        super().__init__()
        self.gate_proj = torch.nn.Linear(d, ffn, bias=False)
        self.up_proj = torch.nn.Linear(d, ffn, bias=False)
        self.down_proj = torch.nn.Linear(ffn, d, bias=False)

    def forward(self, x):
        return self.down_proj(F.silu(self.gate_proj(x)) * self.up_proj(x))


class Layer(torch.nn.Module):
    def __init__(self, d, heads, ffn, experts, top_k):
        super().__init__()
        self.heads = heads
        self.norm1, self.norm2 = torch.nn.RMSNorm(d), torch.nn.RMSNorm(d)
        self.q_proj, self.k_proj, self.v_proj, self.o_proj = (torch.nn.Linear(d, d, bias=False) for _ in range(4))
        self.router = ExpertRouter(d, experts, top_k, score=M.MOARA_SIGMOID, renormalise=1)
        self.experts = torch.nn.ModuleList([Expert(d, ffn) for _ in range(experts)])

    def attention(self, x):
        b, t, d = x.shape
        q, k, v = (f(x).view(b, t, self.heads, -1).transpose(1, 2) for f in (self.q_proj, self.k_proj, self.v_proj))
        y = F.scaled_dot_product_attention(q, k, v, is_causal=True)
        return self.o_proj(y.transpose(1, 2).reshape(b, t, d))

    def mixture(self, x):
        """Every token's experts on its row, weighted; experts without tokens are not called."""
        rows = x.reshape(-1, x.shape[-1])
        index, weight = self.router(rows)
        out = torch.zeros_like(rows)
        for e in index[index >= 0].unique().tolist():
            token, slot = (index == e).nonzero(as_tuple=True)
            y = self.experts[e](rows[token]) * weight[token, slot, None].to(rows.dtype)
            out = out.index_add(0, token, y)
        return out.view_as(x)

    def forward(self, x):
        x = x + self.attention(self.norm1(x))
        return x + self.mixture(self.norm2(x))


class Model(torch.nn.Module):
    def __init__(self, vocab=512, d=128, heads=4, ffn=192, experts=8, top_k=2, layers=2):
        super().__init__()
        self.embed = torch.nn.Embedding(vocab, d)
        self.layers = torch.nn.ModuleList([Layer(d, heads, ffn, experts, top_k) for _ in range(layers)])
        self.norm = torch.nn.RMSNorm(d)
        self.head = torch.nn.Linear(d, vocab, bias=False)

    def forward(self, tokens):
        x = self.embed(tokens)
        for layer in self.layers:
            x = layer(x)
        return self.head(self.norm(x))


def train(steps=40, bits=8, seed=0, rate=1e-2, say=print):
    """Losses of the steps and the largest share of the tokens an expert had in the last one (layer by layer).
    rate: of the balancing bias."""
    torch.manual_seed(seed)
    model = Model().cuda()
    targets, others = moara_targets(model)
    ranks = [32] * M.MOARA_NUM_MODULES
    opt = MoARa(targets, others, lr=1e-2, rank_table=ranks, block_size=64, refresh_interval=20, adamw_bits=bits,
                max_grad_norm=1.0, adamw_seed=seed)
    sched = torch.optim.lr_scheduler.LambdaLR(opt, warmup_cosine(steps))
    tokens = torch.randint(0, 512, (8, 65), generator=torch.Generator().manual_seed(seed)).cuda()
    losses, share = [], []
    for step in range(steps):
        logits = model(tokens[:, :-1])
        loss = F.cross_entropy(logits.flatten(0, 1).float(), tokens[:, 1:].flatten())
        loss.backward()
        opt.step()
        sched.step()
        opt.zero_grad()
        share = [float(layer.router.load().max() / layer.router.load().sum()) for layer in model.layers]
        for layer in model.layers:
            layer.router.balance(rate)
        losses.append(float(loss.detach()))
        if step % 10 == 0 or step == steps - 1:
            say(f"step {step}: loss {losses[-1]:.4f}, gradient norm {float(opt.grad_norm):.3f}, "
                f"largest expert share {max(share):.2f}")
    return losses, share


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--bits", type=int, choices=(8, 32), default=8)
    a = ap.parse_args()
    train(a.steps, a.bits)
