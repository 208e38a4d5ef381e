"""Fine-tunes the example's mixture-of-experts model on synthetic answers with the library's losses: pairs of a better and a
worse answer, or answers with rewards (a clipped policy loss with a penalty on the distance to the starting model and a bonus
for entropy). The routers' balance loss is added, MoARa takes the step.

    python examples/align_moe.py [--objective preference|policy] [--steps 20]
"""
import argparse
import copy
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from examples.train_moe import Model  # noqa: E402
from paper_2609_15037_amd import moara as M  # noqa: E402
from paper_2609_15037_amd.losses import policy_loss, preference_loss, token_logps  # noqa: E402
from paper_2609_15037_amd.optim import MoARa, moara_targets  # noqa: E402

PROMPT, LENGTH, VOCAB = 8, 40, 512


def batch(pairs, generator):
    """Tokens of 2 x pairs answers, better and worse in turn (a better one has more even tokens), and which positions are
    an answer's: prompts are not, nor what follows an answer's end."""
    tokens = torch.randint(0, VOCAB, (2 * pairs, LENGTH), generator=generator)
    tokens[0::2, PROMPT:] &= -1 - (torch.rand(pairs, LENGTH - PROMPT, generator=generator) < 0.6).long()
    end = torch.randint(PROMPT + 4, LENGTH + 1, (2 * pairs, 1), generator=generator)
    at = torch.arange(1, LENGTH)[None]
    return tokens.cuda(), ((at >= PROMPT) & (at < end)).cuda()


def logps(model, tokens, answer, entropy=False, balance=None, aux=None):
    """Log-probabilities of the answers' tokens; the other positions have no label."""
    logits = model(tokens, balance, aux)
    labels = torch.where(answer, tokens[:, 1:], -100)
    return token_logps(logits[:, :-1], labels, entropy=entropy)


def objective(name, model, reference, old, tokens, answer, aux=None):
    """The loss of one batch, and what it is made of."""
    balance = model.layers[0].router.balance_config(balance_coef=1e-2, z_coef=1e-4)
    aux = [] if aux is None else aux
    with torch.no_grad():
        ref = logps(reference, tokens, answer)
    if name == "preference":
        logp = logps(model, tokens, answer, balance=balance, aux=aux)
        loss, _, about = preference_loss(M.moara_preference_default_config(beta=0.2), logp, ref, mask=answer)
        return sum(aux, loss), about
    logp, entropy = logps(model, tokens, answer, True, balance, aux)
    even = ((tokens[:, 1:] % 2 == 0) & answer).sum(dim=1) / answer.sum(dim=1)
    advantages = (even - even.mean()) / (even.std() + 1e-6)
    cfg = M.moara_policy_default_config(kl_coef=0.02, entropy_coef=1e-3, sequence_advantages=1)
    loss, about = policy_loss(cfg, logp, advantages, old_logp=old, ref_logp=ref, entropy=entropy, mask=answer)
    return sum(aux, loss), about


def train(name="preference", steps=20, pairs=8, seed=0, say=print):
    """What each step's loss was made of."""
    torch.manual_seed(seed)
    model = Model(vocab=VOCAB).cuda()
    reference = copy.deepcopy(model).eval().requires_grad_(False)
    targets, others = moara_targets(model)
    opt = MoARa(targets, others, lr=2e-3, rank_table=[32] * M.MOARA_NUM_MODULES, block_size=64, refresh_interval=20,
                adamw_bits=8, max_grad_norm=1.0)
    generator = torch.Generator().manual_seed(seed)
    history = []
    for step in range(steps):
        if step % 4 == 0 or name == "preference":       # four steps on the answers of one policy
            tokens, answer = batch(pairs, generator)
            with torch.no_grad():
                old = logps(model, tokens, answer)
        loss, about = objective(name, model, reference, old, tokens, answer)
        loss.backward()
        opt.step()
        opt.zero_grad()
        history.append(about)
        if step % 5 == 0 or step == steps - 1:
            say(f"step {step}: loss {float(loss.detach()):.4f}, " + ", ".join(f"{x:.4f}" for x in about.tolist()))
    return torch.stack(history)


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--objective", choices=("preference", "policy"), default="preference")
    ap.add_argument("--steps", type=int, default=20)
    a = ap.parse_args()
    train(a.objective, a.steps)
