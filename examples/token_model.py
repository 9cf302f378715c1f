"""A small next-token model on pruned linear layers, trained and then asked, on one MI355X.

    python examples/token_model.py [--steps 200] [--state-bits 8]

Residual blocks of two linear layers whose input gradients are pruned 2:4, block norms between them, token log
probabilities as the loss (with a small entropy bonus), AdamW on fp32 masters that writes the layers' bf16 weights as it
steps.  The data is a Markov chain with four equally likely successors for each token, so the loss has a floor of
ln 4 = 1.386 nats.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2202_00774_amd as sdgp                                                # noqa: E402
from paper_2202_00774_amd.autograd import sdgp_block_norm, sdgp_linear, sdgp_token_logprobs  # noqa: E402
from paper_2202_00774_amd.optim import AdamW                                       # noqa: E402

VOCAB, WIDTH, HIDDEN, BLOCKS, SUCCESSORS = 500, 256, 512, 2, 4


class TokenModel:
    """Weights as bf16 leaves by name, with fp32 masters of the same order for the optimizer."""

    def __init__(self, seed: int = 0):
        g = torch.Generator().manual_seed(seed)
        shapes = {"embed": (VOCAB, WIDTH), "head": (VOCAB, WIDTH), "pre0": (WIDTH,)}
        for b in range(BLOCKS):
            shapes.update({f"up{b}": (HIDDEN, WIDTH), f"down{b}": (WIDTH, HIDDEN), f"post{b}": (WIDTH,), f"gate{b}": (WIDTH,),
                           f"pre{b + 1}": (WIDTH,)})
        self.masters = {}
        for name, shape in shapes.items():
            w = torch.randn(shape, generator=g) * shape[-1] ** -0.5 if len(shape) == 2 else torch.full(shape, 0.5 if "gate" in name else 1.0)
            self.masters[name] = (w * WIDTH ** 0.5 if name == "embed" else w).cuda()
        self.weights = {k: v.to(torch.bfloat16).requires_grad_() for k, v in self.masters.items()}

    def logits(self, tokens: torch.Tensor, step: int = 0) -> torch.Tensor:
        w = self.weights
        y, h = sdgp_block_norm(F.embedding(tokens, w["embed"]), w_pre=w["pre0"])
        for b in range(BLOCKS):
            u = sdgp_linear(F.silu(sdgp_linear(h, w[f"up{b}"], 2, 4, sdgp.GREEDY_ADJUSTED)), w[f"down{b}"], 2, 4, sdgp.RANDOM, seed=step)
            y, h = sdgp_block_norm(y, u, w[f"gate{b}"], w[f"post{b}"], w[f"pre{b + 1}"])
        return sdgp_linear(h, w["head"], 2, 4, sdgp.GREEDY)


def chain(rows: int, length: int, seed: int) -> torch.Tensor:
    """Token sequences: from token t to one of (7 t + 1, 7 t + 2, .. , 7 t + SUCCESSORS) mod VOCAB."""
    g = torch.Generator().manual_seed(seed)
    out = torch.randint(0, VOCAB, (rows, length), generator=g)
    for i in range(1, length):
        out[:, i] = (7 * out[:, i - 1] + 1 + torch.randint(0, SUCCESSORS, (rows,), generator=g)) % VOCAB
    return out.cuda()


def train(model: TokenModel, steps: int, state_bits: int = 8, entropy_bonus: float = 0.001, report=None) -> list[float]:
    names = list(model.weights)
    optimizer = AdamW([model.masters[k] for k in names], lr=3e-3, weight_decay=0.01, state_bits=state_bits,
                      copies=[model.weights[k].detach() for k in names])
    losses = []
    for step in range(steps):
        tokens = chain(64, 33, 1000 + step)
        logp, entropy, _, _ = sdgp_token_logprobs(model.logits(tokens[:, :-1], step), tokens[:, 1:].contiguous())
        loss = -logp.mean() - entropy_bonus * entropy.mean()
        loss.backward()
        grads = [model.weights[k].grad for k in names]
        norm = torch.linalg.vector_norm(torch.stack([g.float().norm() for g in grads]))
        optimizer.step(grads, grad_scale=(1.0 / norm.clamp(min=1.0)).reshape(1))      # clipped to a norm of 1, on the GPU
        for k in names:
            model.weights[k].grad = None
        losses.append(-logp.detach().mean())
        if report and (step + 1) % 20 == 0:
            report(step + 1, losses[-1].item())
    return [loss.item() for loss in losses]


@torch.no_grad()
def ask(model: TokenModel, token: int, length: int = 8):
    """A sequence from `token` on, the most probable next token each time: [(token, its alternatives, their probabilities)]."""
    out = []
    for _ in range(length):
        logits = model.logits(torch.tensor([token], device="cuda"))
        _, _, top_logp, top_ids = sdgp_token_logprobs(logits, None, top=SUCCESSORS + 1)
        ids = top_ids[0].tolist()
        out.append((token, ids, top_logp[0].exp().tolist()))
        token = ids[0]
    return out


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--state-bits", type=int, choices=(8, 32), default=8)
    a = ap.parse_args()
    model = TokenModel()
    train(model, a.steps, a.state_bits, report=lambda step, loss: print(f"step {step:4d}  loss {loss:.3f} nats (floor {torch.tensor(float(SUCCESSORS)).log():.3f})", flush=True))
    for token, ids, p in ask(model, 3):
        print(f"after {token:3d}: " + ", ".join(f"{i} ({q:.2f})" for i, q in zip(ids, p)))


if __name__ == "__main__":
    main()
