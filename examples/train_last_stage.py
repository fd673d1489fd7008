"""A training step of a two-stage pipeline in one process, end to end: the
first stage's hidden state crosses a compressed boundary, the last stage turns
it into a loss over the vocabulary, its gradient goes back across the
boundary, and both stages clip and update their parameters.

The task is a next-token rule (each token is followed by a fixed other one, a
tenth of the positions are padding), so the loss falls from log(vocabulary)
towards 0 within some hundred steps.

  python examples/train_last_stage.py [--steps 200] [--state-bits 8]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2401_07788_amd import boundary, head, optim  # noqa: E402

PADDING = -100


class Pipeline:
    def __init__(self, vocab=2000, hidden=256, dtype=torch.bfloat16, state_bits=8, keep=(3, 10), seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def weight(*shape):
            w = torch.randn(shape, generator=g, device="cuda") / math.sqrt(shape[-1])
            return w.to(dtype).requires_grad_()

        self.embed, self.w1 = weight(vocab, hidden), weight(hidden, hidden)      # first stage
        self.w2, self.vocab = weight(hidden, hidden), weight(vocab, hidden)      # last stage
        self.boundary = boundary.TopkBoundary(*keep)
        opt = dict(lr=4e-3, weight_decay=0.01, state_bits=state_bits, master=True)
        self.stages = [(ps, optim.AdamW(ps, **opt)) for ps in ([self.embed, self.w1], [self.w2, self.vocab])]

    def step(self, tokens, target):
        """one step on tokens and their targets (PADDING: none); returns the mean loss"""
        hidden = torch.tanh(self.embed[tokens] @ self.w1.t())
        hidden = self.boundary(hidden)                                            # across, both ways
        out = hidden + torch.tanh(hidden @ self.w2.t())
        counted = target != PADDING
        weight = counted.float() / counted.sum()
        r = head.linear_xent_step(out.detach(), self.vocab.detach(), target, weight, ignore_index=PADDING)
        out.backward(r.dx)
        self.vocab.grad = r.dw
        for params, opt in self.stages:
            grads = [p.grad for p in params]
            opt.step(grads, clip=optim.grad_norm(grads, 1.0))
            for p in params:
                p.grad = None
        return (r.loss * weight).sum()


def batch(vocab, n, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    tokens = torch.randint(0, vocab, (n,), generator=g, device="cuda")
    target = (tokens * 7 + 3) % vocab
    target[torch.rand(n, generator=g, device="cuda") < 0.1] = PADDING
    return tokens, target


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--vocab", type=int, default=2000)
    ap.add_argument("--state-bits", type=int, default=8, choices=(8, 32))
    a = ap.parse_args()
    model = Pipeline(vocab=a.vocab, state_bits=a.state_bits)
    for k in range(a.steps):
        loss = model.step(*batch(a.vocab, a.tokens, k))
        if k % 20 == 0 or k == a.steps - 1:
            print(f"step {k:4d}  loss {float(loss):.4f}  (log vocabulary {math.log(a.vocab):.4f})", flush=True)


if __name__ == "__main__":
    main()
