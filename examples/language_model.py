"""A small language model trained by n simulated workers with everything the library has for one.

Tokens follow a fixed random chain (each has a few likely successors).  The model looks a token up in the vocabulary matrix W, passes it
through a hidden matrix M with a residual, normalises, and predicts the next token with W again:

    e = W[token];  z = e + M e;  y = layer norm(z);  loss = cross entropy(y W^T, next token)

Every worker has its own batch.  W and the norm's weights are the optimiser's parameter vector x: the gradients go straight into the
worker's row of the (n, d) gradient array, and the compressed step updates x.  The hidden matrix takes the mean of the
workers' gradients as an orthogonalised update with a momentum.

    python examples/language_model.py --steps 60
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2210_07454_b200 import binding, operators  # noqa: E402


class Chain:
    """Tokens with `choices` equally likely successors each."""

    def __init__(self, vocab, choices, seed):
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.next = torch.randint(0, vocab, (vocab, choices), generator=self.gen, device="cuda")

    def batch(self, tokens):
        vocab, choices = self.next.shape
        now = torch.randint(0, vocab, (tokens,), generator=self.gen, device="cuda")
        pick = torch.randint(0, choices, (tokens,), generator=self.gen, device="cuda")
        return now, self.next[now, pick]


class Model:
    def __init__(self, vocab, width, seed):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.vocab, self.width = vocab, width
        self.d = vocab * width + 2 * width
        self.x = torch.zeros(self.d, device="cuda")                      # vocabulary matrix, norm weight, norm bias
        w, gamma, _ = self.parts(self.x)
        w.copy_(torch.randn(vocab, width, generator=gen, device="cuda") / math.sqrt(width))
        gamma.fill_(1.0)
        self.hidden = torch.randn(width, width, generator=gen, device="cuda") / math.sqrt(width)
        self.momentum = torch.zeros_like(self.hidden)

    def parts(self, vector):
        """Views of a d-vector: the vocabulary matrix, the norm's weight and bias."""
        n = self.vocab * self.width
        return vector[:n].view(self.vocab, self.width), vector[n:n + self.width], vector[n + self.width:]

    def gradients(self, token, target, row):
        """Mean loss of one worker's batch; its gradients go into `row` (d), the hidden matrix' is returned."""
        w, gamma, beta = self.parts(self.x)
        dw, dgamma, dbeta = self.parts(row)
        w16, m16 = w.bfloat16(), self.hidden.bfloat16()
        e = w16[token]
        z = e + e @ m16.T
        y, mean, rstd = operators.layer_norm(z, gamma, beta)
        loss, lse = operators.linear_cross_entropy(y, w16, target)
        dloss = torch.full_like(loss, 1.0 / len(loss))
        dy, _ = operators.linear_cross_entropy_backward(dloss, y, w16, target, lse, dweight=dw)
        dz, _, _ = operators.layer_norm_backward(dy, z, gamma, mean, rstd, dweight=dgamma, dbias=dbeta)
        dw.index_add_(0, token, (dz + dz @ m16).float())                 # the looked-up rows' share
        return loss.mean(), dz.T.float() @ e.float()


def train(steps=60, workers=4, vocab=1024, width=128, tokens=512, choices=4, lr=0.02, hidden_lr=0.02, seed=0, log=None):
    """Returns the mean loss of every step (the chain's own entropy, log(choices), is the least there is)."""
    chain, model = Chain(vocab, choices, seed + 1), Model(vocab, width, seed)
    grads = torch.zeros(workers, model.d, device="cuda")
    step = binding.SketchedAMSGrad(model.d, workers, 5, 16384, model.d // 8, seed=seed, lr=lr, beta1=0.9, beta2=0.99, eps=1e-6)
    step.set_stream(torch.cuda.current_stream().cuda_stream)
    losses = []
    for t in range(steps):
        parts = [model.gradients(*chain.batch(tokens), grads[w]) for w in range(workers)]
        step.step(grads, model.x)
        dm = torch.stack([p[1] for p in parts]).mean(0)
        model.hidden.sub_(hidden_lr * operators.orthogonalize(dm, momentum=model.momentum).float())
        losses.append(float(torch.stack([p[0] for p in parts]).mean()))
        if log and (t % 10 == 0 or t == steps - 1):
            log(f"step {t:4d}  loss {losses[-1]:.4f}")
    step.sync()
    operators.sync()
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--workers", type=int, default=4)
    a = ap.parse_args()
    out = train(steps=a.steps, workers=a.workers, log=print)
    print(f"first {out[0]:.4f}, last {out[-1]:.4f}, entropy of the chain {math.log(4):.4f}, of the vocabulary {math.log(1024):.4f}")
