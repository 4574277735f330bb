"""A small language model with a layer of experts, tuned by the clipped policy loss.

The model looks a token up in the vocabulary matrix W, passes it through two of its experts, adds what they say (with dropout) to
the token's own vector, normalises, and predicts the next token with W:

    e = W[token];  z = e + dropout(sum over the token's experts of weight down relu(up e)^2);  y = layer norm(z);  logits = y W^T

It writes answers, token after token. An answer is the better the more of its steps follow a chain that is fixed beforehand; answers to the same
prompt are compared with one another. The policy loss of the answers' tokens has a KL term that keeps the model close to where it began. W and the norm's weights are
the compressed step's parameter vector, their gradients go straight into its gradient array; the experts' matrices take orthogonalised updates.

    python examples/policy_tuning.py --steps 40
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2210_07454_b200 import binding, operators  # noqa: E402


class Experts:
    """A token's vector through `chosen` of its experts: forward keeps what backward needs."""

    def __init__(self, experts, width, hidden, chosen, gen):
        self.chosen = chosen
        self.router = torch.randn(experts, width, generator=gen, device="cuda") / math.sqrt(width)
        self.up = torch.randn(experts, hidden, width, generator=gen, device="cuda") / math.sqrt(width)
        self.down = torch.randn(experts, width, hidden, generator=gen, device="cuda") / math.sqrt(hidden)

    def forward(self, e):
        """e: (tokens, width) bf16. Returns (tokens, width) bf16 and what backward takes."""
        scores = e.float() @ self.router.T
        top, experts = scores.topk(self.chosen, dim=1)
        weights = torch.softmax(top, 1)
        order, places, offsets = operators.sort_by_expert(experts, len(self.router))
        rows = e[order // self.chosen]
        up, down = self.up.bfloat16(), self.down.bfloat16()
        h = operators.grouped_linear(rows, up, offsets)
        a = torch.relu(h).square()
        o = operators.grouped_linear(a, down, offsets)
        mixed = (o[places].float() * weights[:, :, None]).sum(1).bfloat16()
        return mixed, (e, weights, experts, order, places, offsets, rows, up, down, h, a, o)

    def backward(self, dmixed, kept):
        """Returns the gradient of e (fp32) and those of (router, up, down)."""
        e, weights, experts, order, places, offsets, rows, up, down, h, a, o = kept
        d = dmixed.float()
        dweights = (o[places].float() * d[:, None]).sum(2)
        dout = (weights[:, :, None] * d[:, None]).bfloat16().flatten(0, 1)[order]
        da, ddown = operators.grouped_linear_backward(dout, a, down, offsets)
        dh = da * (2 * torch.relu(h))
        drows, dup = operators.grouped_linear_backward(dh, rows, up, offsets)
        dtop = weights * (dweights - (weights * dweights).sum(1, keepdim=True))
        dscores = torch.zeros(len(e), len(self.router), device=e.device).scatter_(1, experts, dtop)
        return drows[places].float().sum(1) + dscores @ self.router, (dscores.T @ e.float(), dup, ddown)


class Model:
    def __init__(self, vocab, width, hidden, experts, chosen, dropout, seed):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.vocab, self.width, self.dropout = vocab, width, dropout
        self.d = vocab * width + 2 * width
        self.x = torch.zeros(self.d, device="cuda")                  # vocabulary matrix, norm weight, norm bias
        w, gamma, _ = self.parts(self.x)
        w.copy_(torch.randn(vocab, width, generator=gen, device="cuda") / math.sqrt(width))
        gamma.fill_(1.0)
        self.experts = Experts(experts, width, hidden, chosen, gen)
        self.momentum = [torch.zeros_like(m) for m in (self.experts.up, self.experts.down)]

    def parts(self, vector):
        n = self.vocab * self.width
        return vector[:n].view(self.vocab, self.width), vector[n:n + self.width], vector[n + self.width:]

    def forward(self, token, target, seed=None):
        """Losses (negative log probabilities) of `target` after `token`, and what backward takes. seed: of the dropout, None: without."""
        w, gamma, beta = self.parts(self.x)
        w16 = w.bfloat16()
        e = w16[token]
        mixed, kept = self.experts.forward(e)
        z = operators.dropout(mixed, self.dropout if seed is not None else 0.0, seed or 0, residual=e)
        y, mean, rstd = operators.layer_norm(z, gamma, beta)
        loss, lse = operators.linear_cross_entropy(y, w16, target)
        return loss, (token, target, seed, w16, gamma, kept, z, y, mean, rstd, lse)

    def backward(self, dloss, state, row):
        """Gradients of W and the norm into `row` (d); those of the experts' layer are returned."""
        token, target, seed, w16, gamma, kept, z, y, mean, rstd, lse = state
        dw, dgamma, dbeta = self.parts(row)
        dy, _ = operators.linear_cross_entropy_backward(dloss, y, w16, target, lse, dweight=dw)
        dz, _, _ = operators.layer_norm_backward(dy, z, gamma, mean, rstd, dweight=dgamma, dbias=dbeta)
        dmixed = operators.dropout_backward(dz, self.dropout, seed) if seed is not None else dz
        de, others = self.experts.backward(dmixed, kept)
        dw.index_add_(0, token, de + dz.float())                     # the looked-up rows' share
        return others

    def answers(self, prompt, length, gen):
        """(answers, length + 1) tokens drawn from the model, the prompt first."""
        w, gamma, beta = self.parts(self.x)
        tokens = [prompt]
        for _ in range(length):
            e = w.bfloat16()[tokens[-1]]
            z = e + self.experts.forward(e)[0]
            y, _, _ = operators.layer_norm(z, gamma, beta)
            p = torch.softmax(y.float() @ w.T, 1)
            tokens.append(torch.multinomial(p, 1, generator=gen)[:, 0])
        return torch.stack(tokens, 1)


def tune(steps=40, prompts=16, answers=8, length=12, vocab=256, width=64, hidden=128, experts=8, chosen=2, dropout=0.05, successors=32, lr=0.01,
         expert_lr=0.01, kl=0.01, seed=0, log=None):
    """Returns the mean reward of every step (the share of steps that follow the chain)."""
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    model = Model(vocab, width, hidden, experts, chosen, dropout, seed)
    follows = torch.zeros(vocab, vocab, dtype=torch.bool, device="cuda")
    follows.scatter_(1, torch.rand(vocab, vocab, generator=gen, device="cuda").topk(successors, 1).indices, True)
    grads = torch.zeros(1, model.d, device="cuda")
    step = binding.SketchedAMSGrad(model.d, 1, 5, 4096, model.d // 4, seed=seed, lr=lr, beta1=0.9, beta2=0.99, eps=1e-6)
    step.set_stream(torch.cuda.current_stream().cuda_stream)
    start = Model(vocab, width, hidden, experts, chosen, dropout, seed)              # the reference: the same model before any step
    offsets = torch.arange(prompts * answers + 1, device="cuda") * length
    rewards = []
    for t in range(steps):
        prompt = torch.randint(0, vocab, (prompts,), generator=gen, device="cuda").repeat_interleave(answers)
        written = model.answers(prompt, length, gen)
        token, target = written[:, :-1].flatten(), written[:, 1:].flatten()
        reward = follows[token, target].float().view(prompts, answers, length).mean(2)
        spread = reward - reward.mean(1, keepdim=True)
        advantages = (spread / (spread.square().mean(1, keepdim=True).sqrt() + 1e-4)).flatten()
        old, _ = model.forward(token, target)
        reference, _ = start.forward(token, target)
        for again in range(2):                                       # two updates on the same answers: the second one's ratios are not 1
            nll, state = model.forward(token, target, seed=(seed << 32) + 2 * t + again)
            args = dict(targets=target, offsets=offsets, reference_nll=reference, kl=kl, advantage_of="sequences")
            result, norm = operators.policy_loss(nll, old, advantages, average="sequences", **args)
            dnll = operators.policy_loss_backward(None, nll, old, advantages, norm, **args)
            drouter, dup, ddown = model.backward(dnll, state, grads[0])
            step.step(grads, model.x)
            layer = model.experts
            layer.router.sub_(lr * drouter)
            for matrix, gradient, momentum in ((layer.up, dup, model.momentum[0]), (layer.down, ddown, model.momentum[1])):
                matrix.sub_(expert_lr * operators.orthogonalize(gradient, momentum=momentum).float())
        rewards.append(float(reward.mean()))
        if log and (t % 5 == 0 or t == steps - 1):
            loss, drift, clipped = result.tolist()
            log(f"step {t:4d}  reward {rewards[-1]:.4f}  loss {loss:+.4f}  drift {drift:.5f}  clipped {clipped:.3f}")
    step.sync()
    operators.sync()
    return rewards


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=40)
    a = ap.parse_args()
    out = tune(steps=a.steps, log=print)
    print(f"reward: first {out[0]:.4f}, last {out[-1]:.4f}")
