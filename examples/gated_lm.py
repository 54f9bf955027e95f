"""A small language model of gated recurrent layers: training, prefill and decoding on one GPU.

The data are synthetic sequences over ``--vocab`` symbols: each follows one of ``--rules`` permutations, p -> next(p), so that
which symbol comes next depends on what a layer's state holds of the sequence so far.  A training step runs the layers forward and backward
(projection, gated scan, output projection, MLP) and one AdamW step over all tensors, whose gradients are scaled to a
largest norm on the GPU.  Afterwards a prompt is read in one call and continued token by token from the layers' states.

    python examples/gated_lm.py [--steps 300] [--dtype bf16] [--bits 8]
"""
import argparse
import os
import sys
import time

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_05583_amd import ops  # noqa: E402

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


class GatedLM:
    """Symbols' vectors, ``layers`` gated recurrent layers, and the product that gives the logits."""

    def __init__(self, vocab, d, layers, dtype, seed=0, device="cuda"):
        g = torch.Generator().manual_seed(seed)

        def weight(k, n):
            return (torch.randn(k, n, generator=g) / k ** 0.5).to(device, dtype)

        def fixed(n, value=0.0):
            return torch.full((n,), value, device=device)

        self.emb, self.head = weight(d, vocab).t().contiguous(), weight(d, vocab)
        self.layers = []
        for _ in range(layers):
            # damping softplus(theta) is positive; a channel forgets in one to some sixty tokens where its gate is half open
            theta = torch.logspace(-1.5, 0.3, d).expm1().log().to(device)
            self.layers.append(ops.GatedLayerParams(weight(d, 3 * d), fixed(3 * d), theta, weight(d, d), fixed(d),
                                                    weight(d, 4 * d), fixed(4 * d), weight(4 * d, d), fixed(d)))
        every = [self.emb, self.head] + [t for p in self.layers for t in p]
        for t in every:
            t.requires_grad_(True)
        # one optimizer state for each type of parameter
        self.groups = [g for g in ([t for t in every if t.dtype == k] for k in (torch.bfloat16, torch.float32)) if g]

    def damped(self):
        return [p._replace(gamma=F.softplus(p.gamma)) for p in self.layers]

    def logits(self, tokens):
        x = F.embedding(tokens, self.emb)
        for p in self.damped():
            x, _ = ops.resonator_gated_layer(x, p)
        return ops.resonator_linear(x, self.head)

    @torch.no_grad()
    def prefill(self, tokens, lengths=None):
        """Logits [B, L, vocab] of a prompt, and every layer's state after it."""
        x, states = self.emb[tokens], []
        for p in self.damped():
            x, h = ops.resonator_gated_layer_fwd(x, p, lengths=lengths, return_state=True)
            states.append(h)
        return ops.resonator_linear_fwd(x, self.head), states

    @torch.no_grad()
    def step(self, tokens, states, layers):
        """Logits [B, vocab] after one more token of every sequence; the states are advanced in place.  ``layers``: what
        damped() returned, which a decoding loop computes once."""
        x = self.emb[tokens]
        for p, h in zip(layers, states):
            x = ops.resonator_gated_layer_step(x, p, h)
        return ops.resonator_linear_fwd(x, self.head)


def sequences(B, L, vocab, rules, generator):
    """[B, L] symbols: a random first one, then those of one of ``rules`` fixed permutations."""
    fixed = torch.Generator().manual_seed(17)
    perm = torch.stack([torch.randperm(vocab, generator=fixed) for _ in range(rules)])
    rule = torch.randint(rules, (B,), generator=generator)
    t = [torch.randint(vocab, (B,), generator=generator)]
    for _ in range(L - 1):
        t.append(perm[rule, t[-1]])
    return torch.stack(t, 1).cuda()


def train(model, steps, B=32, L=128, vocab=32, rules=4, lr=2e-3, bits=32, seed=1, report=None):
    """The losses of ``steps`` steps."""
    g = torch.Generator().manual_seed(seed)
    states = [ops.adamw_state(group, bits=bits) for group in model.groups]
    losses = []
    for step in range(1, steps + 1):
        t = sequences(B, L + 1, vocab, rules, g)
        loss = F.cross_entropy(model.logits(t[:, :-1]).float().flatten(0, 1), t[:, 1:].flatten())
        loss.backward()
        grads = [[p.grad for p in group] for group in model.groups]
        norm = torch.stack([v.float().norm() for group in grads for v in group]).norm()
        scale = (1.0 / norm).clamp(max=1.0).reshape(1)
        for group, gr, state in zip(model.groups, grads, states):
            ops.resonator_adamw_step([p.detach() for p in group], gr, state, step=step, lr=lr, weight_decay=0.01,
                                     grad_scale=scale)
            for p in group:
                p.grad = None
        losses.append(loss.detach())
        if report and step % report == 0:
            print(f"step {step}: loss {losses[-1].item():.3f}", flush=True)
    return [v.item() for v in losses]


@torch.no_grad()
def generate(model, prompt, n):
    """``n`` further tokens, the likeliest ones."""
    logits, states = model.prefill(prompt)
    layers = model.damped()
    out, t = [], logits[:, -1].argmax(-1)
    for _ in range(n):
        out.append(t)
        t = model.step(t, states, layers).argmax(-1)
    return torch.stack(out, 1)


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=300)
    ap.add_argument("--dim", type=int, default=256)
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--vocab", type=int, default=32)
    ap.add_argument("--rules", type=int, default=4)
    ap.add_argument("--dtype", choices=DTYPES, default="bf16")
    ap.add_argument("--bits", type=int, choices=(8, 32), default=32)
    a = ap.parse_args()
    model = GatedLM(a.vocab, a.dim, a.layers, DTYPES[a.dtype])
    began = time.perf_counter()
    losses = train(model, a.steps, vocab=a.vocab, rules=a.rules, bits=a.bits, report=max(1, a.steps // 10))
    torch.cuda.synchronize()
    print(f"{(time.perf_counter() - began) / a.steps * 1e3:.2f} ms a step; loss {losses[0]:.3f} to {losses[-1]:.3f}")
    t = sequences(16, 96, a.vocab, a.rules, torch.Generator().manual_seed(2))
    right = generate(model, t[:, :32], 64) == t[:, 32:]
    print(f"64 tokens after a prompt of 32: {right.float().mean().item() * 100:.1f} % are the rule's")


if __name__ == "__main__":
    main()
