"""A small language model of selective layers: training, prefill and decoding on one GPU.

The data and the loop are those of gated_lm.py; each layer's mixer is a short causal convolution and a selective scan, whose
heads hold a state [P, N] that the data write and read.

    python examples/selective_lm.py [--steps 300] [--dtype bf16] [--bits 8]
"""
import argparse
import os
import sys
import time

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import gated_lm as base  # noqa: E402
from paper_2607_05583_amd import ops  # noqa: E402


class SelectiveLM:
    """Symbols' vectors, ``layers`` selective layers of ``heads`` heads of P = 2 d / heads channels and one group of N ``states``, and the
    product that gives the logits."""

    def __init__(self, vocab, d, layers, dtype, heads=4, states=16, taps=4, seed=0, device="cuda"):
        g = torch.Generator().manual_seed(seed)

        def weight(k, n):
            return (torch.randn(k, n, generator=g) / k ** 0.5).to(device, dtype)

        def fixed(n, value=0.0):
            return torch.full((n,), value, device=device)

        wide = 2 * d
        cols = wide + 2 * states
        self.emb, self.head = weight(d, vocab).t().contiguous(), weight(d, vocab)
        self.layers = []
        for _ in range(layers):
            w = (torch.rand(cols, taps, generator=g) * 2 - 1).to(device) / taps ** 0.5
            # damping softplus(theta) is positive; steps of 1e-3 to 0.1 before the data move them
            theta = torch.linspace(1, 8, heads).expm1().log().to(device)
            steps = torch.logspace(-3, -1, heads).expm1().log().to(device)
            self.layers.append(ops.SelectiveLayerParams(
                weight(d, cols + heads), fixed(cols + heads), w, fixed(cols), theta, steps, fixed(heads, 1.0), weight(wide, d), fixed(d),
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
            x, _ = ops.resonator_selective_layer(x, p)
        return ops.resonator_linear(x, self.head)

    @torch.no_grad()
    def prefill(self, tokens, lengths=None):
        """Logits [B, L, vocab] of a prompt, and every layer's state after it."""
        x, states = self.emb[tokens], []
        for p in self.damped():
            x, s = ops.resonator_selective_layer_fwd(x, p, lengths=lengths, return_state=True)
            states.append(s)
        return ops.resonator_linear_fwd(x, self.head), states

    @torch.no_grad()
    def step(self, tokens, states, layers):
        """Logits [B, vocab] after one more token of every sequence; the states are advanced in place.  ``layers``: what
        damped() returned, which a decoding loop computes once."""
        x = self.emb[tokens]
        for p, s in zip(layers, states):
            x = ops.resonator_selective_layer_step(x, p, s)
        return ops.resonator_linear_fwd(x, self.head)


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=300)
    ap.add_argument("--dim", type=int, default=256)
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--vocab", type=int, default=32)
    ap.add_argument("--rules", type=int, default=4)
    ap.add_argument("--dtype", choices=base.DTYPES, default="bf16")
    ap.add_argument("--bits", type=int, choices=(8, 32), default=32)
    a = ap.parse_args()
    model = SelectiveLM(a.vocab, a.dim, a.layers, base.DTYPES[a.dtype])
    began = time.perf_counter()
    losses = base.train(model, a.steps, vocab=a.vocab, rules=a.rules, bits=a.bits, report=max(1, a.steps // 10))
    torch.cuda.synchronize()
    print(f"{(time.perf_counter() - began) / a.steps * 1e3:.2f} ms a step; loss {losses[0]:.3f} to {losses[-1]:.3f}")
    t = base.sequences(16, 96, a.vocab, a.rules, torch.Generator().manual_seed(2))
    right = base.generate(model, t[:, :32], 64) == t[:, 32:]
    print(f"64 tokens after a prompt of 32: {right.float().mean().item() * 100:.1f} % are the rule's")


if __name__ == "__main__":
    main()
