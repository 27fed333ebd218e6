"""A small language model of gated linear recurrences and gated feed-forward
blocks, trained for a few steps, then served from a prompt token by token.

    python examples/recurrent.py [--steps 60] [--tokens 512]

A block projects a token once, runs the short convolution, the recurrence and
the norm of its outputs with their gate, and adds the result to the residual
stream; then the gated feed-forward part does the same.  Every addition to the
stream and the norms around it are one hla.residual_norm.  Serving keeps, for
each block, the last inputs of its convolution and the state of its
recurrence.  Training and sampling are examples/hybrid.py's.
"""
import argparse
import math
import os
import sys

import torch
from torch import nn

sys.path[:0] = [os.path.dirname(os.path.dirname(os.path.abspath(__file__))), os.path.dirname(os.path.abspath(__file__))]
import paper_2510_27258_amd as hla  # noqa: E402
from hybrid import generate, sequences, train  # noqa: E402


class Recurrence(nn.Module):
    """Projection, short convolution, gated linear recurrence, gated norm, projection."""

    def __init__(self, width, inner, taps=4):
        super().__init__()
        self.inner = inner
        self.proj = nn.Linear(width, 4 * inner, bias=False)
        self.conv = nn.Parameter(torch.randn(inner, taps) * taps ** -0.5)
        # channels that keep 0.9 to 0.999 of themselves a token where their gate is open
        keep = torch.linspace(0.9, 0.999, inner, dtype=torch.float64)
        self.decay = nn.Parameter(torch.log(torch.expm1(-torch.log(keep) / 8)).float())
        self.f_bias, self.g_bias = (nn.Parameter(torch.zeros(inner)) for _ in range(2))
        self.norm = nn.Parameter(torch.ones(64))
        self.out = nn.Linear(inner, width, bias=False)

    def start(self, B):
        w = self.proj.weight
        return (torch.zeros(B, self.conv.shape[1] - 1, self.inner, dtype=w.dtype, device=w.device),
                torch.zeros(B, self.inner, device=w.device))

    def learned(self):
        return self.decay.float(), self.f_bias.float(), self.g_bias.float()

    def join(self, h, z):
        heads = (-1, (self.inner // 64, 64))
        return self.out(hla.gated_norm(h.unflatten(*heads), z.unflatten(*heads), self.norm).flatten(2))

    def forward(self, x):
        u, f, g, z = self.proj(x).split(self.inner, -1)
        return self.join(hla.glr_scan(hla.short_conv(u, self.conv), f, g, *self.learned()), z)

    def prompt(self, x, kept):
        u, f, g, z = self.proj(x).split(self.inner, -1)
        return self.join(hla.glr_prefill(kept[1], hla.conv_prefill(kept[0], u, self.conv), f, g, *self.learned()), z)

    def token(self, x, kept):
        u, f, g, z = (t[:, 0] for t in self.proj(x).split(self.inner, -1))
        h = hla.glr_step(kept[1], hla.conv_step(kept[0], u, self.conv), f, g, *self.learned())
        return self.join(h[:, None], z[:, None])


class FeedForward(nn.Module):
    def __init__(self, width, inner):
        super().__init__()
        self.gate, self.up = (nn.Parameter(torch.randn(inner, width) * width ** -0.5) for _ in range(2))
        self.down = nn.Linear(inner, width, bias=False)

    def forward(self, x):
        return self.down(hla.glu(x, self.gate, self.up))


class Recurrent(nn.Module):
    def __init__(self, vocab=17, width=256, blocks=1, inner=256):
        super().__init__()
        self.embed = nn.Embedding(vocab, width)
        self.first = nn.Parameter(torch.ones(width))
        self.mixers = nn.ModuleList(Recurrence(width, inner) for _ in range(blocks))
        self.mlps = nn.ModuleList(FeedForward(width, 2 * width) for _ in range(blocks))
        # for each of a block's two additions: the norm of what is added, its scale, and the norm of the sum
        self.after, self.scale, self.before = (
            nn.ParameterList(nn.Parameter(torch.full((width,), v)) for _ in range(2 * blocks))
            for v in (1.0, 1 / math.sqrt(2 * blocks), 1.0))
        self.head = nn.Linear(width, vocab, bias=False)

    def start(self, B):
        return [m.start(B) for m in self.mixers]

    def forward(self, ids, first=0, kept=None, how="forward"):
        """Logits of ids [B, n]; how: "forward" (training), "prompt" or "token" (with kept)."""
        x = self.embed(ids)
        u = hla.gated_norm(x[:, :, None], weight=self.first)[:, :, 0]
        stream = x.float()
        for i, (mixer, mlp) in enumerate(zip(self.mixers, self.mlps)):
            for k, part in ((2 * i, lambda v: getattr(mixer, how)(v, *(() if kept is None else (kept[i],)))), (2 * i + 1, mlp)):
                u, stream = hla.residual_norm(stream, part(u), self.before[k], self.after[k], self.scale[k])
        return self.head(u).float()


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--tokens", type=int, default=512)
    a = ap.parse_args()
    torch.manual_seed(0)
    model = Recurrent().cuda().bfloat16()
    train(model, a.steps, n=a.tokens)
    ids = sequences(2, 96, model.embed.num_embeddings, torch.Generator("cuda").manual_seed(99))
    out, logits = generate(model, ids, 32)
    whole = model(out[:, :-1])[:, -logits.shape[1]:]
    right = (out[:, 96:] == (out[:, 95:-1] + out[:, 94:-2]) % model.embed.num_embeddings).float().mean()
    print(f"32 new tokens: {100 * right:.0f} % by the rule; logits of the steps against the whole sequence's: "
          f"{(logits - whole).abs().max():.3g} of {whole.abs().max():.3g}")


if __name__ == "__main__":
    main()
