"""A small hybrid language model: layers of second-order linear attention and
of the selective state space scan, trained for a few steps, then served from a
prompt token by token.

    python examples/hybrid.py [--steps 60] [--tokens 512]

Both layers project a token once, run the short convolution over the
projection, and mix:
  attention  q, k, v -> norm and rotation of q and k -> second-order attention
  scan       x, B, C, dt -> selective state space scan
Training runs whole sequences through the differentiable operators.  Serving
keeps, for each layer, the last inputs of its convolution and the state of its
mixer: hla.conv_prefill, hla.prefill / hla.ssm_prefill over the prompt, then
hla.conv_step, hla.step / hla.ssm_step for every new token.
"""
import argparse
import math
import os
import sys

import torch
import torch.nn.functional as F
from torch import nn

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2510_27258_amd as hla  # noqa: E402


def rms(x):
    return F.rms_norm(x.float(), x.shape[-1:]).to(x.dtype)


class Attention(nn.Module):
    """Second-order attention over H heads of 64."""

    def __init__(self, width, H, positions, taps=4):
        super().__init__()
        self.H, self.d = H, 64
        self.proj = nn.Linear(width, 3 * H * 64, bias=False)
        self.conv = nn.Parameter(torch.randn(3 * H * 64, taps) * taps ** -0.5)
        # rows of unit length, as the attention's sums want them
        self.qw, self.kw = (nn.Parameter(torch.full((64,), 64 ** -0.5)) for _ in range(2))
        self.out = nn.Linear(H * 64, width, bias=False)
        angle = torch.arange(positions)[:, None] * 10000.0 ** (-torch.arange(0, 64, 2).double() / 64)
        # no buffers: they stay in fp32 when the model does not
        self.tables = angle.cos().float(), angle.sin().float()

    def _apply(self, fn):
        super()._apply(fn)
        self.tables = tuple(t.to(self.proj.weight.device) for t in self.tables)
        return self

    def start(self, B):
        w = self.proj.weight
        return (torch.zeros(B, self.conv.shape[1] - 1, self.conv.shape[0], dtype=w.dtype, device=w.device),
                hla.State(B, self.H, 64, 64, dtype=w.dtype, device=w.device))

    def split(self, qkv, positions):
        q, k, v = qkv.unflatten(-1, (3, self.H, 64)).unbind(2)
        q, k = hla.qk_norm_rope(q, k, self.qw, self.kw, *self.tables, positions)
        return q, k, v.transpose(1, 2).contiguous()

    def join(self, o, like):
        return self.out(rms(o.transpose(1, 2)).flatten(2).to(like.dtype))

    def forward(self, x, positions):
        return self.join(hla.hla2_attention(*self.split(hla.short_conv(self.proj(x), self.conv), positions)), x)

    def prompt(self, x, positions, kept):
        qkv = hla.conv_prefill(kept[0], self.proj(x), self.conv)
        return self.join(hla.prefill(kept[1], *self.split(qkv, positions), 64), x)

    def token(self, x, positions, kept):
        qkv = hla.conv_step(kept[0], self.proj(x)[:, 0], self.conv)[:, None]
        q, k, v = (t[:, :, 0] for t in self.split(qkv, positions))
        return self.join(hla.step(kept[1], q.contiguous(), k.contiguous(), v.contiguous())[:, :, None], x)


class Scan(nn.Module):
    """Selective state space scan over H heads of 64 with states of 64 x 64."""

    def __init__(self, width, H, taps=4):
        super().__init__()
        self.H = H
        self.proj = nn.Linear(width, H * 64 + 128 + H, bias=False)
        self.conv = nn.Parameter(torch.randn(H * 64 + 128, taps) * taps ** -0.5)
        self.bias = nn.Parameter(torch.zeros(H * 64 + 128))
        self.A = nn.Parameter(torch.log(torch.arange(1, H + 1).float()))
        self.D = nn.Parameter(torch.ones(H))
        self.dt_bias = nn.Parameter(torch.full((H,), math.log(math.expm1(0.02))))
        self.out = nn.Linear(H * 64, width, bias=False)

    def start(self, B):
        w = self.proj.weight
        return (torch.zeros(B, self.conv.shape[1] - 1, self.conv.shape[0], dtype=w.dtype, device=w.device),
                torch.zeros(B, self.H, 64, 64, device=w.device))

    def split(self, xbc, dt):
        """x, dt, A, B, C, D, dt_bias as the scan takes them: slices of the convolution's output."""
        wide = self.H * 64
        return (xbc[..., :wide].unflatten(-1, (self.H, 64)), dt, -self.A.float().exp(),
                xbc[..., wide:wide + 64].unflatten(-1, (1, 64)), xbc[..., wide + 64:].unflatten(-1, (1, 64)),
                self.D.float(), self.dt_bias.float())

    def join(self, y):
        return self.out(rms(y).flatten(2))

    def project(self, x):
        return self.proj(x).split([self.H * 64 + 128, self.H], -1)

    def forward(self, x, positions):
        xbc, dt = self.project(x)
        return self.join(hla.ssm_scan(*self.split(hla.short_conv(xbc, self.conv, self.bias), dt)))

    def prompt(self, x, positions, kept):
        xbc, dt = self.project(x)
        return self.join(hla.ssm_prefill(kept[1], *self.split(hla.conv_prefill(kept[0], xbc, self.conv, self.bias), dt)))

    def token(self, x, positions, kept):
        xbc, dt = (t[:, 0] for t in self.project(x))
        y = hla.ssm_step(kept[1], *self.split(hla.conv_step(kept[0], xbc, self.conv, self.bias), dt))
        return self.join(y[:, None])


class Hybrid(nn.Module):
    def __init__(self, vocab=17, width=256, pairs=1, H=4, positions=4096):
        super().__init__()
        self.embed = nn.Embedding(vocab, width)
        self.mixers = nn.ModuleList(m for _ in range(pairs) for m in (Scan(width, H), Attention(width, H, positions)))
        self.head = nn.Linear(width, vocab, bias=False)

    def start(self, B):
        return [m.start(B) for m in self.mixers]

    def forward(self, ids, first=0, kept=None, how="forward"):
        """Logits of ids [B, n] at positions first ...; how: "forward" (training), "prompt" or "token" (with kept)."""
        B, n = ids.shape
        positions = torch.arange(first, first + n, device=ids.device)
        x = self.embed(ids)
        for i, m in enumerate(self.mixers):
            x = x + getattr(m, how)(rms(x), positions, *(() if kept is None else (kept[i],)))
        return self.head(rms(x)).float()


def sequences(B, n, vocab, generator):
    """Every token the sum of the two before it: what the convolution can see and the mixers must not lose."""
    ids = torch.randint(0, vocab, (B, 2), generator=generator, device=generator.device)
    for _ in range(n - 2):
        ids = torch.cat([ids, (ids[:, -1:] + ids[:, -2:-1]) % vocab], 1)
    return ids[:, :n]


def train(model, steps, B=8, n=512, seed=0, lr=3e-3, say=print):
    """Adam on copies in fp32 of the bf16 parameters; the losses."""
    g = torch.Generator("cuda").manual_seed(seed)
    params = list(model.parameters())
    master = [p.detach().float().clone() for p in params]
    optimizer = torch.optim.Adam(master, lr=lr)
    losses = []
    for step in range(steps):
        ids = sequences(B, n + 1, model.embed.num_embeddings, g)
        loss = F.cross_entropy(model(ids[:, :-1]).flatten(0, 1), ids[:, 1:].flatten())
        for p in params:
            p.grad = None
        loss.backward()
        for m, p in zip(master, params):
            m.grad = p.grad.float()
        torch.nn.utils.clip_grad_norm_(master, 1.0)
        optimizer.step()
        with torch.no_grad():
            for m, p in zip(master, params):
                p.copy_(m)
        losses.append(loss.item())
        if say and (step % 5 == 0 or step == steps - 1):
            say(f"step {step}: loss {losses[-1]:.3f}", flush=True)
    return losses


@torch.no_grad()
def generate(model, ids, count):
    """Greedy continuation of the prompt ids [B, n]: (ids [B, n + count], logits of the new tokens' positions)."""
    kept = model.start(ids.shape[0])
    logits = [model(ids, 0, kept, "prompt")[:, -1:]]
    for i in range(count):
        ids = torch.cat([ids, logits[-1].argmax(-1)], 1)
        if i + 1 < count:
            logits.append(model(ids[:, -1:], ids.shape[1] - 1, kept, "token"))
    return ids, torch.cat(logits, 1)


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--tokens", type=int, default=512)
    a = ap.parse_args()
    torch.manual_seed(0)
    model = Hybrid().cuda().bfloat16()
    train(model, a.steps, n=a.tokens)
    g = torch.Generator("cuda").manual_seed(99)
    ids = sequences(2, 96, model.embed.num_embeddings, g)
    out, logits = generate(model, ids, 32)
    whole = model(out[:, :-1])[:, -logits.shape[1]:]
    right = (out[:, 96:] == (out[:, 95:-1] + out[:, 94:-2]) % model.embed.num_embeddings).float().mean()
    print(f"32 new tokens: {100 * right:.0f} % by the rule; logits of the steps against the whole sequence's: {(logits - whole).abs().max():.3g} of "
          f"{whole.abs().max():.3g}")


if __name__ == "__main__":
    main()
