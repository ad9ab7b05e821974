"""A softmax attention layer on the library's operators: rotary positions, attention over
whole sequences with its gradient, and several continuations of one prompt, whose keys and values
they share.

    python examples/softmax_mixer.py

takes some optimizer steps, then reads a prompt, goes on from it in several ways token by token,
and checks that this gives what the whole sequences give.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import paper_2308_15152_amd as emu  # noqa: E402
from token_mixer import Rotary  # noqa: E402


class Attention(torch.autograd.Function):
    """o of causal attention, of packed sequences if bounds are given."""

    @staticmethod
    def forward(ctx, q, k, v, bounds):
        o, lse = emu.attention_emu_forward(q, k, v, cu_seqlens=bounds)
        ctx.save_for_backward(q, k, v, o, lse, bounds)
        return o

    @staticmethod
    def backward(ctx, do):
        q, k, v, o, lse, bounds = ctx.saved_tensors
        return *emu.attention_emu_backward(q, k, v, o, lse, do, cu_seqlens=bounds), None


class SoftmaxMixer(torch.nn.Module):
    def __init__(self, width, q_heads, k_heads, size, context, device, dtype=torch.bfloat16):
        super().__init__()
        self.q_heads, self.k_heads, self.size, self.dtype = q_heads, k_heads, size, dtype
        self.parts = [q_heads * size, k_heads * size, k_heads * size]
        self.into = torch.nn.Linear(width, sum(self.parts), bias=False, device=device)
        self.out = torch.nn.Linear(q_heads * size, width, bias=False, device=device)
        self.cos, self.sin = emu.rotary_emu_table(context, size, device=device)

    def inputs(self, x, positions):
        q, k, v = (y.unflatten(-1, (-1, self.size)).to(self.dtype)
                   for y in self.into(x).split(self.parts, -1))
        return *Rotary.apply(q, k, self.cos, self.sin, positions), v

    def forward(self, x, positions, bounds=None):
        """Whole sequences (one row of packed ones with bounds)."""
        o = Attention.apply(*self.inputs(x, positions), bounds)
        return self.out(o.flatten(2).to(x.dtype))

    @torch.no_grad()
    def read(self, x, positions):
        """(output, keys, values) of a prompt."""
        q, k, v = self.inputs(x, positions)
        o, _ = emu.attention_emu_forward(q, k, v)
        return self.out(o.flatten(2).to(x.dtype)), k, v

    @torch.no_grad()
    def step(self, x, positions, prompt, caches, lengths):
        """One token of each continuation; its key and value go into the caches."""
        q, k, v = self.inputs(x, positions)
        which = torch.arange(x.shape[0], device=x.device)
        for cache, y in zip(caches, (k, v)):
            cache[which, lengths.long()] = y[:, 0]
        lengths += 1
        o = emu.attention_emu_step(q, *caches, lengths, *prompt)
        return self.out(o.flatten(2).to(x.dtype))


def run(steps=5, batch=3, tokens=150, more=6, width=96, device="cuda"):
    """(losses, largest relative difference between whole sequences and a prompt followed by
    single tokens)."""
    torch.manual_seed(0)
    mixer = SoftmaxMixer(width, 4, 2, 64, 512, device)
    optimizer = torch.optim.AdamW(mixer.parameters(), lr=1e-3)
    positions = torch.arange(tokens + more, dtype=torch.int32, device=device).expand(batch, -1)
    losses = []
    for _ in range(steps):
        x = torch.randn(batch, tokens, width, device=device)
        y = mixer(x, positions[:, :tokens].contiguous())
        loss = (y[:, 1:] - x[:, :-1]).square().mean()
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        losses.append(float(loss.detach()))

    with torch.no_grad():
        x = torch.randn(batch, tokens + more, width, device=device)
        x[:, :tokens] = x[:1, :tokens]
        whole = mixer(x, positions.contiguous())
        parts = [mixer.read(x[:1, :tokens], positions[:1, :tokens].contiguous())]
        prompt, parts = parts[0][1:], [parts[0][0].expand(batch, -1, -1)]
        caches = [torch.empty(batch, more, 2, 64, dtype=mixer.dtype, device=device)
                  for _ in range(2)]
        lengths = torch.zeros(batch, dtype=torch.int32, device=device)
        for t in range(tokens, tokens + more):
            parts.append(mixer.step(x[:, t:t + 1], positions[:, t:t + 1].contiguous(), prompt,
                                    caches, lengths))
        off = (torch.cat(parts, 1) - whole).abs().max() / whole.abs().max()
    return losses, float(off)


if __name__ == "__main__":
    losses, off = run()
    print("loss %.3f -> %.3f" % (losses[0], losses[-1]))
    print("a prompt and single tokens against the whole sequences: %.1e" % off)
