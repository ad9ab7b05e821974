"""A token mixer of a linear-attention model on the library's operators: rotary
positions on queries and keys, the gated delta rule over the sequence, and its
recurrent form on the states that a prompt leaves.

    python examples/token_mixer.py

trains the mixer for some steps to keep a moving average of its inputs, then reads a prompt and goes
on token by token, and checks that this gives what the whole sequence gives.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_2308_15152_amd as emu  # noqa: E402


class Rotary(torch.autograd.Function):
    """q and k turned by their positions; a rotation's gradient turns back."""

    @staticmethod
    def forward(ctx, q, k, cos, sin, positions):
        ctx.save_for_backward(cos, sin, positions)
        return emu.rotary_emu(q, k, cos, sin, positions=positions)

    @staticmethod
    def backward(ctx, dq, dk):
        cos, sin, positions = ctx.saved_tensors
        dq, dk = emu.rotary_emu(dq.contiguous(), dk.contiguous(), cos, sin, positions=positions,
                                inverse=True)
        return dq, dk, None, None, None


class DeltaRule(torch.autograd.Function):
    """(o, final state) of the gated delta rule."""

    @staticmethod
    def forward(ctx, q, k, v, g, beta, state):
        ctx.save_for_backward(q, k, v, g, beta, state)
        return emu.delta_emu_forward(q, k, v, g, beta, state)

    @staticmethod
    def backward(ctx, do, dstate):
        q, k, v, g, beta, state = ctx.saved_tensors
        return emu.delta_emu_backward(q, k, v, g, beta, do.contiguous(), state,
                                      dstate.contiguous())


class TokenMixer(torch.nn.Module):
    def __init__(self, width, k_heads, v_heads, k_size, v_size, rot, context, device):
        super().__init__()
        self.k_heads, self.v_heads, self.k_size, self.v_size = k_heads, v_heads, k_size, v_size
        self.parts = [k_heads * k_size, k_heads * k_size, v_heads * v_size, v_heads, v_heads]
        self.into = torch.nn.Linear(width, sum(self.parts), bias=False, device=device)
        self.out = torch.nn.Linear(v_heads * v_size, width, bias=False, device=device)
        # four times the positions that the frequencies were made for
        self.cos, self.sin = emu.rotary_emu_table(4 * context, rot, factor=4.0, original=context,
                                                  ramp=(1.0, 32.0), device=device)

    def empty_state(self, batch):
        return torch.zeros(batch, self.v_heads, self.k_size, self.v_size,
                           device=self.out.weight.device)

    def inputs(self, x, positions):
        q, k, v, g, beta = self.into(x).split(self.parts, dim=-1)
        q, k = q.unflatten(-1, (self.k_heads, -1)), k.unflatten(-1, (self.k_heads, -1))
        q, k = Rotary.apply(q.bfloat16(), k.bfloat16(), self.cos, self.sin, positions)
        q = torch.nn.functional.normalize(q.float(), dim=-1).bfloat16()
        k = torch.nn.functional.normalize(k.float(), dim=-1).bfloat16()
        v = v.unflatten(-1, (self.v_heads, -1)).bfloat16()
        g = -torch.nn.functional.softplus(g.float() - 3.0)
        return q, k, v, g, torch.sigmoid(beta.float())

    def forward(self, x, state, positions):
        """Whole sequences: (output, states after them)."""
        o, state = DeltaRule.apply(*self.inputs(x, positions), state)
        return self.out(o.flatten(2).to(x.dtype)), state

    @torch.no_grad()
    def step(self, x, state, positions):
        """One token (or a few); the states are updated in place."""
        o = emu.delta_emu_step(*self.inputs(x, positions), state)
        return self.out(o.flatten(2).to(x.dtype))


def run(steps=100, batch=4, tokens=200, width=128, device="cuda"):
    """(losses, largest relative differences of outputs and of states between
    the whole sequence and a prompt followed by single tokens)."""
    torch.manual_seed(0)
    mixer = TokenMixer(width, 2, 4, 64, 64, 32, 256, device)
    optimizer = torch.optim.AdamW(mixer.parameters(), lr=3e-3)
    at = torch.arange(tokens, dtype=torch.int32, device=device)
    positions = at.expand(batch, tokens)
    back = (at[:, None] - at).float()
    average = torch.where(back >= 0, 0.4 * 0.8 ** back, 0.0)
    losses = []
    for _ in range(steps):
        x = torch.randn(batch, tokens, width, device=device)
        x[..., -1] = 8.0  # a channel that is always on, for keys that all tokens share
        y, _ = mixer(x, mixer.empty_state(batch), positions)
        wanted = torch.matmul(average.expand(batch, -1, -1), x[..., :16].contiguous())
        loss = (y[..., :16] - wanted).square().mean() / wanted.square().mean()
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        losses.append(float(loss.detach()))

    with torch.no_grad():
        x = torch.randn(batch, tokens, width, device=device)
        whole, last = mixer(x, mixer.empty_state(batch), positions)
        prompt = tokens - 8
        y, state = mixer(x[:, :prompt], mixer.empty_state(batch), positions[:, :prompt].contiguous())
        parts = [y]
        for t in range(prompt, tokens):
            parts.append(mixer.step(x[:, t:t + 1], state, positions[:, t:t + 1].contiguous()))
        off = (torch.cat(parts, 1) - whole).abs().max() / whole.abs().max()
        off_state = (state - last).abs().max() / last.abs().max()
    return losses, float(off), float(off_state)


if __name__ == "__main__":
    losses, off, off_state = run()
    print("loss %.3f -> %.3f" % (losses[0], losses[-1]))
    print("a prompt and single tokens against the whole sequence: outputs %.1e, states %.1e"
          % (off, off_state))
