"""Token-mixing layers on the selective state space scan, trained, prefilled and run token by token.

  python examples/selective_scan_layer.py

A layer: a projection to channels and their gate; a short causal convolution (causal_conv); projections to the scan's steps, inputs and
read-outs; the scan with its gate (selective_scan); a projection back.  Between layers the output's norm, its scale, the residual and the next layer's
norm are one call (residual_norm).  Training is selective copying: a few marked tokens lie among others, and the model has to give their
values in order when it is asked for them.
"""
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2605_11196_amd as vla  # noqa: E402


class SelectiveLayer(torch.nn.Module):
    def __init__(self, width, channels, states=16, taps=4, dtype=torch.bfloat16):
        super().__init__()
        self.channels, self.states, self.taps = channels, states, taps
        linear = lambda i, o: torch.nn.Linear(i, o, bias=False, dtype=dtype)
        self.rows, self.delta, self.shared, self.out = linear(width, 2 * channels), linear(channels, channels), linear(channels, 2 * states), linear(channels, width)
        self.conv = torch.nn.Parameter((torch.rand(channels, taps) - 0.5).to(dtype))
        self.conv_bias = torch.nn.Parameter(torch.zeros(channels, dtype=dtype))
        self.log_A = torch.nn.Parameter(torch.arange(1, states + 1).float().log().repeat(channels, 1))
        self.D = torch.nn.Parameter(torch.ones(channels))
        self.delta_bias = torch.nn.Parameter(torch.rand(channels) * 4.6 - 6.9)      # steps from 0.001 to 0.1 to begin with

    def empty(self, batch):
        """The window and the state of sequences that have not begun."""
        like = self.conv
        return like.new_zeros(batch, self.taps - 1, self.channels), torch.zeros(batch, self.channels, self.states, device=like.device)

    def forward(self, x, window, state, lengths=None):
        """x [B,T,width]: the layer's output, and the window and the state behind it."""
        x, z = self.rows(x).split(self.channels, -1)                          # views: read as they are
        x, window = vla.causal_conv(x, self.conv, self.conv_bias, window, lengths=lengths)
        B, C = self.shared(x).split(self.states, -1)
        y, state = vla.selective_scan(x, self.delta(x), -self.log_A.exp(), B, C, self.D, z, state, delta_bias=self.delta_bias, lengths=lengths)
        return self.out(y), window, state

    @torch.no_grad()
    def step(self, x, window, state):
        """One token of each sequence, x [B,width]; window and state move on in place."""
        x, z = self.rows(x).split(self.channels, -1)
        x = vla.causal_conv_step(x, self.conv, window, self.conv_bias)
        B, C = self.shared(x).split(self.states, -1)
        y = vla.selective_scan_step(x, self.delta(x), -self.log_A.exp(), B, C, state, self.D, z, delta_bias=self.delta_bias)
        return self.out(y)


class SelectiveModel(torch.nn.Module):
    def __init__(self, width=64, channels=128, layers=2, dtype=torch.bfloat16):
        super().__init__()
        self.layers = torch.nn.ModuleList(SelectiveLayer(width, channels, dtype=dtype) for _ in range(layers))
        self.norms = torch.nn.Parameter(torch.ones(layers + 1, width))            # before each layer, and the last one
        self.posts = torch.nn.Parameter(torch.ones(layers, width))                # of each layer's output
        self.scales = torch.nn.Parameter(torch.full((layers, width), 0.5))
        self.dtype = dtype

    def empty(self, batch):
        return [layer.empty(batch) for layer in self.layers]

    def run(self, x, mix):
        """x [B,T,width] float32, the residual stream; mix(i, rows): what layer i makes of its normed rows."""
        h = vla.residual_norm(x, None, self.norms[0])[1].to(self.dtype)
        for i in range(len(self.layers)):
            x, h = vla.residual_norm(x, mix(i, h), self.norms[i + 1], post_weight=self.posts[i], scale=self.scales[i])
        return h.float()

    def forward(self, x, carried=None, lengths=None):
        carried = self.empty(x.shape[0]) if carried is None else carried
        behind = []

        def mix(i, rows):
            out, *state = self.layers[i](rows, *carried[i], lengths)
            behind.append(state)
            return out

        return self.run(x, mix), behind

    @torch.no_grad()
    def step(self, x, carried):
        """One token of each sequence, x [B,width]; what is carried moves on in place."""
        return self.run(x.unsqueeze(1), lambda i, rows: self.layers[i].step(rows[:, 0], *carried[i]).unsqueeze(1))[:, 0]


def copying_batch(gen, batch, tokens, marked, width, device):
    """Tokens [B, tokens + marked, width] whose first column marks some of them and whose second asks, and the marked ones' other columns in order."""
    x = torch.randn((batch, tokens + marked, width), generator=gen, device=device)
    place = torch.rand((batch, tokens), generator=gen, device=device).argsort(1)[:, :marked].sort(1)[0]
    x[:, :, :2] = 0.0
    x[:, :, 0].scatter_(1, place, 4.0)
    want = x.gather(1, place.unsqueeze(-1).expand(-1, -1, width))[:, :, 2:]
    x[:, tokens:, 2:] = 0.0
    x[:, tokens:, 1] = 4.0
    return x, want


def main(steps=500, batch=64, tokens=24, marked=2, width=64, device="cuda"):
    torch.manual_seed(0)
    gen = torch.Generator(device=device)
    gen.manual_seed(1)
    model = SelectiveModel(width).to(device)
    optimiser = torch.optim.AdamW(model.parameters(), lr=3e-3, weight_decay=0.0)
    first = last = None
    for i in range(steps):
        x, want = copying_batch(gen, batch, tokens, marked, width, device)
        loss = (model(x)[0][:, tokens:, 2:] - want).square().mean()
        optimiser.zero_grad()
        loss.backward()
        optimiser.step()
        last = loss.detach()
        first = last if first is None else first
        if i % 100 == 0 or i + 1 == steps:
            print(f"step {i}: copying error {last.item():.4f}", flush=True)
    # the same sequence whole, and as a prompt followed by single tokens on what it carries
    with torch.no_grad():
        x = copying_batch(gen, 4, tokens, marked, width, device)[0]
        whole, behind = model(x)
        y, carried = model(x[:, :tokens])
        rest = [model.step(x[:, t], carried) for t in range(tokens, tokens + marked)]
        off = (torch.cat((y, torch.stack(rest, 1)), 1) - whole).abs().max() / whole.abs().max()
        off_state = max((a[1] - b[1]).abs().max() / b[1].abs().max() for a, b in zip(carried, behind))
    print(f"prompt and single tokens against the whole sequence: outputs {off.item():.1e}, states {off_state.item():.1e} of the largest")
    return first.item(), last.item(), off.item(), off_state.item()


if __name__ == "__main__":
    main()
