"""A token-mixing layer on the gated delta rule, trained, prefilled and run token by token.

  python examples/gated_delta_layer.py

The layer: one projection to queries, keys, values and two gates per head; norm of queries and keys to unit length with the position
rotation (qk_norm_rope); the gated delta rule (gated_delta, gated_delta_decode_step); a projection back.  Training is associative
recall: pairs of tokens (key, value) are shown, then the keys again, and the layer has to give the values.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2605_11196_amd as vla  # noqa: E402


class GatedDeltaLayer(torch.nn.Module):
    def __init__(self, width, heads, key_heads, d, places=4096, dtype=torch.bfloat16):
        super().__init__()
        self.heads, self.key_heads, self.d = heads, key_heads, d
        self.qkv = torch.nn.Linear(width, (2 * key_heads + heads) * d, bias=False, dtype=dtype)
        self.gates = torch.nn.Linear(width, 2 * heads, dtype=torch.float32)
        self.out = torch.nn.Linear(heads * d, width, bias=False, dtype=dtype)
        self.q_weight = torch.nn.Parameter(torch.ones(d, dtype=dtype))
        angle = torch.arange(places).unsqueeze(1) * 10000.0 ** (-torch.arange(d // 4) * 4.0 / d)   # the first half of a head is rotated
        self.register_buffer("cos", angle.cos())
        self.register_buffer("sin", angle.sin())
        torch.nn.init.constant_(self.gates.bias[heads:], -4.0)   # decays near one to begin with

    def mixed(self, x, **where):
        """Queries, keys, values and gates of tokens x [B,T,width] at their positions, heads before tokens."""
        B, T, _ = x.shape
        rows = self.qkv(x).view(B, T, -1, self.d).transpose(1, 2)
        q, k, v = rows.split((self.key_heads, self.key_heads, self.heads), 1)     # views: read as they are
        q, k = vla.qk_norm_rope(q, k, self.q_weight, None, self.cos, self.sin, norm="l2", **where)
        beta, g = self.gates(x.float()).transpose(1, 2).split(self.heads, 1)
        return q, k, v, -torch.nn.functional.softplus(g), torch.sigmoid(beta)

    def forward(self, x, state=None, lengths=None):
        o, state = vla.gated_delta(*self.mixed(x), state, lengths=lengths)
        return self.out(o.transpose(1, 2).flatten(2)), state

    @torch.no_grad()
    def step(self, x, state, positions):
        """One token of each sequence: x [B,width], positions int32 [B]; the state is updated in place."""
        q, k, v, g, beta = self.mixed(x.unsqueeze(1), positions=positions.unsqueeze(1))
        one = lambda t: t[:, :, 0]
        o = vla.gated_delta_decode_step(one(q), one(k), one(v), one(g), one(beta), state)
        return self.out(o.flatten(1))


def recall_batch(gen, batch, pairs, width, keys, device):
    """Tokens [B, 2 pairs, width]: a key in the first half of a token and its value in the second, then the keys in another order; and
    what belongs to them."""
    key = keys[torch.rand((batch, keys.shape[0]), generator=gen, device=device).argsort(1)[:, :pairs]]
    value = torch.randn((batch, pairs, width // 2), generator=gen, device=device)
    order = torch.rand((batch, pairs), generator=gen, device=device).argsort(1).unsqueeze(-1)
    pick = lambda x: x.gather(1, order.expand_as(x))
    shown = torch.cat((key, value), -1)
    asked = torch.cat((pick(key), torch.zeros_like(value)), -1)
    return torch.cat((shown, asked), 1), pick(value)


def main(steps=300, batch=64, pairs=24, width=128, device="cuda"):
    torch.manual_seed(0)
    gen = torch.Generator(device=device)
    gen.manual_seed(1)
    keys = torch.randn((256, width // 2), generator=gen, device=device)
    layer = GatedDeltaLayer(width, heads=4, key_heads=2, d=64).to(device)
    optimiser = torch.optim.AdamW(layer.parameters(), lr=3e-3, weight_decay=0.0)
    first = last = None
    for i in range(steps):
        x, want = recall_batch(gen, batch, pairs, width, keys, device)
        y, _ = layer(x.bfloat16())
        loss = (y[:, pairs:, :width // 2].float() - want).square().mean()
        optimiser.zero_grad()
        loss.backward()
        optimiser.step()
        last = loss.detach()
        first = last if first is None else first
        if i % 100 == 0 or i + 1 == steps:
            print(f"step {i}: recall error {last.item():.4f}", flush=True)
    # the same sequence whole, and as a prompt followed by single tokens on its state
    with torch.no_grad():
        x = recall_batch(gen, 4, pairs, width, keys, device)[0].bfloat16()
        whole, state = layer(x)
        y, running = layer(x[:, :pairs])
        rest = []
        for t in range(pairs, 2 * pairs):
            rest.append(layer.step(x[:, t], running, torch.full((4,), t, device=device, dtype=torch.int32)))
        off = (torch.cat((y, torch.stack(rest, 1)), 1).float() - whole.float()).abs().max() / whole.float().abs().max()
        off_state = (running - state).abs().max() / state.abs().max()
    print(f"prompt and single tokens against the whole sequence: outputs {off.item():.1e}, state {off_state.item():.1e} of the largest")
    return first.item(), last.item(), off.item(), off_state.item()


if __name__ == "__main__":
    main()
