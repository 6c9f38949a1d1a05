"""A token mixer built from the library's operators, used as a model uses it:

    in projection -> causal convolution -> step size, B and C projections -> selective scan, gated
                  -> group norm of the heads -> out projection

for prompts (forward), training (backward) and decoding (step, one token at a time over a cache).

    python examples/selective_mixer.py        # a few training steps, then a prompt continued token by token
"""

import math
import os
import sys

import torch
from torch import nn

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2506_04761_amd as ll  # noqa: E402


class SelectiveMixer(nn.Module):
    """A mixer of `d_model` channels, `expand` times as many inside, `n` states a channel and `taps` taps.  Projections
    have the dtype `dtype`; the operators' own parameters are float32."""

    def __init__(self, d_model, expand=2, n=16, heads=8, taps=4, dtype=torch.bfloat16, device="cuda"):
        super().__init__()
        d = self.d = expand * d_model
        self.n, self.heads, self.taps, self.rank = n, heads, taps, max(1, d_model // 16)
        kw = {"bias": False, "dtype": dtype, "device": device}
        self.into = nn.Linear(d_model, 2 * d, **kw)             # input and gate
        self.select = nn.Linear(d, self.rank + 2 * n, **kw)     # low-rank step size, B, C
        self.step_size = nn.Linear(self.rank, d, **kw)
        self.out = nn.Linear(d, d_model, **kw)
        f = {"dtype": torch.float32, "device": device}
        self.conv_weight = nn.Parameter(torch.randn(d, taps, **f) / math.sqrt(taps))
        self.conv_bias = nn.Parameter(torch.zeros(d, **f))
        self.log_rate = nn.Parameter(torch.log(torch.arange(1, n + 1, **f)).repeat(d, 1))
        step = torch.exp(torch.rand(d, **f) * math.log(100.0) + math.log(0.001))
        self.dt_bias = nn.Parameter(step + torch.log(-torch.expm1(-step)))
        self.skip = nn.Parameter(torch.ones(d, **f))
        self.norm_weight = nn.Parameter(torch.ones(d, **f))
        self.norm_bias = nn.Parameter(torch.zeros(d, **f))

    def _select(self, u):
        p = self.select(u)
        return self.step_size(p[..., :self.rank]), p[..., self.rank:self.rank + self.n], p[..., self.rank + self.n:]

    def _normed(self, y):
        """The heads of every token, normalised by themselves."""
        flat = ll.group_norm(y.reshape(-1, 1, self.d), self.heads, self.norm_weight, self.norm_bias, act=ll.LL_ACT_NONE)
        return self.out(flat.view(y.shape))

    def forward(self, h, lengths=None, cache=None):
        """h [B, T, d_model]; `lengths` int32 [B] for sequences that end early.  With a cache (see new_cache) the
        sequences continue it, and it is brought up to their ends; gradients end at it."""
        x, z = self.into(h).chunk(2, -1)
        if cache is None:
            u = ll.causal_conv(x, self.conv_weight, self.conv_bias, lengths=lengths)
        elif torch.is_grad_enabled():
            # the backward reads the states that it started from, which the cache does not keep
            u, end = ll.causal_conv(x, self.conv_weight, self.conv_bias, initial_state=cache["conv"].clone(),
                                    lengths=lengths, return_final_state=True)
            cache["conv"].copy_(end.detach())
        else:
            u = ll.ll_causal_conv_fwd(x, self.conv_weight, self.conv_bias, initial_state=cache["conv"],
                                      final_state=cache["conv"], lengths=lengths)
        dt, B, C = self._select(u)
        a = (u, dt, -torch.exp(self.log_rate), B, C, self.skip, z, self.dt_bias)
        if cache is None:
            y = ll.selective_scan(*a, lengths=lengths)
        elif torch.is_grad_enabled():
            y, end = ll.selective_scan(*a, initial_state=cache["scan"].clone(), lengths=lengths, return_final_state=True)
            cache["scan"].copy_(end.detach())
        else:
            y = ll.ll_selective_scan_fwd(*a, initial_state=cache["scan"], final_state=cache["scan"], lengths=lengths)
        return self._normed(y)

    def new_cache(self, batch):
        w = self.into.weight
        return {"conv": w.new_zeros((batch, self.taps - 1, self.d)),
                "scan": torch.zeros((batch, self.d, self.n), dtype=torch.float32, device=w.device)}

    @torch.no_grad()
    def step(self, h, cache):
        """One token h [B, d_model]; the cache is advanced in place."""
        x, z = self.into(h).chunk(2, -1)
        u = ll.ll_causal_conv_step(x, self.conv_weight, self.conv_bias, cache["conv"])
        dt, B, C = self._select(u)
        y = ll.ll_selective_scan_step(u, dt, -torch.exp(self.log_rate), B, C, cache["scan"], self.skip, z, self.dt_bias)
        return self._normed(y)


def train(mixer, steps=20, batch=4, tokens=200, seed=0):
    """Trains the mixer to repeat the token before; returns the losses."""
    g = torch.Generator("cuda").manual_seed(seed)
    opt = torch.optim.Adam(mixer.parameters(), lr=3e-3)
    d = mixer.into.in_features
    losses = []
    for _ in range(steps):
        h = torch.randn((batch, tokens, d), generator=g, device="cuda").to(mixer.into.weight.dtype)
        loss = (mixer(h)[:, 1:].float() - h[:, :-1].float()).square().mean()
        opt.zero_grad()
        loss.backward()
        opt.step()
        losses.append(loss.item())
    return losses


@torch.no_grad()
def decode_error(mixer, prompts=(37, 20), tokens=16, seed=1):
    """A prompt of each length continued token by token, against one pass over the whole: max difference / max."""
    g = torch.Generator("cuda").manual_seed(seed)
    batch, longest = len(prompts), max(prompts)
    h = torch.randn((batch, longest + tokens, mixer.into.in_features), generator=g, device="cuda").to(mixer.into.weight.dtype)
    n = torch.tensor(prompts, dtype=torch.int32, device="cuda")
    cache = mixer.new_cache(batch)
    mixer(h[:, :longest], lengths=n, cache=cache)
    got = [mixer.step(torch.stack([h[b, p + t] for b, p in enumerate(prompts)]), cache) for t in range(tokens)]
    whole = mixer(h, lengths=n + tokens)
    want = torch.stack([whole[b, p:p + tokens] for b, p in enumerate(prompts)])
    return ((torch.stack(got, 1) - want).abs().max() / want.abs().max()).item()


def main():
    torch.manual_seed(0)
    mixer = SelectiveMixer(256)
    losses = train(mixer)
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f} in {len(losses)} steps")
    print(f"decoding against one pass: {decode_error(mixer):.2e} of the largest output")


if __name__ == "__main__":
    main()
