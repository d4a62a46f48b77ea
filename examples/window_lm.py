"""A small language model whose attention layers run on this library: window heads (norm and
rotation of queries and keys, sliding-window attention with sinks), beside them MoSA heads
if asked for, trained on a made-up language and then continued token by token through
the decoding step's ring caches.

    python examples/window_lm.py                # window heads: trains, then generates
    python examples/window_lm.py --mosa 4       # 4 MoSA heads beside them (trains only: expert
                                                # choice looks at whole sequences)

The language: a sentence repeats its own first ``period`` random tokens, so that each later token
is found ``period`` tokens back, inside the window.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2505_00315_gb300 as mosa  # noqa: E402


class NormRope(torch.autograd.Function):
    """q, k -> normalised and turned q, k (positions 0..T-1)."""

    @staticmethod
    def forward(ctx, q, k, gamma_q, gamma_k):
        ctx.save_for_backward(q, k, gamma_q, gamma_k)
        return mosa.mosa_qk_norm_rope(q, k, gamma_q, gamma_k)

    @staticmethod
    def backward(ctx, dq, dk):
        q, k, gamma_q, gamma_k = ctx.saved_tensors
        g, _ = mosa.mosa_qk_norm_rope_backward(q, k, gamma_q, gamma_k, dq, dk)
        return g["dq"], g["dk"], g["dgamma_q"].to(gamma_q.dtype), g["dgamma_k"].to(gamma_k.dtype)


class WindowAttention(torch.autograd.Function):
    """q, k, v -> attention within a window, the first tokens always visible."""

    @staticmethod
    def forward(ctx, q, k, v, window, sinks):
        O, lse, ws = mosa.mosa_window_forward(q, k, v, window, sinks)
        ctx.save_for_backward(q, k, v, O, lse, ws)
        ctx.window, ctx.sinks = window, sinks
        return O

    @staticmethod
    def backward(ctx, dO):
        q, k, v, O, lse, ws = ctx.saved_tensors
        g = mosa.mosa_window_backward(q, k, v, O, lse, dO, ws, ctx.window, ctx.sinks)
        return g["dq"], g["dk"], g["dv"], None, None


class MosaHeads(torch.autograd.Function):
    """X -> sum of the MoSA heads' outputs (Sec. 2.2), with the first token kept and RoPE."""

    @staticmethod
    def forward(ctx, X, W_r, W_q, W_k, W_v, W_o, k):
        W = [w.to(X.dtype).contiguous() for w in (W_r, W_q, W_k, W_v, W_o)]
        Y, I, r, _, ws = mosa.mosa_forward(X, *W, k, first_token=True, rope=True)
        ctx.save_for_backward(X, *W, I, r, ws)
        return Y.to(X.dtype)

    @staticmethod
    def backward(ctx, dY):
        X, W_r, W_q, W_k, W_v, W_o, I, r, ws = ctx.saved_tensors
        g = mosa.mosa_backward(X, W_r, W_q, W_k, W_v, W_o, I, r, dY.contiguous(), ws, rope=True)
        return (g["dX"].to(X.dtype), g["dW_r"], g["dW_q"], g["dW_k"], g["dW_v"], g["dW_o"], None)


class Layer(torch.nn.Module):
    """Pre-norm attention layer: H window heads on Hkv key / value heads, and n_mosa MoSA heads."""

    def __init__(self, d, H, Hkv, hp, window, sinks, n_mosa=0, k=16):
        super().__init__()
        self.H, self.Hkv, self.hp, self.window, self.sinks, self.k = H, Hkv, hp, window, sinks, k
        self.norm = torch.nn.LayerNorm(d)
        self.qkv = torch.nn.Linear(d, (H + 2 * Hkv) * hp, bias=False)
        self.out = torch.nn.Linear(H * hp, d, bias=False)
        self.gamma_q, self.gamma_k = (torch.nn.Parameter(torch.ones(hp)) for _ in range(2))
        self.mosa = None
        if n_mosa:
            shapes = [(d, n_mosa)] + 3 * [(n_mosa, d, hp)] + [(n_mosa, hp, d)]
            self.mosa = torch.nn.ParameterList(torch.randn(s) * d ** -0.5 for s in shapes)

    def split(self, h):
        """q, k, v: views of one projection, heads side by side."""
        x = self.qkv(h).unflatten(-1, (self.H + 2 * self.Hkv, self.hp))
        return x.split((self.H, self.Hkv, self.Hkv), dim=-2)

    def forward(self, x):
        h = self.norm(x).to(torch.bfloat16)
        q, k, v = self.split(h)
        q, k = NormRope.apply(q, k, self.gamma_q.to(h.dtype), self.gamma_k.to(h.dtype))
        y = self.out(WindowAttention.apply(q, k, v, self.window, self.sinks).flatten(-2))
        if self.mosa is not None:
            y = y + MosaHeads.apply(h, *self.mosa, self.k)
        return x + y

    def caches(self, B, device):
        """Ring caches of the sinks and the window's tokens."""
        shape = (B, self.Hkv, self.sinks + self.window, self.hp)
        return [torch.empty(shape, device=device, dtype=torch.bfloat16).transpose(1, 2) for _ in range(2)]

    def step(self, x, cache, lens, state):
        """One new token of each sequence, x [B, d]; lens counts it."""
        h = self.norm(x).to(torch.bfloat16)
        q, k, v = self.split(h)
        O, state["ws"] = mosa.mosa_window_decode(
            q, k, v, *cache, lens, self.window, self.sinks, gamma_q=self.gamma_q.to(h.dtype),
            gamma_k=self.gamma_k.to(h.dtype), workspace=state.get("ws"))
        return x + self.out(O.flatten(-2))


class Model(torch.nn.Module):
    def __init__(self, vocab, d=256, layers=2, H=4, Hkv=2, hp=64, window=48, sinks=2, n_mosa=0):
        super().__init__()
        self.emb = torch.nn.Embedding(vocab, d)
        self.layers = torch.nn.ModuleList(Layer(d, H, Hkv, hp, window, sinks, n_mosa)
                                          for _ in range(layers))
        self.head = torch.nn.Linear(d, vocab, bias=False)

    def forward(self, tokens):
        x = self.emb(tokens)
        for layer in self.layers:
            x = layer(x)
        return self.head(x)

    @torch.no_grad()
    def generate(self, prompt, n):
        """prompt [B, P] and n tokens more, all of them one at a time through the caches."""
        B, P = prompt.shape
        caches = [layer.caches(B, prompt.device) for layer in self.layers]
        states = [{} for _ in self.layers]
        lens = torch.zeros(B, device=prompt.device, dtype=torch.int32)
        out, token = [prompt], prompt[:, 0]
        for t in range(P + n - 1):
            lens += 1
            x = self.emb(token)
            for layer, cache, state in zip(self.layers, caches, states):
                x = layer.step(x, cache, lens, state)
            token = prompt[:, t + 1] if t + 1 < P else self.head(x).argmax(-1)
            if t + 1 >= P:
                out.append(token[:, None])
        return torch.cat(out, 1)


def sentences(B, T, period, vocab, gen):
    x = torch.randint(0, vocab, (B, period), generator=gen, device="cuda")
    return x.repeat(1, T // period + 1)[:, :T]


def main(steps=150, n_mosa=0, seed=0, T=160, period=24, vocab=64, quiet=False):
    """Trains; returns the first and the last loss, and where there are no MoSA heads the share of
    generated tokens that are right and the model's largest difference between its two ways of running."""
    torch.manual_seed(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    model = Model(vocab, n_mosa=n_mosa).cuda()
    opt = torch.optim.Adam(model.parameters(), lr=2e-3)
    losses = []
    for i in range(steps):
        x = sentences(32, T + 1, period, vocab, gen)
        with torch.autocast("cuda", dtype=torch.bfloat16):
            logits = model(x[:, :-1])
        loss = torch.nn.functional.cross_entropy(logits[:, period:].float().flatten(0, 1),
                                                 x[:, period + 1:].flatten())
        opt.zero_grad()
        loss.backward()
        opt.step()
        losses.append(float(loss.detach()))
        if not quiet and (i % 25 == 0 or i == steps - 1):
            print(f"step {i:4d}  loss {losses[-1]:.4f}")
    if n_mosa:
        return losses[0], losses[-1], None, None
    x = sentences(8, T, period, vocab, gen)
    with torch.autocast("cuda", dtype=torch.bfloat16):
        got = model.generate(x[:, :2 * period], T - 2 * period)
        right = float((got[:, 2 * period:] == x[:, 2 * period:]).float().mean())
        # the whole text at once and token by token: the same logits
        caches = [layer.caches(8, x.device) for layer in model.layers]
        states, lens, far = [{} for _ in model.layers], torch.zeros(8, device="cuda", dtype=torch.int32), 0.0
        with torch.no_grad():
            whole = model(x).float()
            for t in range(T):
                lens += 1
                h = model.emb(x[:, t])
                for layer, cache, state in zip(model.layers, caches, states):
                    h = layer.step(h, cache, lens, state)
                far = max(far, float((model.head(h).float() - whole[:, t]).norm() / whole[:, t].norm()))
    if not quiet:
        print(f"generated tokens that are right: {right:.3f}; whole text against token by token: {far:.4f}")
    return losses[0], losses[-1], right, far


if __name__ == "__main__":
    a = argparse.ArgumentParser()
    a.add_argument("--steps", type=int, default=150)
    a.add_argument("--mosa", type=int, default=0)
    a = a.parse_args()
    main(a.steps, a.mosa)
