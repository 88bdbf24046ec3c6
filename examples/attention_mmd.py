"""An attention block trained on the squared MMD, then run token by token.

    python examples/attention_mmd.py

Training: the block maps noise tokens to points, y = Wo attention(rotary(Wq z),
rotary(Wk z), Wv z) + Ws z, and learns to make them fall like a target cloud.
The loss is gauss_sum_mmd2 of each problem's points against its target; its
gradient with respect to the points is the MMD-flow gradient of Sec. 3 (one
gauss_sum_grad_q), which then goes back through gauss_sum_attention_vjp and the
transposed rotation.  Serving: a causal block with a cache of rotated keys
takes one token per call and must give the rows of the full forward pass.
"""
from __future__ import annotations

import math
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch  # noqa: E402

import paper_2609_04910_gb300 as gs  # noqa: E402


class Block:
    """Weights of one attention block (fp32) and its forward and backward pass."""

    def __init__(self, width, heads, key_heads, head_dim, points, gen):
        self.heads, self.key_heads, self.head_dim = heads, key_heads, head_dim
        sizes = {"q": (width, heads * head_dim), "k": (width, key_heads * head_dim),
                 "v": (width, key_heads * head_dim), "o": (heads * head_dim, points),
                 "s": (width, points)}
        self.w = {n: torch.randn(s, generator=gen, device="cuda") / math.sqrt(s[0])
                  for n, s in sizes.items()}
        # Half of each head turns with the position, in a context stretched by four.
        self.freqs, self.scale = gs.rotary_frequencies(head_dim // 2, scaling="yarn", factor=4.0,
                                                       original_length=1024)
        self.tau = 1.0 / math.sqrt(head_dim)

    def project(self, z, positions):
        """Rotated queries and keys, and values, in bf16."""
        B, N, _ = z.shape
        q, k, v = ((z @ self.w[n]).view(B, N, h, self.head_dim).bfloat16()
                   for n, h in (("q", self.heads), ("k", self.key_heads), ("v", self.key_heads)))
        q, k = gs.gauss_sum_rotary(q, positions, self.freqs, k=k, scale=self.scale)
        return q, k, v

    def forward(self, z, positions, causal=False):
        q, k, v = self.project(z, positions)
        out, lse = gs.gauss_sum_attention(q, k, v, self.tau, causal=causal)
        y = out.flatten(2).float() @ self.w["o"] + z @ self.w["s"]
        return y, (z, positions, q, k, v, out, lse)

    def backward(self, dy, kept):
        """Gradients of the weights for the gradient dy of the points."""
        z, positions, q, k, v, out, lse = kept
        flat = z.flatten(0, 1)
        dy = dy.flatten(0, 1)
        g = (dy @ self.w["o"].T).view_as(out).to(out.dtype)
        dq, dk, dv = gs.gauss_sum_attention_vjp(q, k, v, out, lse, g, self.tau)
        dq, dk = gs.gauss_sum_rotary(dq, positions, self.freqs, k=dk, scale=self.scale,
                                     transpose=True, q_out=dq, k_out=dk)
        grads = {"o": out.flatten(0, 1).flatten(1).float().T @ dy, "s": flat.T @ dy}
        for n, d in (("q", dq), ("k", dk), ("v", dv)):
            grads[n] = flat.T @ d.flatten(0, 1).flatten(1).float()
        return grads


def mmd2_and_gradient(y, target, tau):
    """Squared MMD of each problem and the gradient of their sum in y."""
    B, N, P = y.shape
    both = torch.cat([y, target], 1)
    weights = torch.cat([torch.full((B, N), 1.0 / N, device="cuda"),
                         torch.full((B, N), -1.0 / N, device="cuda")], 1)
    mmd2 = gs.gauss_sum_mmd2(both, weights, tau)
    # d/dy_m of sum_ij w_i Phi_ij w_j is 2 w_m times the q-gradient of s at y_m
    # (gauss_sum_grad_q takes one problem a call).
    grads = [gs.gauss_sum_grad_q(y[b].contiguous(), both[b].contiguous(), weights[b], tau,
                                 want_s=False)[0] for b in range(B)]
    return mmd2, torch.stack(grads) * (2.0 / N)


def train(steps=150, B=4, N=512, width=32, points=4, rate=0.02, seed=0):
    """Mean squared MMD at every step."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    block = Block(width, 8, 2, 64, points, gen)
    first = {n: torch.zeros_like(w) for n, w in block.w.items()}
    second = {n: torch.zeros_like(w) for n, w in block.w.items()}
    positions = torch.arange(N, device="cuda", dtype=torch.int32)
    # A cloud much wider in some directions than in others.
    spread = torch.tensor([3.0, 0.1, 1.0, 0.1], device="cuda").repeat(-(-points // 4))[:points]
    losses = []
    for step in range(1, steps + 1):
        z = torch.randn(B, N, width, generator=gen, device="cuda")
        target = torch.randn(B, N, points, generator=gen, device="cuda") * spread
        y, kept = block.forward(z, positions)
        mmd2, dy = mmd2_and_gradient(y, target, tau=1.0 / points)
        losses.append(mmd2.mean())
        for n, g in block.backward(dy, kept).items():       # Adam
            first[n].lerp_(g, 0.1)
            second[n].lerp_(g * g, 0.01)
            m, s = first[n] / (1 - 0.9 ** step), second[n] / (1 - 0.99 ** step)
            block.w[n] -= rate * m / (s.sqrt() + 1e-8)
    return torch.stack(losses).tolist()


def decode(B=3, N=200, width=32, seed=1):
    """Largest difference between token-by-token outputs and the full causal pass."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    block = Block(width, 8, 2, 64, 4, gen)
    z = torch.randn(B, N, width, generator=gen, device="cuda")
    positions = torch.arange(N, device="cuda", dtype=torch.int32)
    _, (_, _, _, _, _, full, _) = block.forward(z, positions, causal=True)
    keys = torch.full((B, N + 56, block.key_heads, block.head_dim), float("nan"),
                      device="cuda", dtype=torch.bfloat16)      # whatever the cache held before
    values = keys.clone()
    lengths = torch.zeros(B, dtype=torch.int32, device="cuda")
    worst = 0.0
    for t in range(N):
        q, k, v = block.project(z[:, t:t + 1], positions[t:t + 1])
        keys[:, t:t + 1], values[:, t:t + 1] = k, v
        lengths += 1
        out, _ = gs.gauss_sum_attention(q, keys, values, block.tau, causal=True, k_lengths=lengths)
        worst = max(worst, float((out[:, 0].float() - full[:, t].float()).abs().max()))
    return worst


if __name__ == "__main__":
    losses = train()
    for i in range(0, len(losses), 25):
        print(f"step {i:4d}: mean squared MMD {losses[i]:.4f}")
    print(f"last step: mean squared MMD {losses[-1]:.4f}")
    print(f"token by token against the full pass: {decode():.2e}")
    gs.gauss_sum_device_status()
