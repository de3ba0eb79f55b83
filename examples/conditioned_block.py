"""The conditioned half of a DiT block on the library's operators.

    python examples/conditioned_block.py [--tokens N] [--prompt T] [--heads H]

runs synthetic tokens through cross attention to a prompt's states and a gated
feed-forward (random weights), forward and backward, and prints the times.  The
block runs

    gated_norm            modulated norm of the residual stream
    (query projection, and keys and values of the prompt in one product)
    cross_attention       the tokens' queries over the prompt's states
    (output projection)
    gated_norm            residual update and the next norm
    gated_ffn             gate and up projections with the activation
    (down projection)
    gated_norm            the last residual update
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2609_36757_gb300 import fastvr as FV  # noqa: E402

BF16 = torch.bfloat16


class Conditioned:
    """Weights and modulation of a block of `heads` heads (kv_heads of them for
    the prompt's keys and values), a prompt of `states` channels and `hidden`
    feed-forward channels."""

    WEIGHTS = ("w_q", "w_kv", "w_o", "w_gate", "w_up", "w_down")

    def __init__(self, heads: int, kv_heads: int, states: int, hidden: int,
                 batch: int = 1, seed: int = 0, head_dim: int = 128,
                 activation: str = "silu"):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
        weight = lambda n, m: (rnd(n, m) * m ** -0.5).to(BF16)
        self.kv_heads, self.d = kv_heads, head_dim
        D = self.dim = heads * head_dim
        self.w_q = weight(D, D)
        self.w_kv = weight(2 * kv_heads * head_dim, states)
        self.w_o = weight(D, D)
        self.w_gate, self.w_up = weight(hidden, D), weight(hidden, D)
        self.w_down = weight(D, hidden)
        # timestep modulation, one vector per batch entry
        self.mod = {n: 0.2 * rnd(batch, 1, D) for n in
                    ("scale", "shift", "gate", "scale2", "shift2", "gate2")}
        self.norm = FV.make_norm_config(pre="layer")
        self.cross = FV.make_cross_config()
        self.ffn = FV.make_ffn_config(activation)

    def prompt(self, states):
        """k, v views of one fused projection of states [B, T, channels]."""
        B, T, _ = states.shape
        kv = (states @ self.w_kv.T).view(B, T, -1, self.d)
        return kv.split(self.kv_heads, 2)

    def forward(self, x, k, v, kv_len=None, keep: bool = False):
        """x [B, L, dim] over the prompt's k and v; the residual stream after
        the block, and with keep what the gradients need."""
        B, L, D = x.shape
        m = self.mod
        _, n1 = FV.gated_norm(self.norm, x, None, scale=m["scale"],
                              shift=m["shift"], want_r=False)
        q = (n1 @ self.w_q.T).view(B, L, -1, self.d)
        got = FV.cross_attention(self.cross, q, k, v, kv_len, want_lse=keep)
        o, lse = got if keep else (got, None)
        y1 = o.view(B, L, D) @ self.w_o.T
        r1, n2 = FV.gated_norm(self.norm, x, y1, m["gate"], m["scale2"],
                               m["shift2"])
        got = FV.gated_ffn(self.ffn, n2, self.w_gate, self.w_up,
                           want_saved=keep)
        h, saved = got if keep else (got, None)
        y2 = h @ self.w_down.T
        r2, _ = FV.gated_norm(self.norm, r1, y2, m["gate2"], want_h=False)
        return (r2, (n1, q, o, lse, y1, r1, n2, h, saved, y2)) if keep else r2


def train_step(block: Conditioned, x, states, dr, kv_len=None):
    """Forward and backward, dr the gradient of the residual stream after the
    block.  Returns (r, gradients by name)."""
    B, L, D = x.shape
    m = block.mod
    k, v = block.prompt(states)
    r2, (n1, q, o, lse, y1, r1, n2, h, saved, y2) = block.forward(
        x, k, v, kv_len, keep=True)
    flat = lambda t: t.flatten(0, 1)
    g = FV.gated_norm_bwd(block.norm, dr, None, r2, y2, m["gate2"])
    grads = {"gate2": g.dgate, "w_down": flat(g.dy).T @ flat(h)}
    f = FV.gated_ffn_bwd(block.ffn, g.dy @ block.w_down, n2, block.w_gate,
                         block.w_up, saved)
    grads.update(w_gate=f.dw_gate, w_up=f.dw_up)
    g = FV.gated_norm_bwd(block.norm, g.dx, f.dx, r1, y1, m["gate"],
                          m["scale2"])
    grads.update(gate=g.dgate, scale2=g.dscale, shift2=g.dshift,
                 w_o=flat(g.dy).T @ flat(o.view(B, L, D)))
    do = (g.dy @ block.w_o).view_as(o)
    c = FV.cross_attention_bwd(block.cross, q, k, v, o, do, lse, kv_len)
    dq = c.dq.view(B, L, D)
    dkv = torch.cat([c.dk, c.dv], 2).flatten(2)
    grads.update(w_q=flat(dq).T @ flat(n1), w_kv=flat(dkv).T @ flat(states),
                 states=dkv @ block.w_kv)
    # the residual branch's gradient joins inside the call
    g = FV.gated_norm_bwd(block.norm, g.dx, dq @ block.w_q, x, None,
                          scale=m["scale"])
    grads.update(x=g.dx, scale=g.dscale, shift=g.dshift)
    return r2, grads


def main() -> None:
    ap = argparse.ArgumentParser()
    ap.add_argument("--tokens", type=int, default=3180)
    ap.add_argument("--prompt", type=int, default=226)
    ap.add_argument("--heads", type=int, default=12)
    ap.add_argument("--hidden", type=int, default=4096)
    a = ap.parse_args()
    block = Conditioned(a.heads, a.heads, 1024, a.hidden)
    g = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").to(BF16)
    x, states = rnd(1, a.tokens, block.dim), rnd(1, a.prompt, 1024)
    dr = rnd(1, a.tokens, block.dim)
    k, v = block.prompt(states)
    for name, f in (("forward", lambda: block.forward(x, k, v)),
                    ("one token", lambda: block.forward(x[:, :1], k, v)),
                    ("training step",
                     lambda: train_step(block, x, states, dr))):
        for _ in range(3):
            f()
        start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        start.record()
        for _ in range(10):
            f()
        end.record()
        torch.cuda.synchronize()
        print(f"{name:14s} {start.elapsed_time(end) / 10:.3f} ms")
    if FV.fastvr_get_device_status() != FV.FASTVR_OK:
        raise RuntimeError("device-side failure")


if __name__ == "__main__":
    main()
