"""A block of a streaming DiT on the library's operators.

    python examples/streaming_block.py [--chunks N] [--heads H] [--rows R --cols C]

streams synthetic chunks through one block (random weights) twice, over a
bfloat16 cache and over a 4-bit one, and prints both caches' bytes, those of
the 4-bit cache's workspace, the time per chunk and how far the outputs are
apart.  Per chunk the block runs

    gated_norm            modulated norm of the residual stream
    (QKV projection)      a plain matrix product
    rotary                positions on queries and keys, straight from the
                          projection's output
    append, forward       the chunk's keys and values into the cache, its
                          queries over the visible window
    (output projection)
    gated_norm            residual update and the next norm

`train_step` runs the training form of the same block over a whole clip,
forward and backward, and returns the gradients.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2609_36757_gb300 import fastvr as FV  # noqa: E402

BF16 = torch.bfloat16


class Block:
    """Weights and modulation of one attention block of `heads` heads of 128
    (kv_heads of them for keys and values), for frames of rows x cols tokens."""

    def __init__(self, heads: int, kv_heads: int, rows: int, cols: int,
                 batch: int = 1, seed: int = 0, head_dim: int = 128):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
        self.heads, self.kv_heads, self.d = heads, kv_heads, head_dim
        self.rows, self.cols, self.batch = rows, cols, batch
        D = self.dim = heads * head_dim
        width = (heads + 2 * kv_heads) * head_dim
        self.w_qkv = (rnd(width, D) * D ** -0.5).to(BF16)
        self.w_out = (rnd(D, D) * D ** -0.5).to(BF16)
        self.post_weight = 1 + 0.1 * rnd(D)
        # timestep modulation of the block, one vector per batch entry
        self.mod = {n: 0.2 * rnd(batch, 1, D)
                    for n in ("scale", "shift", "gate", "scale2", "shift2")}
        side = head_dim // 2 // 3
        self.rot = FV.make_rotary_config(
            head_dim, sections=[head_dim // 2 - 2 * side, side, side])
        self.norm_in = FV.make_norm_config(pre="layer")
        self.norm_out = FV.make_norm_config(pre="layer", post="rms")

    @property
    def frame(self) -> int:
        return self.rows * self.cols

    def positions(self, first_frame: int, frames: int):
        """(frame, row, column) of every token, int32 [frames * frame, 3]."""
        t, y, x = torch.meshgrid(
            torch.arange(first_frame, first_frame + frames, device="cuda"),
            torch.arange(self.rows, device="cuda"),
            torch.arange(self.cols, device="cuda"), indexing="ij")
        return torch.stack([t, y, x], -1).reshape(-1, 3).to(torch.int32)

    def project(self, h):
        """q, k, v views of one fused projection."""
        B, L, _ = h.shape
        qkv = (h @ self.w_qkv.T).view(B, L, -1, self.d)
        return qkv.split([self.heads, self.kv_heads, self.kv_heads], 2)

    def chunk(self, cache, x, first_frame: int):
        """One chunk x [B, f * frame, dim] through the block; returns the
        residual stream after it and the next block's normalised input."""
        B, L, D = x.shape
        m = self.mod
        _, h = FV.gated_norm(self.norm_in, x, None, scale=m["scale"],
                             shift=m["shift"], want_r=False)
        q, k, v = self.project(h)
        q, k = FV.rotary(self.rot, q, k,
                         self.positions(first_frame, L // self.frame))
        if isinstance(cache, FV.StreamingAttention4):
            cache.append(k, v)
        else:  # the bfloat16 cache takes contiguous tensors, a head each
            G = self.heads // self.kv_heads
            cache.append(k.repeat_interleave(G, 2),
                         v.repeat_interleave(G, 2))
        o = cache.forward(q)
        y = o.view(B, L, D) @ self.w_out.T
        return FV.gated_norm(self.norm_out, x, y, m["gate"], m["scale2"],
                             m["shift2"], post_weight=self.post_weight)


def attention_config(block: Block, frames_per_chunk: int, window: int):
    return FV.make_config(block.batch, block.heads, block.d, block.frame,
                          frames_per_chunk, window)


def train_step(block: Block, x, dr, dh, frames_per_chunk: int, window: int):
    """Forward and backward of the block over a whole clip x [B, L, dim] (one
    head per key head), dr and dh the gradients of its two outputs.  Returns
    (r, h, gradients by name)."""
    B, L, D = x.shape
    m, cfg = block.mod, attention_config(block, frames_per_chunk, window)
    pos = block.positions(0, L // block.frame)
    _, n = FV.gated_norm(block.norm_in, x, None, scale=m["scale"],
                         shift=m["shift"], want_r=False)
    q, k, v = block.project(n)
    q, k = FV.rotary(block.rot, q, k, pos)
    v = v.contiguous()
    o, lse = FV.blockcausal_attention(cfg, q, k, v, want_lse=True)
    of = o.view(B, L, D)
    y = of @ block.w_out.T
    r, h = FV.gated_norm(block.norm_out, x, y, m["gate"], m["scale2"],
                         m["shift2"], post_weight=block.post_weight)

    g2 = FV.gated_norm_bwd(block.norm_out, dr, dh, r, y, m["gate"],
                           m["scale2"], post_weight=block.post_weight)
    do = g2.dy @ block.w_out
    grads = {"w_out": g2.dy.flatten(0, 1).T @ of.flatten(0, 1),
             "gate": g2.dgate, "scale2": g2.dscale, "shift2": g2.dshift,
             "post_weight": g2.dpost_weight}
    dq, dk, dv = FV.blockcausal_attention_bwd(
        cfg, q, k, v, o, do.view_as(o).contiguous(), lse)
    dq, dk = FV.rotary_bwd(block.rot, dq, dk, pos, out=(dq, dk))  # in place
    dqkv = torch.cat([dq, dk, dv], 2).view(B, L, -1)
    grads["w_qkv"] = dqkv.flatten(0, 1).T @ n.flatten(0, 1)
    dn = dqkv @ block.w_qkv
    # the residual branch's gradient joins inside the call
    g1 = FV.gated_norm_bwd(block.norm_in, g2.dx, dn, x, None,
                           scale=m["scale"])
    grads.update(x=g1.dx, scale=g1.dscale, shift=g1.dshift)
    return r, h, grads


def stream(block: Block, cache, chunks, frames_per_chunk: int):
    """Outputs of the chunks and milliseconds per chunk."""
    outs, marks = [], []
    for i, x in enumerate(chunks):
        start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        start.record()
        outs.append(block.chunk(cache, x, i * frames_per_chunk))
        end.record()
        marks.append((start, end))
    torch.cuda.synchronize()
    if cache.status() != FV.FASTVR_OK:
        raise RuntimeError("device-side failure")
    return outs, [s.elapsed_time(e) for s, e in marks]


def main() -> None:
    ap = argparse.ArgumentParser()
    ap.add_argument("--chunks", type=int, default=8)
    ap.add_argument("--heads", type=int, default=12)
    ap.add_argument("--rows", type=int, default=30)
    ap.add_argument("--cols", type=int, default=53)
    ap.add_argument("--frames", type=int, default=2, help="per chunk")
    ap.add_argument("--window", type=int, default=4, help="earlier chunks")
    a = ap.parse_args()
    block = Block(a.heads, a.heads, a.rows, a.cols)
    cfg = attention_config(block, a.frames, a.window)
    g = torch.Generator(device="cuda").manual_seed(1)
    xs = [torch.randn(1, a.frames * block.frame, block.dim, generator=g,
                      device="cuda").to(BF16) for _ in range(a.chunks)]
    caches = {"bfloat16": FV.StreamingAttention(cfg),
              "4-bit": FV.StreamingAttention4(cfg)}
    outs = {}
    for name, cache in caches.items():
        stream(block, cache, xs[:2], a.frames)  # warm-up
        cache.reset()
        outs[name], ms = stream(block, cache, xs, a.frames)
        work = getattr(cache, "workspace", None)  # can serve many streams
        work = 0 if work is None else work.numel()
        print(f"{name:8s} cache {cache.nbytes / 2**20:8.1f} MiB, workspace "
              f"{work / 2**20:8.1f} MiB, {ms[-1]:.3f} ms for the last chunk")
    a16, a4 = (outs[n][-1][0].float() for n in caches)
    print(f"residual streams differ by {float((a4 - a16).norm() / a16.norm()):.2e}"
          " (relative L2)")


if __name__ == "__main__":
    main()
