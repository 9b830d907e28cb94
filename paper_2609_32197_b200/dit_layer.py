"""One layer of a video diffusion transformer around the block-sparse attention: the token-wise operators as they are
used together, forward, and a training step of the layer's feed-forward half.

    x1 = x + Wo attention(rotary(Wq n), rotary(Wk n), Wv n),   n = norm(x) (1 + scale1) + shift1
    y  = x1 + Wd (a(Wg m) * (Wu m)),                           m = norm(x1) (1 + scale2) + shift2

The norms, the rotary positions, the block mask, the attention and the gated feed-forward are the library's calls; the
plain projections are torch products.  All buffers are made once, so that a step is stream-ordered work alone.

    python -m paper_2609_32197_b200.dit_layer --workload tiny [--steps 20]
"""
from __future__ import annotations

import argparse
import math

import torch

from . import binding, synth


def axis_pairs(head_dim: int):
    """Channel pairs of the t, h and w coordinates: all of the head, h and w alike."""
    side = head_dim // 6
    return head_dim // 2 - 2 * side, side, side


class DitLayer:
    """Weights (random, seeded), conditioning, tables, buffers and workspaces of one layer; one sequence."""

    def __init__(self, wl: synth.Workload, hidden: int, seed: int = 0, dtype=torch.bfloat16, device="cuda"):
        self.wl, self.hidden, self.dtype = wl, hidden, dtype
        H, d, N = wl.heads, wl.head_dim, wl.n_tokens
        self.width = H * d
        gen = torch.Generator(device=device).manual_seed(seed)

        def rand(*dims, scale=1.0):
            return torch.empty(dims, dtype=dtype, device=device).normal_(0.0, scale, generator=gen)

        D = self.width
        self.w_qkv = rand(3 * D, D, scale=D ** -0.5)
        self.w_out = rand(D, D, scale=D ** -0.5)
        self.w_gate_up = rand(2 * hidden, D, scale=D ** -0.5)  # rows of Wg, then of Wu
        self.w_gate, self.w_up = self.w_gate_up[:hidden], self.w_gate_up[hidden:]
        self.w_down = rand(D, hidden, scale=hidden ** -0.5)
        # what the conditioning network gives for this sequence
        self.scale1, self.scale2 = (1.0 + rand(1, D, scale=0.2).float() for _ in range(2))
        self.shift1, self.shift2 = (rand(1, D, scale=0.2).float() for _ in range(2))

        self.shape = binding.make_shape(H, d, wl.grid, wl.n_text, wl.block, layout="NHD")
        self.norm = binding.make_norm(N, D, dtype=dtype, weight_dtype=torch.float32)
        self.ffn = binding.make_ffn(N, D, hidden, "silu", dtype)
        pairs = axis_pairs(d)
        self.rotary = binding.make_rotary(pairs, wl.grid, "interleaved", 0, dtype)
        freq = [binding.sparsp_rotary_frequencies(n, 10000.0)[0] for n in pairs]
        self.table = binding.make_rotary_table(self.rotary, torch.cat(freq))
        g = binding.sparsp_geometry(self.shape)
        self.topk = wl.topk_abs or binding.sparsp_resolve_topk(wl.topk_pct[0], g.n_video_blocks)
        self.mask = binding.alloc_mask_outputs(self.shape, self.topk, with_list=False)["mask"]
        self.workspace = binding.make_workspace(self.shape, 1)
        self.ffn_workspace = binding.make_ffn_workspace(self.ffn, backward=True)
        self.norm_workspace = binding.make_norm_workspace(self.norm)

        def empty(*dims, dtype=dtype):
            return torch.empty(dims, dtype=dtype, device=device)

        self.n = empty(N, D)
        self.qkv = [empty(N, D) for _ in range(3)]
        self.o = empty(N, D)
        self.m, self.mean, self.rstd = empty(N, D), empty(N, dtype=torch.float32), empty(N, dtype=torch.float32)
        self.h, self.gate, self.up = (empty(N, hidden) for _ in range(3))

    def attention_half(self, x: torch.Tensor) -> torch.Tensor:
        D = self.width
        q, k, v = self.qkv
        binding.sparsp_layer_norm_fwd(self.norm, x, self.scale1, self.shift1, self.n, None, None)
        for i, out in enumerate(self.qkv):
            torch.matmul(self.n, self.w_qkv[i * D:(i + 1) * D].T, out=out)
        binding.sparsp_rotary_apply(self.shape, self.rotary, self.table, None, (0, 0, 0), q, k, q, k, False, None)
        binding.sparsp_block_mask(self.shape, q, k, self.topk, self.mask, None, None, None, None, self.workspace)
        binding.sparsp_sparse_attn_fwd(self.shape, q, k, v, self.mask, 0.0, self.o, None, self.workspace)
        return torch.addmm(x, self.o, self.w_out.T)

    def feed_forward_half(self, x1: torch.Tensor, training: bool = False) -> torch.Tensor:
        keep = (self.gate, self.up) if training else (None, None)
        stats = (self.mean, self.rstd) if training else (None, None)
        binding.sparsp_layer_norm_fwd(self.norm, x1, self.scale2, self.shift2, self.m, *stats)
        binding.sparsp_gated_ffn_fwd(self.ffn, self.m, self.w_gate, self.w_up, self.h, *keep, self.ffn_workspace)
        return torch.addmm(x1, self.h, self.w_down.T)

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        """x, y [tokens][width]"""
        return self.feed_forward_half(self.attention_half(x))

    def feed_forward_backward(self, x1: torch.Tensor, dy: torch.Tensor) -> dict:
        """Gradients of the feed-forward half after feed_forward_half(x1, training=True), for dy at its output."""
        dh = dy @ self.w_down
        grads = {"w_down": dy.T @ self.h, "w_gate": torch.empty_like(self.w_gate), "w_up": torch.empty_like(self.w_up)}
        dm = torch.empty_like(self.m)
        binding.sparsp_gated_ffn_bwd(self.ffn, dh, self.m, self.w_gate, self.w_up, self.gate, self.up, dm,
                                     grads["w_gate"], grads["w_up"], self.ffn_workspace)
        grads["scale2"], grads["shift2"] = torch.empty_like(self.scale2), torch.empty_like(self.shift2)
        dx = torch.empty_like(x1)
        binding.sparsp_layer_norm_bwd(self.norm, dm, x1, self.scale2, self.mean, self.rstd, dx, grads["scale2"],
                                      grads["shift2"], self.norm_workspace)
        grads["x"] = dx + dy
        return grads

    def status(self) -> int:
        """SPARSP_OK unless a kernel reported a problem."""
        return next((s for s in (binding.sparsp_status(w) for w in (self.workspace, self.ffn_workspace)) if s), 0)


def _time(f, steps: int) -> float:
    for _ in range(3):
        f()
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    torch.cuda.synchronize()
    begin.record()
    for _ in range(steps):
        f()
    end.record()
    torch.cuda.synchronize()
    return begin.elapsed_time(end) / steps * 1e3


def main(argv=None):
    ap = argparse.ArgumentParser(description="One layer: times of its halves and of a training step of the second.")
    ap.add_argument("--workload", default="tiny", choices=sorted(synth.WORKLOADS))
    ap.add_argument("--hidden", type=int, default=0, help="feed-forward width; default 8/3 of the layer's, in steps of 256")
    ap.add_argument("--steps", type=int, default=20)
    args = ap.parse_args(argv)
    wl = synth.WORKLOADS[args.workload]
    width = wl.heads * wl.head_dim
    hidden = args.hidden or math.ceil(width * 8 / 3 / 256) * 256
    layer = DitLayer(wl, hidden)
    x = torch.empty(wl.n_tokens, width, dtype=torch.bfloat16, device="cuda").normal_(0.0, 1.0)
    dy = torch.empty_like(x).normal_(0.0, 1.0)
    x1 = layer.attention_half(x)

    def train():
        layer.feed_forward_half(x1, training=True)
        layer.feed_forward_backward(x1, dy)

    print(f"{wl.name}: {wl.n_tokens} tokens, width {width}, feed-forward {hidden}")
    for name, f in (("attention half", lambda: layer.attention_half(x)),
                    ("feed-forward half", lambda: layer.feed_forward_half(x1)),
                    ("training step of the feed-forward half", train)):
        print(f"  {name}: {_time(f, args.steps):.1f} us")
    if layer.status() != binding.SPARSP_OK:
        raise SystemExit(binding.sparsp_last_error())


if __name__ == "__main__":
    main()
