"""One layer of a video diffusion transformer around the block-sparse attention: the token-wise operators as they are
used together, forward, and a training step of the layer's feed-forward half.

    x1 = x + Wo attention(rotary(Wq n), rotary(Wk n), Wv n),   n = norm(x) (1 + scale1) + shift1
    y  = x1 + Wd (a(Wg m) * (Wu m)),                           m = norm(x1) (1 + scale2) + shift2

The norms, the rotary positions, the block mask, the attention and the gated feed-forward are the library's calls; the
plain projections are torch products.  All buffers are made once, so that a step is stream-ordered work alone.

GatedDitLayer is the layer whose condition also gates what each half adds, and whose projections can be in 4 bits:

    x1 = x + gate1 Wo attention(...),  y = x1 + gate2 Wd (a(Wg m) * (Wu m))

with its residual steps in one call each, the norm behind the first of them included, and a training step of what follows
the attention that ends with clipped gradients.

    python -m paper_2609_32197_b200.dit_layer --workload tiny [--steps 20] [--gated] [--projections nvfp4]
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

    def project_qkv(self):
        D = self.width
        for i, out in enumerate(self.qkv):
            torch.matmul(self.n, self.w_qkv[i * D:(i + 1) * D].T, out=out)

    def attention(self, x: torch.Tensor):
        """Fills o, what the output projection takes."""
        q, k, v = self.qkv
        binding.sparsp_layer_norm_fwd(self.norm, x, self.scale1, self.shift1, self.n, None, None)
        self.project_qkv()
        binding.sparsp_rotary_apply(self.shape, self.rotary, self.table, None, (0, 0, 0), q, k, q, k, False, None)
        binding.sparsp_block_mask(self.shape, q, k, self.topk, self.mask, None, None, None, None, self.workspace)
        binding.sparsp_sparse_attn_fwd(self.shape, q, k, v, self.mask, 0.0, self.o, None, self.workspace)

    def attention_half(self, x: torch.Tensor) -> torch.Tensor:
        self.attention(x)
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


class Fp4Linear:
    """y = x W^T with W, and x as it comes, in 4 bits.  `exponent` is that of x (nvfp4; from what x is seen to be: magnitudes
    above 2688 2^exponent become that).  The copy of W in 4 bits is that of requantize(), which follows a W that has changed."""

    def __init__(self, weight: torch.Tensor, tokens: int, fmt: str, exponent: int = 0):
        cols, depth = weight.shape
        device, dtype = weight.device, weight.dtype
        self.source, self.exponent = weight, exponent if fmt == "nvfp4" else 0
        self.described = binding.make_fp4(cols, depth, fmt, 0, dtype, weight.stride(0))
        self.weight = binding.make_fp4_operand(self.described, device)
        self.values = torch.empty_strided(weight.shape, weight.stride(), dtype=dtype, device=device)  # what W stands for
        self.input = binding.make_fp4(tokens, depth, fmt, self.exponent, dtype)
        self.product = binding.make_fp4_product(tokens, cols, depth, fmt, self.exponent, dtype)
        self.workspace = binding.make_fp4_product_workspace(self.product, device)
        self.requantize()

    def requantize(self, keep_exponent: bool = False):
        """W as it is now, in the same buffers.  Its exponent (nvfp4) follows its largest value, which is asked of the device, and a
        captured product goes on with the exponent of its capture; kept, all is stream-ordered work, and magnitudes above
        2688 2^exponent become that."""
        if not keep_exponent and self.described.format == binding.FP4_FORMATS["nvfp4"]:
            most = float(self.source.abs().max())
            if math.isfinite(most):
                self.described.exponent = min(math.ceil(math.log2(max(most, 2.0 ** -60) / (6 * 448))), 100)
                self.product.exponent = self.exponent + self.described.exponent
        binding.sparsp_fp4_quantize(self.described, self.source, *self.weight, self.values)

    def quantize(self, x, operand, values=None):
        binding.sparsp_fp4_quantize(self.input, x, *operand, values)

    def __call__(self, operand, out):
        binding.sparsp_fp4_product(self.product, *operand, *self.weight, None, out, self.workspace)


class GatedDitLayer(DitLayer):
    """projections: "bf16" (torch products), "mxfp4" or "nvfp4" for all but the feed-forward's first two.  In 4 bits
    update_weights() follows every change of w_qkv, w_out or w_down; activation_exponent (nvfp4) holds activations up to 2688
    times its power of two, 168 as it is, and what is above becomes that."""

    def __init__(self, wl: synth.Workload, hidden: int, seed: int = 0, dtype=torch.bfloat16, device="cuda",
                 projections: str = "bf16", activation_exponent: int = -4):
        super().__init__(wl, hidden, seed, dtype, device)
        N, D = wl.n_tokens, self.width
        gen = torch.Generator(device=device).manual_seed(seed + 1)
        self.gate1, self.gate2 = (torch.empty(1, D, device=device).normal_(0.0, 0.5, generator=gen) for _ in range(2))
        self.step1 = binding.make_gated_norm(N, D, dtype=dtype, weight_dtype=torch.float32)
        self.step2 = binding.make_gated_norm(N, D, norm_r="none", dtype=dtype, weight_dtype=torch.float32)
        self.step_workspace = binding.make_gated_norm_workspace(self.step1, device)
        self.grad_workspace = binding.make_grad_workspace(device)

        def empty(*dims, dtype=dtype):
            return torch.empty(dims, dtype=dtype, device=device)

        self.a, self.f, self.x1 = empty(N, D), empty(N, D), empty(N, D)  # what each half adds, and the stream between them
        self.stats = empty(N, 2, dtype=torch.float32)
        self.grad_norm = empty(1, dtype=torch.float32)
        self.grads = {k: torch.empty_like(getattr(self, k))
                      for k in ("w_gate", "w_up", "w_down", "gate1", "gate2", "scale2", "shift2")}
        self.grad_lists = [binding.make_grad_list([g for g in self.grads.values() if g.dtype == t])
                           for t in (dtype, torch.float32)]
        self.fp4 = {}
        if projections != "bf16":
            for name, weight in [("out", self.w_out), ("down", self.w_down)] + [
                    (f"qkv{i}", self.w_qkv[i * D:(i + 1) * D]) for i in range(3)]:
                self.fp4[name] = Fp4Linear(weight, N, projections, activation_exponent)
            self.operand = binding.make_fp4_operand(self.fp4["out"].input, device)  # of the width's activations
            self.hidden_operand = binding.make_fp4_operand(self.fp4["down"].input, device)
            self.h_values = empty(N, hidden)

    def update_weights(self):
        """The 4-bit copies of the projections' weights, as these are now."""
        for linear in self.fp4.values():
            linear.requantize()

    def project_qkv(self):
        if not self.fp4:
            return super().project_qkv()
        self.fp4["qkv0"].quantize(self.n, self.operand)
        for i, out in enumerate(self.qkv):
            self.fp4[f"qkv{i}"](self.operand, out)

    def project_out(self):
        if not self.fp4:
            torch.matmul(self.o, self.w_out.T, out=self.a)
        else:
            self.fp4["out"].quantize(self.o, self.operand)
            self.fp4["out"](self.operand, self.a)

    def project_down(self, training: bool):
        if not self.fp4:
            torch.matmul(self.h, self.w_down.T, out=self.f)
        else:
            self.fp4["down"].quantize(self.h, self.hidden_operand, self.h_values if training else None)
            self.fp4["down"](self.hidden_operand, self.f)

    def behind_attention(self, x: torch.Tensor, training: bool = False) -> torch.Tensor:
        """y from the layer's input x and what the attention half adds, a."""
        keep = (self.gate, self.up) if training else (None, None)
        binding.sparsp_gated_norm_fwd(self.step1, x, self.a, self.gate1, None, None, self.scale2, self.shift2, self.x1, self.m,
                                      None, self.stats if training else None)
        binding.sparsp_gated_ffn_fwd(self.ffn, self.m, self.w_gate, self.w_up, self.h, *keep, self.ffn_workspace)
        self.project_down(training)
        y = torch.empty_like(x)
        binding.sparsp_gated_norm_fwd(self.step2, self.x1, self.f, self.gate2, None, None, None, None, y, None, None, None)
        return y

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        """x, y [tokens][width]"""
        self.attention(x)
        self.project_out()
        return self.behind_attention(x)

    def training_step(self, x: torch.Tensor, dy: torch.Tensor, max_norm: float = math.inf) -> dict:
        """Gradients of what follows the attention, for dy at the layer's output, forward pass included: of its weights,
        clipped together to max_norm, and "x" and "a", the gradients of what it takes.  Roundings to 4 bits have the
        gradient of nothing (straight through): products go on with the values that were multiplied.  w_down is rounded anew
        in each step, under the exponent of the last update_weights()."""
        if self.fp4:
            self.fp4["down"].requantize(keep_exponent=True)
        self.behind_attention(x, training=True)
        w_down, h = (self.fp4["down"].values, self.h_values) if self.fp4 else (self.w_down, self.h)
        grads = self.grads  # (of one step: the next writes them again)
        df, dm, dx, da = (torch.empty_like(x) for _ in range(4))
        binding.sparsp_gated_norm_bwd(self.step2, None, dy, None, self.f, self.gate2, None, None, None, None, None, None, df,
                                      grads["gate2"], None, None, None, None, self.step_workspace)
        torch.matmul(df.T, h, out=grads["w_down"])
        binding.sparsp_gated_ffn_bwd(self.ffn, df @ w_down, self.m, self.w_gate, self.w_up, self.gate, self.up, dm,
                                     grads["w_gate"], grads["w_up"], self.ffn_workspace)
        binding.sparsp_gated_norm_bwd(self.step1, dm, dy, self.x1, self.a, self.gate1, None, None, self.scale2, None,
                                      self.stats, dx, da, grads["gate1"], None, None, grads["scale2"], grads["shift2"],
                                      self.step_workspace)
        for i, g in enumerate(self.grad_lists):  # one norm over both types
            binding.sparsp_grad_squares(g, self.grad_workspace, accumulate=i > 0)
        for g in self.grad_lists:
            binding.sparsp_grad_clip(g, max_norm, self.grad_norm, self.grad_workspace)
        return {**grads, "x": dx, "a": da}

    def status(self) -> int:
        return super().status() or next((s for s in (binding.sparsp_status(f.workspace) for f in self.fp4.values()) if s), 0)


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


def _gated(wl, width: int, hidden: int, args):
    layer = GatedDitLayer(wl, hidden, projections=args.projections)
    x, dy = (torch.empty(wl.n_tokens, width, dtype=torch.bfloat16, device="cuda").normal_(0.0, 1.0) for _ in range(2))
    layer.forward(x)
    print(f"{wl.name}: {wl.n_tokens} tokens, width {width}, feed-forward {hidden}, projections in {args.projections}")
    for name, f in (("layer", lambda: layer.forward(x)),
                    ("training step behind the attention, clipped", lambda: layer.training_step(x, dy, 1.0))):
        print(f"  {name}: {_time(f, args.steps):.1f} us")
    if layer.status() != binding.SPARSP_OK:
        raise SystemExit(binding.sparsp_last_error())


def main(argv=None):
    ap = argparse.ArgumentParser(description="One layer: times of its halves and of a training step of the second.")
    ap.add_argument("--workload", default="tiny", choices=sorted(synth.WORKLOADS))
    ap.add_argument("--hidden", type=int, default=0, help="feed-forward width; default 8/3 of the layer's, in steps of 256")
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--gated", action="store_true", help="the layer with gates, its steps in one call each")
    ap.add_argument("--projections", default="bf16", choices=("bf16", "mxfp4", "nvfp4"), help="of the gated layer")
    args = ap.parse_args(argv)
    wl = synth.WORKLOADS[args.workload]
    width = wl.heads * wl.head_dim
    hidden = args.hidden or math.ceil(width * 8 / 3 / 256) * 256
    if args.gated or args.projections != "bf16":
        return _gated(wl, width, hidden, args)
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
