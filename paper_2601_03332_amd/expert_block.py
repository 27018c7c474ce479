"""A residual block of a language model with a mixture of 8-bit experts in front of a KAN layer, on the operators of this package:

    python -m paper_2601_03332_amd.expert_block [--tokens 1 16 512 8192]

    residual <- residual + x;  n = norm(residual)                        lutkan_rmsnorm_fp8: one pass, out in 8 bits
    p, e = top(softmax(n R^T))                                           lutkan_matmul_fp8 (the router R), then torch on [tokens, experts]
    z_s = n_t W_e^T for each of a token's experts                        lutkan_grouped_matmul_fp8, rows sorted by expert
    x <- sum over a token's experts of p * KAN(z_s)                      lutkan_forward: the compiled 8-bit table layer

The norm keeps the experts' outputs of about unit size, so that they stay in the KAN layer's knot domain.  Nothing waits for the GPU: the
groups' sizes stay there.  main() prints, for each number of tokens, the time of one pass and how far the block's output is from the same
block with unquantised weights, activations and splines (random weights: the figures show the operators at work, not a trained model).
"""
from __future__ import annotations

import argparse
import math

import numpy as np


class ExpertBlock:
    """router [experts, width] and experts [experts, inner, width]: weights of any of the three float types, converted here;
    layer: a LutLayer inner -> width."""

    def __init__(self, norm, router, experts, layer, top: int = 2, eps: float = 1e-6):
        from . import LutKanError, lutkan_quantise_fp8
        if experts.dim() != 3 or experts.shape[1] != layer.d or experts.shape[2] != layer.m or not 1 <= top <= experts.shape[0]:
            raise LutKanError("ExpertBlock: experts are [experts, layer.d, layer.m], top is at most their number")
        if tuple(router.shape) != (experts.shape[0], layer.m):           # (an expert that is not there would be counted out of bounds)
            raise LutKanError(f"ExpertBlock: router is [experts, layer.m], here [{experts.shape[0]}, {layer.m}]")
        self.norm, self.layer, self.top, self.eps = norm, layer, top, eps
        self.router, self.experts = lutkan_quantise_fp8(router), lutkan_quantise_fp8(experts)

    def __call__(self, x, residual):
        """x [tokens, width], residual [tokens, width] -> (x, residual) of the next block, in their types."""
        import torch

        from . import lutkan_forward, lutkan_grouped_matmul_fp8, lutkan_matmul_fp8, lutkan_rmsnorm_fp8
        codes, scales, residual = lutkan_rmsnorm_fp8(x, self.norm, residual=residual, eps=self.eps)
        p, expert = torch.softmax(lutkan_matmul_fp8(codes, scales, *self.router), dim=1).topk(self.top, dim=1)
        expert = expert.flatten()
        order = torch.sort(expert, stable=True).indices
        sizes = torch.zeros(self.experts[0].shape[0], dtype=torch.int64, device=x.device).scatter_add_(0, expert, torch.ones_like(expert))
        z = lutkan_grouped_matmul_fp8(codes, scales, *self.experts, sizes, rows=order // self.top)
        y = torch.empty((expert.numel(), self.layer.m), dtype=torch.float32, device=x.device)
        y[order] = lutkan_forward(self.layer, z)                      # back in the tokens' order
        return (y.view(x.shape[0], self.top, self.layer.m) * p[..., None]).sum(dim=1).to(x.dtype), residual


def _unquantised(x, residual, norm, router, experts, spline, top, eps):
    """The same block in 32 bits; `spline` is the B-spline layer that the table was compiled from."""
    import torch

    from . import bspline_kan_forward
    h = x.float() + residual.float()
    n = h * torch.rsqrt(h.square().mean(dim=1, keepdim=True) + eps) * norm.float()
    p, expert = torch.softmax(n @ router.t(), dim=1).topk(top, dim=1)
    out = torch.zeros((x.shape[0], spline.m), device=x.device)
    for e in range(experts.shape[0]):
        token, place = torch.where(expert == e)
        if token.numel():
            out[token] += p[token, place, None] * bspline_kan_forward(spline, (n[token] @ experts[e].t()).contiguous())
    return out


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, nargs="+", default=[1, 16, 512, 8192])
    ap.add_argument("--experts", type=int, default=8)
    ap.add_argument("--top", type=int, default=2)
    args = ap.parse_args()
    import torch

    from . import CLIP_X, CLOSED, SYM_INT8, lutkan_compile
    width, inner, G, L, half = 1024, 256, 8, 64, 4.0
    rng = np.random.default_rng(7)
    knots = (-half + (np.arange(G + 7) - 3) * (2 * half / G)).astype(np.float32)
    coef = (rng.standard_normal((inner, width, G + 3)) / math.sqrt(inner)).astype(np.float32)
    art = lutkan_compile(inner, width, G, 3, knots, coef, L, SYM_INT8, CLOSED, CLIP_X)
    gen = torch.Generator(device="cuda:0").manual_seed(7)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda:0")
    norm, router, experts = 1 + 0.1 * normal(width), normal(args.experts, width) / math.sqrt(width), normal(args.experts, inner, width) / math.sqrt(width)
    block = ExpertBlock(norm, router, experts, art.to_device("cuda:0"), args.top)
    spline = art.bspline_to_device("cuda:0")
    print(f"width {width}, {args.experts} experts of {inner}, {args.top} a token, KAN {inner} -> {width} (G = {G}, L = {L}, int8)")
    for tokens in args.tokens:
        x, residual = normal(tokens, width).bfloat16(), 2 * normal(tokens, width).bfloat16()
        y, _ = block(x, residual)
        ref = _unquantised(x, residual, norm, router, experts, spline, args.top, block.eps)
        torch.cuda.synchronize()
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        for _ in range(20):
            block(x, residual)
        end.record()
        torch.cuda.synchronize()
        off = float((y.float() - ref).norm() / ref.norm())
        print(f"{tokens:6d} tokens: {begin.elapsed_time(end) / 20 * 1000:9.1f} us a pass, output {off:.3f} from the unquantised block's", flush=True)


if __name__ == "__main__":
    main()
