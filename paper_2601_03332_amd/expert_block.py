"""A residual block of a language model with a mixture of 8-bit experts in front of a KAN layer, on the operators of this package:

    python -m paper_2601_03332_amd.expert_block [--tokens 1 16 512 8192] [--codes fp8 int8]

    residual <- residual + x;  n = norm(residual)                        lutkan_rmsnorm_fp8: one pass, out in 8 bits
    p, e = top(softmax(n R^T))                                           lutkan_matmul_fp8 (the router R), then torch on [tokens, experts]
    rows, places <- e sorted                                             lutkan_expert_sort
    z_s = n_t W_e^T for each of a token's experts                        lutkan_grouped_matmul_fp8, rows sorted by expert
    x <- sum over a token's experts of p * KAN(z_s)                      lutkan_forward: the compiled 8-bit table layer; lutkan_expert_combine

The norm's output and the weights are 8-bit floating point with a scale per 128 columns (codes="fp8"), or 8-bit integers with a scale per token
and per output (codes="int8": the operators of the same names with _int8).

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

    def __init__(self, norm, router, experts, layer, top: int = 2, eps: float = 1e-6, codes: str = "fp8"):
        from . import LutKanError, lutkan_quantise_fp8, lutkan_quantise_int8
        if codes not in ("fp8", "int8"):
            raise LutKanError(f"ExpertBlock: codes are 'fp8' or 'int8', here {codes!r}")
        if experts.dim() != 3 or experts.shape[1] != layer.d or experts.shape[2] != layer.m or not 1 <= top <= experts.shape[0]:
            raise LutKanError("ExpertBlock: experts are [experts, layer.d, layer.m], top is at most their number")
        if tuple(router.shape) != (experts.shape[0], layer.m):           # (an expert that is not there would be counted out of bounds)
            raise LutKanError(f"ExpertBlock: router is [experts, layer.m], here [{experts.shape[0]}, {layer.m}]")
        self.norm, self.layer, self.top, self.eps, self.codes = norm, layer, top, eps, codes
        quantise = lutkan_quantise_int8 if codes == "int8" else lutkan_quantise_fp8
        self.router, self.experts = quantise(router), quantise(experts)

    def __call__(self, x, residual):
        """x [tokens, width], residual [tokens, width] -> (x, residual) of the next block, in their types."""
        import torch

        from . import (lutkan_expert_combine, lutkan_expert_sort, lutkan_forward, lutkan_grouped_matmul_fp8, lutkan_grouped_matmul_int8, lutkan_matmul_fp8,
                       lutkan_matmul_int8, lutkan_rmsnorm_fp8, lutkan_rmsnorm_int8)
        norm, product, by_expert = ((lutkan_rmsnorm_int8, lutkan_matmul_int8, lutkan_grouped_matmul_int8) if self.codes == "int8" else
                                    (lutkan_rmsnorm_fp8, lutkan_matmul_fp8, lutkan_grouped_matmul_fp8))
        codes, scales, residual = norm(x, self.norm, residual=residual, eps=self.eps)
        p, expert = torch.softmax(product(codes, scales, *self.router), dim=1).topk(self.top, dim=1)
        rows, places, sizes = lutkan_expert_sort(expert, self.experts[0].shape[0])
        z = by_expert(codes, scales, *self.experts, sizes, rows=rows)
        return lutkan_expert_combine(lutkan_forward(self.layer, z), places, p, dtype=x.dtype), residual


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
    ap.add_argument("--codes", nargs="+", default=["fp8"], choices=["fp8", "int8"])
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
    layer = art.to_device("cuda:0")
    blocks = [ExpertBlock(norm, router, experts, layer, args.top, codes=codes) for codes in args.codes]
    spline = art.bspline_to_device("cuda:0")
    print(f"width {width}, {args.experts} experts of {inner}, {args.top} a token, KAN {inner} -> {width} (G = {G}, L = {L}, int8)")
    for tokens in args.tokens:
        x, residual = normal(tokens, width).bfloat16(), 2 * normal(tokens, width).bfloat16()
        for block in blocks:
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
            which = f", {block.codes:>4s}" if len(blocks) > 1 else ""
            print(f"{tokens:6d} tokens{which}: {begin.elapsed_time(end) / 20 * 1000:9.1f} us a pass, output {off:.3f} from the unquantised block's", flush=True)


if __name__ == "__main__":
    main()
