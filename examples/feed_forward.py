"""The feed-forward block of a decoder layer with the library's operators, as a serving loop would call them.

    python examples/feed_forward.py [--tokens 16] [--hidden 4096] [--inter 14336] [--expanded 15360]

    residual += x;  t = RMSNorm(residual) in 8 bits          xq_f8_norm_quant
    h = silu(t Wg^T) * (t Wu^T)                                  xq_f8_gated
    out = h Wd^T, either
      - W4A4 on the expanded, rotated channels (h in bf16)       xq_expanded_linear
      - in 8 bits (h in 8 bits)                                  xq_f8_gemm

Weights are random.  Prints how far each output is from the same block in fp32 torch, and the time of a pass.
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2503_17513_b200 import xq  # noqa: E402


class FeedForward:
    """What a program keeps for one layer: weights objects, workspaces, buffers of the largest token count."""

    def __init__(self, gamma, Wg, Wu, Wd, expanded, tokens):
        inter, hidden = Wg.shape
        self.gamma = gamma
        self.gate, self.up, self.down8 = (xq.xq_f8_prepare_weights(w) for w in (Wg, Wu, Wd))
        self.down4 = xq.xq_prepare_weights(Wd.cpu().view(torch.int16).numpy().view(np.uint16), expanded)
        self.ws, self.ws8 = xq.new_f8_workspace(tokens, self.gate), xq.new_f8_workspace(tokens, self.down8)
        self.ws4 = xq.new_workspace(tokens, self.down4)
        self.t, self.h8 = xq.new_f8_rows(tokens, hidden), xq.new_f8_rows(tokens, inter)
        self.h = torch.empty((tokens, inter), dtype=torch.bfloat16, device="cuda")

    def __call__(self, x, residual, out, eight):
        """out = feed-forward(norm(residual + x)); residual is updated in place."""
        M = x.shape[0]
        (tc, ts), (hc, hs) = (tuple(a[:M] for a in pair) for pair in (self.t, self.h8))
        xq.xq_f8_norm_quant(x, self.gamma, 1e-5, tc, ts, residual=residual, sum_out=residual)
        if eight:
            xq.xq_f8_gated(tc, ts, M, self.gate, self.up, self.ws, out_codes=hc, out_scales=hs)
            xq.xq_f8_gemm(hc, hs, M, self.down8, out, self.ws8)
        else:
            xq.xq_f8_gated(tc, ts, M, self.gate, self.up, self.ws, out=self.h[:M])
            xq.xq_expanded_linear(self.h[:M], self.down4, out, self.ws4)


def reference(x, residual, gamma, Wg, Wu, Wd):
    t = residual.float() + x.float()
    y = t * torch.rsqrt(t.square().mean(1, keepdim=True) + 1e-5) * gamma.float()
    return (torch.nn.functional.silu(y @ Wg.float().T) * (y @ Wu.float().T)) @ Wd.float().T


def run(tokens, hidden, inter, expanded, passes=50, say=print):
    g = torch.Generator(device="cuda").manual_seed(0)

    def normal(rows, cols, scale):
        return (scale * torch.randn(rows, cols, generator=g, device="cuda")).bfloat16()

    Wg, Wu, Wd = normal(inter, hidden, 0.02), normal(inter, hidden, 0.02), normal(hidden, inter, 0.02)
    gamma = (1 + 0.1 * torch.randn(hidden, generator=g, device="cuda")).bfloat16()
    x, residual = normal(tokens, hidden, 1.0), normal(tokens, hidden, 1.0)
    want = reference(x, residual, gamma, Wg, Wu, Wd)
    layer = FeedForward(gamma, Wg, Wu, Wd, expanded, tokens)
    out, found = torch.empty((tokens, hidden), dtype=torch.bfloat16, device="cuda"), {}
    for eight in (False, True):
        layer(x, residual.clone(), out, eight)
        assert xq.xq_poll_status(layer.ws) == xq.OK and xq.xq_poll_status(layer.ws8 if eight else layer.ws4) == xq.OK
        rel = float((out.float() - want).norm() / want.norm())
        stream = residual.clone()
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        for _ in range(passes):
            layer(x, stream, out, eight)
        b.record()
        b.synchronize()
        name = "8-bit down projection" if eight else f"W4A4 down projection on {expanded} channels"
        say(f"{tokens} tokens, {name}: relative error {rel:.3f} of fp32, {a.elapsed_time(b) / passes * 1e3:.1f} us a pass")
        found[name.split(" ")[0]] = rel
    return found


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, default in (("tokens", 16), ("hidden", 4096), ("inter", 14336), ("expanded", 15360)):
        ap.add_argument("--" + name, type=int, default=default)
    a = ap.parse_args()
    run(a.tokens, a.hidden, a.inter, a.expanded)
