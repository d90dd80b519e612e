"""The 8-bit operators together with the expanded W4A4 layer: the feed-forward block of examples/feed_forward.py."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import f8
from paper_2503_17513_b200 import synth

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("feed_forward", os.path.join(ROOT, "examples", "feed_forward.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("tokens", [1, 20, 150])
def test_example_runs_and_is_near_fp32(example, tokens):
    """Error of the block: 8-bit tokens and weights are each off by at most 2^-4 relative per element, 0.027 rms (three mantissa
    bits), W4A4 by about 0.15 rms; independent errors add in squares: below 0.1 and 0.25."""
    rel = example.run(tokens, 512, 1024, 1088, passes=3, say=lambda *a: None)
    assert rel["8-bit"] < 0.1 and rel["W4A4"] < 0.25


@pytest.mark.parametrize("M", [3, 40])
def test_gated_result_feeds_the_expanded_layer(example, oracle, M):
    """bf16 result of the gated pair -> xq_expanded_linear, against the oracle's layer on the same bf16 rows."""
    xq = example.xq
    K, I, N, Ip = 256, 512, 136, 544
    g = np.random.default_rng(5)
    codes, scales = f8.quantize_rows(g.standard_normal((M, K)))
    hg, hu = (xq.xq_f8_weights_import(*f8.quantize_blocks(g.standard_normal((I, K)) * 0.1)) for _ in range(2))
    ws = xq.new_f8_workspace(M, hg)
    h = torch.empty((M, I), dtype=torch.bfloat16, device="cuda")
    xq.xq_f8_gated(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), M, hg, hu, ws, out=h)
    wb = synth.weights(N, I, seed=3, tag="f8block")
    w4 = xq.xq_prepare_weights(wb, Ip)
    ws4 = xq.new_workspace(M, w4)
    out = torch.empty((M, N), dtype=torch.int16, device="cuda")
    xq.xq_expanded_linear(h, w4, out, ws4)
    assert xq.xq_poll_status(ws) == xq.OK and xq.xq_poll_status(ws4) == xq.OK
    hb = h.view(torch.int16).cpu().numpy().view(np.uint16)
    want = synth.bf16_bits_to_f32(oracle.expanded_linear(oracle.plan(I, Ip), hb, wb)[0]).astype(np.float64)
    got = synth.bf16_bits_to_f32(out.cpu().numpy().view(np.uint16)).astype(np.float64)
    assert np.linalg.norm(got - want) / np.linalg.norm(want) <= 2e-2


def test_norm_result_feeds_the_expanded_layer(example, oracle):
    """The norm's bf16 rows are the tokens of an expanded layer."""
    xq = example.xq
    M, K, N, Kp = 5, 512, 72, 544
    x = torch.from_numpy(np.random.default_rng(6).standard_normal((M, K))).to(torch.bfloat16).cuda()
    gamma = torch.ones(K, dtype=torch.bfloat16, device="cuda")
    y = torch.empty_like(x)
    xq.xq_f8_norm_quant(x, gamma, 1e-5, *xq.new_f8_rows(M, K), y=y)
    wb = synth.weights(N, K, seed=4, tag="f8norm")
    w4 = xq.xq_prepare_weights(wb, Kp)
    ws4 = xq.new_workspace(M, w4)
    out = torch.empty((M, N), dtype=torch.int16, device="cuda")
    xq.xq_expanded_linear(y, w4, out, ws4)
    assert xq.xq_poll_status(ws4) == xq.OK
    yb = y.view(torch.int16).cpu().numpy().view(np.uint16)
    want = synth.bf16_bits_to_f32(oracle.expanded_linear(oracle.plan(K, Kp), yb, wb)[0]).astype(np.float64)
    got = synth.bf16_bits_to_f32(out.cpu().numpy().view(np.uint16)).astype(np.float64)
    assert np.linalg.norm(got - want) / np.linalg.norm(want) <= 2e-2
