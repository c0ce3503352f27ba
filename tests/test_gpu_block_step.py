"""Whole training steps of the classifier of bench.py --config block (products with activation and residual, a gated block,
softmax loss, gradients, their norm, the clipped update) against automatic differentiation in 64 bits on the CPU, within the
library's fp32 tolerance of 1e-4 of the largest value; eager and replayed from a graph."""
import os
import sys

import pytest
import torch
import torch.nn.functional as F

from gpu_util import TOL_F32

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))


@pytest.fixture(scope="module")
def B():
    assert torch.cuda.is_available()
    from paper_1504_04343_amd import binding
    return binding


def reference(weights, moments, x, label, max_norm, rate, momentum, decay):
    w = [t.detach().requires_grad_() for t in weights]
    r = F.relu(F.linear(x, w[0], w[1]))
    h = F.silu(F.linear(r, w[2])) * F.linear(r, w[3])
    y = F.linear(h, w[4]) + r
    loss = F.cross_entropy(F.linear(y, w[5], w[6]), label)
    grads = torch.autograd.grad(loss, w)
    norm = torch.sqrt(sum((g ** 2).sum() for g in grads))
    s = min(1.0, max_norm / float(norm))
    moments = [momentum * m + rate * (s * g + decay * t.detach()) for m, g, t in zip(moments, grads, w)]
    return float(loss.detach()), float(norm), [t.detach() - m for t, m in zip(w, moments)], moments


def close(name, got, want):
    off = float((got.cpu().double() - want).abs().max() / want.abs().max())
    assert off <= TOL_F32, (name, off)


@pytest.mark.parametrize("M", [3, 70, 200])
def test_steps_against_automatic_differentiation(B, M):
    from bench import Block
    blk = Block(B, torch, M, 120, 72, 100, 10, False, seed=M)
    weights, moments = [w.cpu().double() for w in blk.weights], [m.cpu().double() for m in blk.moments]
    for max_norm in (0.5, 100.0, 0.5):
        loss, norm, weights, moments = reference(weights, moments, blk.x.cpu().double(), blk.label.cpu().long(), max_norm, 0.1, 0.9,
                                                 0.01)
        blk.step(0.1, 0.9, 0.01, max_norm)
        assert abs(float(blk.loss) - loss) <= TOL_F32 * abs(loss)
        assert abs(float(blk.clip[0]) - norm) <= TOL_F32 * norm
        for i, (w, v) in enumerate(zip(weights, moments)):
            close("weight %d" % i, blk.weights[i], w)
            close("moment %d" % i, blk.moments[i], v)


@pytest.mark.parametrize("bf16", [False, True])
def test_the_step_from_a_graph(B, bf16):
    """Two blocks from the same seed, one stepped eagerly and one from a graph: the same bits after every step."""
    from bench import Block
    one, two = (Block(B, torch, 40, 136, 64, 96, 12, bf16, seed=5) for _ in range(2))
    one.step()
    two.step()
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            two.step()
    torch.cuda.synchronize()
    for r in range(3):
        one.step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(one.weights + one.moments + one.grads, two.weights + two.moments + two.grads):
            assert torch.equal(a, b), r
