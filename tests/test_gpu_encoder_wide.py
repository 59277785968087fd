"""The encoder layers for rows wider than 8 KB, forward (more than a wavefront's registers) and backward (and more than 4096 columns,
whose sums of the parameters' gradients a block's wavefronts could not add up in LDS): the stages and gradients of
test_gpu_encoder.py and test_gpu_encoder_backward.py, with their bounds, for layers that take the block-per-row forms of the layer norm."""
import pytest
import torch

import paper_2006_16668_amd as moe
import test_gpu_encoder as forward
import test_gpu_encoder_backward as backward
from workloads import MoEConfig, make_encoder_weights, make_inputs, make_upstream

pytestmark = pytest.mark.gpu

# (config, sequences B, length L, heads, d): just over 8 KB, one to four vectors a thread backward, over 32 KB
CASES = [
    (MoEConfig("wide_f32", G=2, S=48, M=2052, H=64, E=4, C=24, act_dtype="f32", seed=61), 3, 32, 2, 16),
    (MoEConfig("wide_bf16", G=3, S=40, M=4104, H=136, E=5, C=20, act_dtype="bf16", seed=62), 4, 30, 3, 24),
    (MoEConfig("wider_f32", G=1, S=64, M=4100, H=32, E=4, C=32, act_dtype="f32", seed=63), 2, 32, 2, 16),
    (MoEConfig("widest_bf16", G=1, S=64, M=16392, H=64, E=4, C=40, act_dtype="bf16", seed=64), 2, 32, 2, 64),
]
ids = lambda v: v.name if isinstance(v, MoEConfig) else None


@pytest.mark.parametrize("cfg,B,L,heads,d", CASES, ids=ids)
def test_stages_and_pair(cfg, B, L, heads, d):
    forward.test_encoder_stages_and_pair(cfg, B, L, heads, d)


@pytest.mark.parametrize("cfg,B,L,heads,d", CASES, ids=ids)
def test_pair_backward(cfg, B, L, heads, d):
    backward.test_encoder_pair_backward(cfg, B, L, heads, d)


def test_the_same_bits_again():
    cfg, B, L, heads, d = CASES[1]
    dims, inp, w = moe.EncoderDims(B, L, heads, d), make_inputs(cfg, device="cuda:0"), make_encoder_weights(cfg, heads, d, device="cuda:0")
    dy, daux = make_upstream(cfg, device="cuda:0")
    (_, _, dx1, g1), (_, _, dx2, g2) = (backward._gpu_backward(cfg, dims, inp, w, dy, daux) for _ in range(2))
    assert torch.equal(dx1, dx2) and all(torch.equal(a, b) for k in ("ln_gamma", "ln_beta") for a, b in zip(g1[k], g2[k]))
