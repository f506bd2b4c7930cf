"""Group norm on batches of many images, on both sides of each choice that the number and the size of the images make: images that one CTA keeps in registers and
larger ones, several chunks an image and one, 256 and 512 threads, chunks joined by the second pass and by a launch of their own.

Tolerances are those of test_gpu_norm: of the sums here the longest chain of additions is a thread's rounds (at most 38), the threads' rows (at most 64) and, in the
weights' sums, an eighth of the chunks (at most 56): 158 of the 335 steps of 2^-24 that are allowed."""
import numpy as np
import pytest
import torch

import paper_2304_04237_b200 as sa
from oracle import operators as ops
from test_gpu_norm import back, call, check, inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,shape", [
    # bf16, 96 channels: an image of up to 336 pixels in one CTA; beyond, each is one chunk from 297 images on (backward: from 223)
    ("bf16", (296, 20, 20, 96, 32)), ("bf16", (297, 20, 20, 96, 32)), ("bf16", (300, 20, 20, 96, 8)), ("bf16", (300, 1, 336, 96, 32)), ("bf16", (300, 1, 337, 96, 32)),
    ("bf16", (2, 1, 336, 96, 32)), ("bf16", (2, 1, 337, 96, 32)), ("bf16", (222, 13, 13, 96, 8)), ("bf16", (223, 13, 13, 96, 8)), ("bf16", (300, 28, 28, 96, 32)),
    # fp32: up to 168 pixels
    ("f32", (400, 14, 14, 96, 32)), ("f32", (400, 12, 14, 96, 32)), ("f32", (297, 13, 13, 96, 8)),
    # 512 threads, a pixel at a time: 8 pixels in one CTA; beyond, one chunk from 149 images on (backward: from 112)
    ("bf16", (148, 3, 3, 4096, 32)), ("bf16", (149, 3, 3, 4096, 32)), ("bf16", (160, 4, 4, 4096, 16)), ("bf16", (160, 2, 4, 4096, 32)), ("f32", (150, 4, 4, 2048, 64))], ids=str)
def test_many_images(dtype, shape):
    B, H, W, C, groups = shape
    x, dy, (gamma, beta) = inputs(B, H, W, C, dtype, seed=B + H * W)
    check(call(x, gamma, beta, groups, "silu", dy), ops.group_norm(back(x), back(gamma), back(beta), groups, 1e-5, "silu", back(dy)), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B", [1, 31, 257, 100000])
def test_weights_of_a_batch_of_single_pixels(B, dtype):
    """Equal gradients, whose roundings all go the same way.  32 of an eighth of the images are added up in fp32, which is off by 31 half steps at most, the rest in
    fp64; dz u has four roundings of its own (deviation, scale, product, rstd)."""
    C, groups = 32, 2
    x = inputs(B, 1, 1, C, dtype, seed=B)[0]
    dy = torch.full_like(x, 0.7)
    dx, y = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = (torch.empty(B, groups, device="cuda") for _ in range(2))
    dgamma, dbeta = (torch.empty(C, device="cuda") for _ in range(2))
    sa.slide_attn_group_norm_forward(x, None, None, groups, 1e-5, sa.ACT_NONE, y, mean, rstd)
    sa.slide_attn_group_norm_backward(x, None, None, groups, sa.ACT_NONE, mean, rstd, dy, dx, dgamma, dbeta)
    assert (np.abs(back(dbeta) - back(dy).sum((0, 1, 2))) <= 32 * 2.0 ** -24 * back(dbeta)).all()
    u = (back(x).reshape(B, groups, -1) - back(mean)[..., None]) * back(rstd)[..., None] * float(dy[0, 0, 0, 0])     # with the statistics that the call was given
    assert (np.abs(back(dgamma) - u.sum(0).ravel()) <= 36 * 2.0 ** -24 * np.abs(u).sum(0).ravel()).all()
