"""Group norm with an activation, forward and backward, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2304_04237_b200 as sa
from oracle import operators as ops

pytestmark = pytest.mark.gpu

TD = {"f32": torch.float32, "bf16": torch.bfloat16}
ACT = {"none": sa.ACT_NONE, "silu": sa.ACT_SILU, "gelu": sa.ACT_GELU}
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}        # of the rounding of a result to its type, relative
# fp32 arithmetic.  A thread adds up to a few hundred values one after the other, then 2^8 threads and 16 CTAs pairwise: a sum is off by at most
# 300 * 2^-24 = 1.8e-5 of the sum of absolute values, in the mean far less.  Elementwise: some ten operations of 2^-24, 2^-21 for exp and the slope.
SUMS, ELEMENTS = 2e-5, 2e-5


def inputs(B, H, W, C, dtype, seed, mean=0.5):
    r = np.random.default_rng(seed)
    x = r.normal(size=(B, H, W, C)) * (0.5 + r.random(C)) + mean * r.normal(size=C)
    to = lambda a: torch.from_numpy(a).to(TD[dtype]).cuda()  # noqa: E731
    return to(x), to(r.normal(size=(B, H, W, C))), [torch.from_numpy((c + 0.3 * r.normal(size=C)).astype(np.float32)).cuda() for c in (1.0, 0.0)]


def back(t):
    return t.double().cpu().numpy()


def call(x, gamma, beta, groups, act, dy=None, eps=1e-5):
    B, C = x.shape[0], x.shape[-1]
    y = torch.full_like(x, float("nan"))
    mean, rstd = (torch.full((B, groups), float("nan"), device="cuda") for _ in range(2))
    sa.slide_attn_group_norm_forward(x, gamma, beta, groups, eps, ACT[act], y, mean, rstd)
    got = {"y": y, "mean": mean, "rstd": rstd}
    if dy is not None:
        dx = torch.full_like(x, float("nan"))
        dgamma, dbeta = (torch.full((C,), float("nan"), device="cuda") for _ in range(2))
        sa.slide_attn_group_norm_backward(x, gamma, beta, groups, ACT[act], mean, rstd, dy, dx, dgamma, dbeta)
        got.update(dx=dx, dgamma=dgamma, dbeta=dbeta)
    return got


def check(got, ref, dtype, magnitude=1.0):
    for n in ("mean", "rstd"):
        assert (np.abs(back(got[n]) - ref[n]) <= ELEMENTS * np.maximum(magnitude, np.abs(ref[n]))).all(), n
    for n in ("y", "dx"):
        if n in got:
            off = np.abs(back(got[n]) - ref[n])
            limit = HALF_STEP[dtype] * np.abs(ref[n]) + ELEMENTS * np.maximum(magnitude, np.abs(ref[n])) * (ref["rstd"].max() if n == "dx" else 1)
            assert (off <= limit).all(), (n, float((off / limit).max()))
    for n in ("dgamma", "dbeta"):
        if n in got:
            off, limit = np.abs(back(got[n]) - ref[n]), SUMS * ref[n + "_abs"] + 1e-6
            assert (off <= limit).all(), (n, float((off / limit).max()))


SHAPES = [  # B, H, W, C, groups: one pixel; one group; a channel a group; groups that end inside 16 bytes; odd maps; several slabs; images of one row
    (1, 1, 1, 8, 1), (1, 1, 1, 64, 8), (3, 1, 5, 24, 3), (2, 7, 9, 96, 32), (1, 14, 14, 32, 8), (2, 13, 11, 40, 40), (1, 56, 56, 64, 1),
    (2, 28, 42, 192, 32), (1, 64, 64, 512, 32), (5, 3, 2, 16, 2), (1, 1, 300, 72, 9), (3, 17, 19, 200, 25)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_forward_and_backward(shape, act, dtype):
    B, H, W, C, groups = shape
    x, dy, (gamma, beta) = inputs(B, H, W, C, dtype, seed=H * W + C)
    check(call(x, gamma, beta, groups, act, dy), ops.group_norm(back(x), back(gamma), back(beta), groups, 1e-5, act, back(dy)), dtype)


@pytest.mark.parametrize("groups", [1, 8, 2048, 4096])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("half", [False, True])
def test_as_many_channels_as_there_may_be(dtype, groups, half):
    C = (2048 if dtype == "f32" else 4096) // (2 if half else 1) + (-8 * groups if half and groups < 9 else 0)
    x, dy, (gamma, beta) = inputs(2, 7, 5, C, dtype, seed=C)
    groups = min(groups, C)
    check(call(x, gamma, beta, groups, "silu", dy), ops.group_norm(back(x), back(gamma), back(beta), groups, 1e-5, "silu", back(dy)), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_group_over_a_large_map(dtype):
    """One group over 256 (512) channels and 160 x 160 pixels: 26 MB."""
    C = 256 if dtype == "f32" else 512
    x, dy, (gamma, beta) = inputs(1, 160, 160, C, dtype, seed=3)
    got = call(x, gamma, beta, 1, "silu", dy)
    check(got, ops.group_norm(back(x), back(gamma), back(beta), 1, 1e-5, "silu", back(dy)), dtype)


@pytest.mark.parametrize("affine", [(False, False), (True, False), (False, True)])
def test_without_gamma_or_beta(affine):
    x, dy, wb = inputs(2, 9, 8, 48, "f32", seed=4)
    gamma, beta = (t if on else None for t, on in zip(wb, affine))
    ref = ops.group_norm(back(x), None if gamma is None else back(gamma), None if beta is None else back(beta), 6, 1e-5, "gelu", back(dy))
    got = call(x, gamma, beta, 6, "gelu", dy)
    check(got, ref, "f32")
    dx = torch.empty_like(x)
    sa.slide_attn_group_norm_backward(x, gamma, beta, 6, sa.ACT_GELU, got["mean"], got["rstd"], dy, dx, None, None)
    assert torch.equal(dx, got["dx"])


@pytest.mark.parametrize("pad", [False, True])
def test_a_mean_far_from_zero(pad):
    """Deviations of 1 about a mean of 4096; with `pad`, the first rows are zeros, which are far from the others' mean."""
    r = np.random.default_rng(5)
    x = (4096 + r.normal(size=(2, 40, 24, 32))).astype(np.float32)
    if pad:
        x[:, :4] = 0
    ref = ops.group_norm(x, None, None, 4, 1e-5, "none")
    got = call(torch.from_numpy(x).cuda(), None, None, 4, "none")
    # The mean is off by no more than ELEMENTS of itself, 0.08 of what y is in units of; the variance, from deviations from it, by that squared.
    # Held to what a rounding of x alone costs: 2^-24 * 4096 = 2.4e-4 of a deviation, and four such steps in the mean.
    assert np.abs(back(got["mean"]) - ref["mean"]).max() <= 4 * 2.4e-4 * 2
    assert (np.abs(back(got["rstd"]) - ref["rstd"]) <= 1e-5 * ref["rstd"]).all()
    assert (np.abs(back(got["y"]) - ref["y"]) <= 8 * 2.4e-4 * ref["rstd"].max() + 1e-5 * np.abs(ref["y"])).all()


def test_constant_groups_and_nonfinite_values_stay_in_their_group():
    x, dy, _ = inputs(2, 6, 6, 32, "f32", seed=6)
    x[0, :, :, :8] = 3.0
    x[1, 2, 3, 9] = float("inf")
    x[1, 2, 3, 17] = float("nan")
    got = call(x, None, None, 4, "none", dy)
    assert (got["y"][0, :, :, :8] == 0).all() and torch.allclose(got["rstd"][0, 0], torch.tensor(1e-5 ** -0.5, device="cuda"))
    ref = ops.group_norm(back(x)[:, :, :, :8], None, None, 1, 1e-5, "none", back(dy)[:, :, :, :8])
    assert (np.abs(back(got["dx"][1, :, :, :8]) - ref["dx"][1]) <= 1e-5 * 8).all()
    for name in ("y", "dx"):
        bad = ~torch.isfinite(got[name])
        assert bad[1, :, :, 8:24].all() and not bad[0].any() and not bad[1, :, :, :8].any() and not bad[1, :, :, 24:].any()


def test_the_same_bits_every_time_and_nothing_beside_the_outputs():
    x, dy, (gamma, beta) = inputs(3, 30, 22, 96, "bf16", seed=7)
    want = call(x, gamma, beta, 32, "gelu", dy)
    room = torch.full((x.numel() + 2048,), 7.0, device="cuda", dtype=x.dtype)
    y = room[1024:1024 + x.numel()].view(x.shape)
    for _ in range(20):
        again = call(x, gamma, beta, 32, "gelu", dy)
        assert all(torch.equal(want[n], again[n]) for n in want)
    sa.slide_attn_group_norm_forward(x, gamma, beta, 32, 1e-5, sa.ACT_GELU, y, want["mean"], want["rstd"])
    assert torch.equal(y, want["y"]) and (room[:1024] == 7).all() and (room[-1024:] == 7).all()
