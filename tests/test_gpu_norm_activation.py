"""The activations behind the group norm and their slopes in steps of the result, tails included: z is known to the last bit from what the call itself gives, so only the
activation's arithmetic is compared.

Errors in units of u = 2^-24, half a step of fp32.  GELU, z times the integral up to z: the exponential's argument is off by three roundings, z^2 / 2 * 3 u of the
result, its approximation by 4 u; the reciprocal, its argument and what they move the polynomial by 4 u; the polynomial's roundings, up to twice as large as its value, and
its fit 8 u; three products 3 u: (20 + 1.5 z^2) u of the result and, of the slope, of the sum of its two terms' sizes.  SiLU, z g with g = 1 / (1 + exp(-z)): the exponential
is off by (4 + 1.5 |z|) u, of which g takes 1 - g; sum, reciprocal and product 4 u: (10 + 1.5 |z|) u.  Its slope, g (1 + z (1 - g)), has an error of 1 - g that
is g's, in units of 1: |z| g times that on top.  A result that is stored as bf16 is off by half a step, 2^-8, more."""
import math

import numpy as np
import pytest
import torch

import paper_2304_04237_b200 as sa

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TD = {"f32": torch.float32, "bf16": torch.bfloat16}
STORED = {"f32": U, "bf16": 2.0 ** -8}
ACT = {"silu": sa.ACT_SILU, "gelu": sa.ACT_GELU}
REACH = {"silu": 60.0, "gelu": 12.5}                       # results beyond are below fp32's normal numbers
erfc = np.vectorize(math.erfc, otypes=[np.float64])


def fit(z, dtype):
    return np.minimum(1.1e-7, 1.1e-4 * 0.5 * erfc(np.abs(z) / math.sqrt(2.0))) if dtype == "bf16" else 0.0


def value_and_limit(z, act, dtype):
    if act == "gelu":
        y = z * 0.5 * erfc(-z / math.sqrt(2.0))
        return y, (20 + 1.5 * z * z) * U * np.abs(y) + np.abs(z) * fit(z, dtype)
    y = z / (1.0 + np.exp(-z))
    return y, (10 + 1.5 * np.abs(z)) * U * np.abs(y)


def slope_and_limit(z, act, dtype):
    if act == "gelu":
        cdf, rest = 0.5 * erfc(-z / math.sqrt(2.0)), z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
        return cdf + rest, (20 + 1.5 * z * z) * U * (cdf + np.abs(rest)) + fit(z, dtype)
    g, less = 1.0 / (1.0 + np.exp(-z)), 1.0 / (1.0 + np.exp(z))                # 1 - g without cancellation
    own = (4 + (4 + 1.5 * np.abs(z)) * less) * U
    return g * (1 + z * less), (6 * U + own) * g * (1 + np.abs(z) * less) + np.abs(z) * g * g * own


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("pixels", [500, 20000])           # one launch, and several chunks
def test_values(pixels, act, dtype):
    r = np.random.default_rng(pixels)
    x = torch.from_numpy(r.uniform(-1, 1, size=(1, pixels, 1, 16))).to(TD[dtype]).cuda()
    gamma = torch.full((16,), REACH[act] * 0.57, device="cuda")               # x has a deviation of 0.577
    y, mean, rstd = torch.empty_like(x), torch.empty(1, 1, device="cuda"), torch.empty(1, 1, device="cuda")
    sa.slide_attn_group_norm_forward(x, gamma, None, 1, 1e-5, ACT[act], y, mean, rstd)
    z = ((x.float() - mean) * (gamma * rstd)).double().cpu().numpy()          # as the kernel rounds it, step by step
    assert z.min() < -0.95 * REACH[act] and z.max() > 0.95 * REACH[act]
    want, limit = value_and_limit(z, act, dtype)
    off = np.abs(y.double().cpu().numpy() - want) / (limit + STORED[dtype] * np.abs(want) + 2.0 ** -126)
    assert off.max() <= 1, (float(off.max()), float(z.flat[off.argmax()]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_slopes(act, dtype):
    """dbeta of a single pixel and a gradient of ones is the slope itself, in fp32 whatever the maps' type; with mean 0 and rstd 1, z is x."""
    x = torch.linspace(-REACH[act], REACH[act], 2048, device="cuda").to(TD[dtype]).view(1, 1, 1, -1)
    x[..., ::7] /= 16                                                          # more of them near zero
    dx, dgamma, dbeta = torch.empty_like(x), torch.empty(2048, device="cuda"), torch.empty(2048, device="cuda")
    mean, rstd = torch.zeros(1, 1, device="cuda"), torch.ones(1, 1, device="cuda")
    sa.slide_attn_group_norm_backward(x, None, None, 1, ACT[act], mean, rstd, torch.ones_like(x), dx, dgamma, dbeta)
    z = x.double().cpu().numpy().ravel()
    want, limit = slope_and_limit(z, act, dtype)
    off = np.abs(dbeta.double().cpu().numpy() - want) / (limit + 2.0 ** -126)
    assert off.max() <= 1, (float(off.max()), float(z[off.argmax()]))


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_values_that_are_not_finite(act):
    """+infinity keeps its value, a NaN stays one, and zero is zero."""
    x = torch.tensor([float("inf"), float("nan"), 0.0, -0.0, 1.0, -1.0, 2.0, 3.0], device="cuda").view(1, 1, 1, 8)
    dx, dgamma, dbeta = torch.empty_like(x), torch.empty(8, device="cuda"), torch.empty(8, device="cuda")
    mean, rstd = torch.zeros(1, 8, device="cuda"), torch.ones(1, 8, device="cuda")
    sa.slide_attn_group_norm_backward(x, None, None, 8, ACT[act], mean, rstd, torch.ones_like(x), dx, dgamma, dbeta)
    assert torch.isnan(dbeta[1]) and (dbeta[2:4] == 0.5).all() and torch.isfinite(dbeta[2:]).all()
