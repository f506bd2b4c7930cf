"""Dropout from the counter-based generator, with its residual and its gradient, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2304_04237_b200 as sa
from oracle import operators as ops

pytestmark = pytest.mark.gpu

TD = {"f32": torch.float32, "bf16": torch.bfloat16}
# the product and the sum in fp32 (the scale is off by 2^-24, product and sum are rounded once more), then the result's type
STEPS = {"f32": 3 * 2.0 ** -24, "bf16": 2.0 ** -8 + 3 * 2.0 ** -24}
SEED, OFFSET = 0x123456789ABCDEF, 0x0FEDCBA987654321


def rng(seed=SEED, offset=OFFSET):
    return torch.tensor([seed, offset], dtype=torch.int64, device="cuda")


def maps(shape, dtype, seed, n=2):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn(shape, device="cuda", generator=gen).to(TD[dtype]) for _ in range(n)]


def back(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("unit", [sa.DROP_ELEMENTS, sa.DROP_IMAGES])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.97, 1.0])
@pytest.mark.parametrize("shape", [(1,), (3,), (5, 1), (9, 7), (2, 13, 5, 24), (6, 4, 4, 32), (3, 40, 30, 8), (2, 8195)], ids=str)
def test_forward_and_backward(shape, p, unit, dtype):
    x, residual = maps(shape, dtype, 1)
    images = unit == sa.DROP_IMAGES
    scale = 1 / (1 - p) if p < 1 else 1.0
    for res in (residual, None):
        y = torch.full_like(x, float("nan"))
        sa.slide_attn_dropout_forward(x, res, p, unit, rng(), y)
        ref = ops.dropout(back(x), None if res is None else back(res), p, images, SEED, OFFSET)
        size = np.abs(back(x)) * scale + (0 if res is None else np.abs(back(res)))
        assert (np.abs(back(y) - ref) <= STEPS[dtype] * size).all()
    dx = torch.full_like(x, float("nan"))
    sa.slide_attn_dropout_backward(x, p, unit, rng(), dx)
    assert torch.equal(dx, y)


@pytest.mark.parametrize("unit", [sa.DROP_ELEMENTS, sa.DROP_IMAGES])
def test_in_place(unit):
    x, residual = maps((4, 11, 9, 16), "bf16", 2)
    want = torch.empty_like(x)
    sa.slide_attn_dropout_forward(x, residual, 0.3, unit, rng(), want)
    for which in (0, 1):
        a, b = x.clone(), residual.clone()
        sa.slide_attn_dropout_forward(a, b, 0.3, unit, rng(), (a, b)[which])
        assert torch.equal((a, b)[which], want)


def test_dropped_infinities_and_nans_do_not_matter():
    x, residual = maps((1000,), "f32", 3)
    mask = torch.from_numpy(ops.kept(1000, 0.5, SEED, OFFSET)).cuda()
    bad = torch.where(mask, x, torch.tensor(float("nan"), device="cuda"))
    bad[~mask & (torch.arange(1000, device="cuda") % 2 == 0)] = float("inf")
    y = torch.empty_like(x)
    sa.slide_attn_dropout_forward(bad, residual, 0.5, sa.DROP_ELEMENTS, rng(), y)
    assert torch.equal(y[~mask], residual[~mask]) and torch.isfinite(y).all()


@pytest.mark.parametrize("seed,offset", [(0, 0), (-1, -1), (2 ** 62 + 5, -(2 ** 62))])
def test_seeds_and_offsets_of_64_bits(seed, offset):
    x = torch.ones(4096, device="cuda")
    y = torch.empty_like(x)
    sa.slide_attn_dropout_forward(x, None, 0.5, sa.DROP_ELEMENTS, rng(seed, offset), y)
    assert ((back(y) != 0) == ops.kept(4096, 0.5, seed % 2 ** 64, offset % 2 ** 64)).all()


def test_elements_past_32_bits():
    """2^34 + 40 elements (bf16): the counter's upper word and offsets past 2^32 bytes.  Checked at the ends of the range and about 2^34."""
    n = 2 ** 34 + 40
    x = torch.ones(n, device="cuda", dtype=torch.bfloat16)
    sa.slide_attn_dropout_forward(x, None, 0.5, sa.DROP_ELEMENTS, rng(), x)
    for first in (0, 2 ** 31 - 64, 2 ** 32 - 64, 2 ** 34 - 64):
        count = min(256, n - first)
        assert ((back(x[first:first + count]) != 0) == ops.kept(count, 0.5, SEED, OFFSET, first=first)).all()
    del x
    torch.cuda.empty_cache()


def test_a_captured_call_draws_what_the_state_says_when_it_is_replayed():
    x, residual = maps((2, 9, 7, 16), "f32", 4)
    state, y, dx = rng(), torch.empty_like(x), torch.empty_like(x)
    sa.slide_attn_dropout_forward(x, residual, 0.4, sa.DROP_ELEMENTS, state, y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sa.slide_attn_dropout_forward(x, residual, 0.4, sa.DROP_ELEMENTS, state, y)
        sa.slide_attn_dropout_backward(x, 0.4, sa.DROP_ELEMENTS, state, dx)
        state[1] += 1
    for k in range(3):
        graph.replay()
        torch.cuda.synchronize()
        ref = ops.dropout(back(x), back(residual), 0.4, False, SEED, OFFSET + k)
        assert np.abs(back(y) - ref).max() < 1e-5 and np.abs(back(dx) + back(residual) - ref).max() < 1e-5
    del graph
