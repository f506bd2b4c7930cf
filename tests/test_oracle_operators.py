"""Pins of the operators' definitions (oracle/operators.py): published vectors, closed forms, library routines, central differences."""
import math

import numpy as np
import pytest
import torch

from oracle import operators as ops

RNG = np.random.default_rng


@pytest.mark.parametrize("counter,key,words", [      # known answers that the generator's authors publish with it
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
])
def test_generator_known_answers(counter, key, words):
    assert ops.philox(counter, key) == words


def test_kept_share_and_limits():
    n = 20000
    for p in (0.1, 0.5):
        share = ops.kept(n, p, 7, 9).mean()
        assert abs(share - (1 - p)) < 5 * math.sqrt(p * (1 - p) / n)
    assert ops.kept(100, 0.0, 1, 2).all() and not ops.kept(100, 1.0, 1, 2).any()
    assert (ops.kept(64, 0.5, 3, 4)[10:30] == ops.kept(20, 0.5, 3, 4, first=10)).all()
    assert (ops.kept(64, 0.5, 3, 4) != ops.kept(64, 0.5, 3, 5)).any() and (ops.kept(64, 0.5, 3, 4) != ops.kept(64, 0.5, 4, 4)).any()


@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
def test_norm_is_the_libraries(act):
    r = RNG(1)
    x, gamma, beta = r.normal(size=(2, 5, 4, 12)) + 3, r.normal(size=12), r.normal(size=12)
    t = torch.nn.functional.group_norm(torch.from_numpy(x).permute(0, 3, 1, 2), 4, torch.from_numpy(gamma), torch.from_numpy(beta), 1e-5)
    t = {"none": lambda z: z, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu}[act](t).permute(0, 2, 3, 1).numpy()
    assert np.allclose(ops.group_norm(x, gamma, beta, 4, 1e-5, act)["y"], t, atol=1e-12)


@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
def test_norm_gradients_are_differences(act):
    r = RNG(2)
    x, gamma, beta, dy = r.normal(size=(2, 3, 2, 8)), r.normal(size=8), r.normal(size=8), r.normal(size=(2, 3, 2, 8))
    got = ops.group_norm(x, gamma, beta, 4, 1e-5, act, dy)
    loss = lambda: float((ops.group_norm(x, gamma, beta, 4, 1e-5, act)["y"] * dy).sum())  # noqa: E731
    for name, t in (("dx", x), ("dgamma", gamma), ("dbeta", beta)):
        for at in np.ndindex(t.shape):
            keep, h = t[at], 1e-5
            t[at] = keep + h
            up = loss()
            t[at] = keep - h
            down = loss()
            t[at] = keep
            assert abs((up - down) / (2 * h) - got[name][at]) < 1e-7


def test_one_block_and_whole_lists_are_dense_attention():
    r = RNG(3)
    q, k, v = (r.normal(size=(1, 5, 6, 2, 8)) for _ in range(3))
    t = [torch.from_numpy(a).reshape(30, 2, 8).transpose(0, 1) for a in (q, k, v)]
    want = (torch.softmax(t[0] @ t[1].transpose(1, 2) / math.sqrt(8), -1) @ t[2]).transpose(0, 1).reshape(q.shape).numpy()
    for block, blocks in (((5, 6), 1), ((2, 4), 6)):
        idx = np.broadcast_to(np.arange(blocks)[::-1], (1, 2, blocks, blocks))
        assert np.allclose(ops.sparse(q, k, v, idx, block)["out"], want, atol=1e-13)


def test_lists_with_holes_and_repeats():
    r = RNG(4)
    q, k, v = (r.normal(size=(1, 4, 4, 1, 8)) for _ in range(3))
    idx = np.array([[-1, 7], [2, 2], [0, 3], [4, 1]], np.int32).reshape(1, 1, 4, 2)
    got = ops.sparse(q, k, v, idx, (2, 2))
    assert (got["out"][0, :2, :2] == 0).all() and np.isneginf(got["lse"][0, :2, :2]).all()
    once = ops.sparse(q, k, v, np.array([[0], [2], [0], [1]], np.int32).reshape(1, 1, 4, 1), (2, 2))
    assert np.allclose(got["out"][0, :2, 2:], once["out"][0, :2, 2:])                       # each pixel twice: the same weights
    assert np.allclose(got["lse"][0, :2, 2:], once["lse"][0, :2, 2:] + math.log(2))
    assert np.allclose(got["out"][0, 2:, 2:], once["out"][0, 2:, 2:])


def test_sparse_gradients_are_differences():
    r = RNG(5)
    q, k, v, g = (r.normal(size=(1, 3, 5, 2, 4)) for _ in range(4))
    idx = r.integers(-1, 6, size=(1, 2, 6, 3)).astype(np.int32)
    got = ops.sparse(q, k, v, idx, (2, 2), dout=g)
    loss = lambda: float((ops.sparse(q, k, v, idx, (2, 2))["out"] * g).sum())  # noqa: E731
    for name, t in (("dq", q), ("dk", k), ("dv", v)):
        for at in np.ndindex(t.shape):
            keep, h = t[at], 1e-5
            t[at] = keep + h
            up = loss()
            t[at] = keep - h
            down = loss()
            t[at] = keep
            assert abs((up - down) / (2 * h) - got[name][at]) < 1e-8
    for n in ("out", "dq", "dk", "dv"):
        assert (np.abs(got[n]) <= got[n + "_abs"] + 1e-12).all()


def test_select_order_ties_and_nan():
    q = np.ones((1, 2, 8, 1, 4))
    k = np.zeros((1, 2, 8, 1, 4))
    for s, value in enumerate((1.0, 3.0, 3.0, 2.0)):
        k[0, :, 2 * s:2 * s + 2] = value
    assert ops.select(q, k, (2, 2), 4)[0, 0].tolist() == [[1, 2, 3, 0]] * 4
    k[0, 0, 2, 0, 0] = np.nan
    assert ops.select(q, k, (2, 2), 4)[0, 0].tolist() == [[2, 3, 0, 1]] * 4
