"""Block-sparse attention: choosing blocks, forward and backward, against the definitions in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2304_04237_b200 as sa
from oracle import operators as ops

pytestmark = pytest.mark.gpu

TD = {"f32": torch.float32, "bf16": torch.bfloat16}
# Errors relative to the sums of absolute values (`*_abs`).  fp32: of the nine products of three bf16 parts three are left out, 2^-23 of |q||k| at most, and the
# six that are added up are truncated to 2^-24 each: 2^-21 of sum |q||k| / sqrt(d), here up to some 15, which
# moves exponents by up to 7e-6; the exponent's own rounding 1e-6; the rest is a dozen steps of 2^-24.  bf16: one rounding (half a step of 2^-8) of
# each weight beside those, and of the result.
TERMS = {"f32": 2e-5, "bf16": 2.0 ** -8 + 2e-5}
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def back(t):
    return t.double().cpu().numpy()


def inputs(shape, dtype, seed, n=4):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn(shape, device="cuda", generator=gen).to(TD[dtype]) for _ in range(n)]


def blocks_of(H, W, block):
    return -(-H // block[0]) * -(-W // block[1])


def call(q, k, v, idx, block, dout=None):
    out = torch.full_like(q, float("nan"))
    lse = torch.full(q.shape[:4], float("nan"), device="cuda")
    sa.slide_attn_sparse_forward(q, k, v, idx, block, out, lse)
    got = {"out": out, "lse": lse}
    if dout is not None:
        grads = [torch.full_like(q, float("nan")) for _ in range(3)]
        sa.slide_attn_sparse_backward(q, k, v, idx, block, out, lse, dout, *grads)
        got.update(zip(("dq", "dk", "dv"), grads))
    return got


def check(got, ref, dtype, logits=1):
    """logits: how many times larger they are than the comment above says."""
    lse, want = back(got["lse"]), ref["lse"]
    assert (np.isneginf(lse) == np.isneginf(want)).all()
    fine = ~np.isneginf(want)
    assert (np.abs(lse - want)[fine] <= 2e-5 * np.maximum(1, np.abs(want[fine]))).all()
    for n in ("out", "dq", "dk", "dv"):
        if n in got:
            off = np.abs(back(got[n]) - ref[n])
            limit = (TERMS[dtype] + (logits - 1) * 1e-5) * ref[n + "_abs"] + HALF_STEP[dtype] * np.abs(ref[n]) + 1e-30
            assert (off <= limit).all(), (n, float((off / limit).max()))


CASES = [  # B, H, W, heads, d, block, top
    (1, 1, 1, 1, 16, (1, 1), 1),          # one token
    (1, 14, 14, 1, 32, (7, 7), 2),
    (2, 16, 16, 2, 32, (8, 8), 3),
    (1, 13, 19, 3, 16, (4, 5), 4),        # blocks that end with the map
    (2, 9, 23, 1, 64, (8, 8), 3),
    (1, 40, 33, 2, 32, (16, 12), 5),      # blocks of three tiles of rows
    (1, 1, 77, 2, 32, (1, 16), 3),        # a sequence
    (1, 37, 1, 1, 64, (32, 1), 2),
    (2, 20, 20, 1, 32, (5, 5), 16),       # every block
    (1, 64, 64, 1, 16, (32, 32), 2),      # the largest blocks
    (1, 12, 12, 2, 32, (3, 3), 1),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_forward_and_backward(case, dtype):
    B, H, W, heads, d, block, top = case
    q, k, v, g = inputs((B, H, W, heads, d), dtype, seed=H + W)
    R = blocks_of(H, W, block)
    gen = torch.Generator(device="cuda").manual_seed(9)
    idx = torch.rand(B, heads, R, R, device="cuda", generator=gen).argsort(-1)[..., :top].int().contiguous()
    got = call(q, k, v, idx, block, g)
    check(got, ops.sparse(back(q), back(k), back(v), idx.cpu().numpy(), block, back(g), back(got["out"])), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_lists_with_holes_repeats_and_numbers_that_are_no_block(dtype):
    B, H, W, heads, d, block = 2, 17, 22, 2, 32, (5, 6)
    q, k, v, g = inputs((B, H, W, heads, d), dtype, seed=21)
    R = blocks_of(H, W, block)
    gen = torch.Generator(device="cuda").manual_seed(3)
    idx = torch.randint(-4, R + 4, (B, heads, R, 7), device="cuda", generator=gen, dtype=torch.int32)
    idx[:, 0, 1] = -1                                              # queries that see nothing
    idx[1, 1, 2] = torch.iinfo(torch.int32).max
    idx[1, 1, 3] = torch.iinfo(torch.int32).min
    idx[0, 1, :, :3] = 4                                           # one block that all see three times over
    idx[idx == 6] = 5                                              # and one that nobody sees
    got = call(q, k, v, idx, block, g)
    check(got, ops.sparse(back(q), back(k), back(v), idx.cpu().numpy(), block, back(g), back(got["out"])), dtype)
    unseen = torch.tensor(ops.block_pixels(H, W, block)[6], device="cuda")
    for n in ("dk", "dv"):
        assert (got[n].view(B, H * W, heads, d)[:, unseen] == 0).all()
    alone = torch.tensor(ops.block_pixels(H, W, block)[1], device="cuda")
    for n in ("out", "dq"):
        assert (got[n].view(B, H * W, heads, d)[:, alone, 0] == 0).all()


def test_long_lists_of_queries():
    """More blocks of queries see a block than the keys' kernel lists at a time: 256 lists of 64 entries, all of them the same block."""
    B, H, W, heads, d, block = 1, 32, 32, 1, 16, (2, 2)
    q, k, v, g = inputs((B, H, W, heads, d), "f32", seed=5)
    idx = torch.full((1, 1, 256, 64), 100, device="cuda", dtype=torch.int32)
    idx[0, 0, ::3, 0] = 7
    got = call(q, k, v, idx, block, g)
    ref = ops.sparse(back(q), back(k), back(v), idx.cpu().numpy(), block, back(g), back(got["out"]))
    check(got, ref, "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [16, 64])
def test_more_blocks_than_the_gpu_takes_at_a_time(d, dtype):
    """Every CTA takes one block after the other; some blocks are seen by most of the others, some by none, and parts of blocks hold nothing."""
    B, H, W, heads, block = 30, 22, 33, 2, (9, 10)                # blocks of two tiles, of which those at the lower edge fill one
    q, k, v, g = inputs((B, H, W, heads, d), dtype, seed=13 + d)
    gen = torch.Generator(device="cuda").manual_seed(4)
    idx = torch.randint(-2, blocks_of(H, W, block), (B, heads, 12, 3), device="cuda", generator=gen, dtype=torch.int32)
    idx[::2, :, :, 0] = 5
    idx[idx == 2] = -1
    idx[3] = -1                                                    # an image where nobody sees anything
    got = call(q, k, v, idx, block, g)
    check(got, ops.sparse(back(q), back(k), back(v), idx.cpu().numpy(), block, back(g), back(got["out"])), dtype)
    assert all((got[n][3] == 0).all() for n in ("out", "dq", "dk", "dv")) and torch.isneginf(got["lse"][3]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_extreme_values(dtype):
    """Scores of -inf mask keys, all of a query's among them; scores of hundreds overflow nothing; what no list names does not matter."""
    B, H, W, heads, d, block = 1, 8, 12, 1, 32, (4, 4)
    q, k, v, g = inputs((B, H, W, heads, d), dtype, seed=6)
    idx = torch.tensor([[0, 1], [1, 2], [0, 3], [3, 3], [2, 0], [1, 0]], device="cuda", dtype=torch.int32).view(1, 1, 6, 2)
    q[0, :, :4] *= 30
    for t in (k, v):
        t[0, 4:, 4:8] = float("nan")                               # block 4, which nobody sees
        t[0, 4:, 8:] = float("inf")                                # block 5
    q[..., 0] = q[..., 0].abs() + 0.1
    k[0, 1, 1, 0, 0] = float("-inf")                               # one key of block 0
    got = call(q, k, v, idx, block)
    kr = back(k)
    ref = ops.sparse(back(q), kr, back(v), idx.cpu().numpy(), block)
    for n in ("out", "lse"):
        assert np.isfinite(back(got[n])).all()
    check(got, ref, dtype, logits=30)
    k[0, 4:, :4, 0, 0] = float("-inf")                             # all of block 3: the queries of block 3 see nothing else
    got = call(q, k, v, idx, block, g)
    assert (got["out"][0, 4:, :4] == 0).all() and torch.isneginf(got["lse"][0, 4:, :4]).all()
    assert torch.isfinite(got["out"]).all() and torch.isfinite(got["dv"]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", CASES + [(2, 128, 128, 1, 16, (4, 4), 64)], ids=str)
def test_select(case, dtype):
    B, H, W, heads, d, block, top = case
    q, k = inputs((B, H, W, heads, d), dtype, seed=H * W, n=2)
    idx = torch.full((B, heads, blocks_of(H, W, block), top), -7, device="cuda", dtype=torch.int32)
    sa.slide_attn_select_blocks(q, k, block, idx)
    assert (idx.cpu().numpy() == ops.select(back(q), back(k), block, top)).all()


def test_select_ties_infinities_and_nans():
    B, H, W, heads, d, block = 1, 8, 16, 2, 16, (4, 4)
    q, k = inputs((B, H, W, heads, d), "f32", seed=8, n=2)
    k[0, :4, 4:8] = k[0, :4, :4]                                   # blocks 0 and 1 alike
    k[0, 4:, 12:] = 0
    k[0, 4:, 8:12] = -0.0                                          # blocks 6 and 7: zero
    k[0, 5, 1, 0, 3] = float("nan")                                # block 4 of head 0
    q[0, :4, :4, 1] = 0                                            # a block of queries whose scores are all zero
    k[0, 6, 6, 1, 2] = float("inf")                                # block 5 of head 1
    idx = torch.empty(1, heads, 8, 8, device="cuda", dtype=torch.int32)
    sa.slide_attn_select_blocks(q, k, block, idx)
    with np.errstate(invalid="ignore"):
        want = ops.select(back(q), back(k), block, 8)
    assert (idx.cpu().numpy() == want).all()


def test_offsets_past_32_bits():
    """Maps of 2.3e9 elements: the last image as by itself."""
    B, H, W, heads, d, block = 140, 32, 1024, 8, 64, (32, 32)
    shape = (B, H, W, heads, d)
    free, _ = torch.cuda.mem_get_info()
    if free < 30e9:
        pytest.skip("needs 24 GB")
    gen = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (torch.randn(shape, device="cuda", dtype=torch.bfloat16, generator=gen) for _ in range(3))
    idx = torch.empty(B, heads, 32, 1, device="cuda", dtype=torch.int32)
    sa.slide_attn_select_blocks(q, k, block, idx)
    out = torch.empty_like(q)
    lse = torch.empty(shape[:4], device="cuda")
    sa.slide_attn_sparse_forward(q, k, v, idx, block, out, lse)
    part = [t[-1:].clone() for t in (q, k, v)]
    idx1, out1, lse1 = torch.empty_like(idx[-1:]), torch.empty_like(part[0]), torch.empty_like(lse[-1:])
    sa.slide_attn_select_blocks(part[0], part[1], block, idx1)
    sa.slide_attn_sparse_forward(*part, idx1, block, out1, lse1)
    assert torch.equal(idx1, idx[-1:]) and torch.equal(out1, out[-1:]) and torch.equal(lse1, lse[-1:])
    del q, k, v, out, part
    torch.cuda.empty_cache()


def test_the_same_bits_every_time_and_nothing_beside_the_outputs():
    B, H, W, heads, d, block = 2, 30, 26, 2, 32, (7, 7)
    q, k, v, g = inputs((B, H, W, heads, d), "bf16", seed=11)
    R = blocks_of(H, W, block)
    idx = torch.randint(-1, R, (B, heads, R, 4), device="cuda", dtype=torch.int32)
    want = call(q, k, v, idx, block, g)
    for _ in range(20):
        again = call(q, k, v, idx, block, g)
        assert all(torch.equal(want[n], again[n]) for n in want)
    n, room = q.numel(), [torch.full((q.numel() + 2048,), 7.0, device="cuda", dtype=q.dtype) for _ in range(3)]
    views = [r[1024:1024 + n].view(q.shape) for r in room]
    sa.slide_attn_sparse_backward(q, k, v, idx, block, want["out"], want["lse"], g, *views)
    for name, view, r in zip(("dq", "dk", "dv"), views, room):
        assert torch.equal(view, want[name]) and (r[:1024] == 7).all() and (r[-1024:] == 7).all()
