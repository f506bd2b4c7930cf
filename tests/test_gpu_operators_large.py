"""Group norm and block-sparse attention's gradients on maps of more than 2^31 elements, and the operators' first calls made by several host threads at once."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import paper_2304_04237_b200 as sa
from oracle import operators as ops
from test_gpu_norm import back, call, check

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def nothing_kept():
    """Leaves no memory in torch's cache, which other large tests look at."""
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def room(gigabytes):
    if torch.cuda.mem_get_info()[0] < gigabytes * 1e9:
        pytest.skip(f"needs {gigabytes} GB")


@pytest.mark.parametrize("shape", [(3, 1000, 1500, 512, 32), (290, 300, 300, 96, 8)], ids=str)
def test_norm_past_32_bits(shape):
    """2.3e9 and 2.5e9 elements; the last image against the definition.  The longest chain of additions is a thread's: 4286 rounds of the second shape (an image is
    one or two chunks), of values of either sign whose roundings have either sign: three times the root of their number in half steps, 200 of the 335 allowed."""
    B, H, W, C, groups = shape
    room(90)
    gen = torch.Generator(device="cuda").manual_seed(B)
    x, dy = (torch.randn(B, H, W, C, device="cuda", dtype=torch.bfloat16, generator=gen) for _ in range(2))
    gamma, beta = 1 + 0.1 * torch.randn(C, device="cuda", generator=gen), 0.1 * torch.randn(C, device="cuda", generator=gen)
    got = call(x, gamma, beta, groups, "silu", dy)
    for name in ("y", "dx"):
        assert all(torch.isfinite(image).all() for image in got[name])
    c = C // groups                                                            # the first and the last group
    for channels in (slice(0, c), slice(C - c, C)):
        g = channels.start // c
        part = [back(t[-1:, :, :, channels]) for t in (x, dy)]
        ref = ops.group_norm(part[0], back(gamma[channels]), back(beta[channels]), 1, 1e-5, "silu", part[1])
        last = {"y": got["y"][-1:, :, :, channels], "dx": got["dx"][-1:, :, :, channels], "mean": got["mean"][-1:, g:g + 1], "rstd": got["rstd"][-1:, g:g + 1]}
        check(last, ref, "bf16")
    # the weights' gradients, image by image in fp64
    want, size = (torch.zeros(2, C, device="cuda", dtype=torch.float64) for _ in range(2))
    for b in range(B):
        u = ((x[b].double().view(-1, groups, c) - got["mean"][b].double()[:, None]) * got["rstd"][b].double()[:, None]).view(-1, C)
        z = u * gamma.double() + beta.double()
        s = torch.sigmoid(z)
        dz = dy[b].double().view(-1, C) * (s + z * s * (1 - s))
        for i, t in enumerate((dz * u, dz)):
            want[i] += t.sum(0)
            size[i] += t.abs().sum(0)
    for i, name in enumerate(("dgamma", "dbeta")):
        assert ((got[name].double() - want[i]).abs() <= 2e-5 * size[i]).all()


def test_sparse_gradients_past_32_bits():
    """Maps of 2.3e9 elements: the last image as by itself."""
    B, H, W, heads, d, block = 140, 32, 1024, 8, 64, (32, 32)
    room(60)
    gen = torch.Generator(device="cuda").manual_seed(2)
    q, k, v, g = (torch.randn(B, H, W, heads, d, device="cuda", dtype=torch.bfloat16, generator=gen) for _ in range(4))
    idx = torch.randint(-1, 32, (B, heads, 32, 1), device="cuda", dtype=torch.int32, generator=gen)

    def run(q, k, v, g, idx):
        out, dq, dk, dv = (torch.full_like(q, float("nan")) for _ in range(4))
        lse = torch.empty(q.shape[:4], device="cuda")
        sa.slide_attn_sparse_forward(q, k, v, idx, block, out, lse)
        sa.slide_attn_sparse_backward(q, k, v, idx, block, out, lse, g, dq, dk, dv)
        return out, lse, dq, dk, dv

    whole = [t[-1:].clone() for t in run(q, k, v, g, idx)]
    alone = run(*(t[-1:].clone() for t in (q, k, v, g, idx)))
    assert all(torch.equal(a, b) for a, b in zip(whole, alone))


THREADS = r"""
import threading
import torch
import paper_2304_04237_b200 as sa

torch.cuda.init()
N = 8
gate = threading.Barrier(N)

def work(i, results, wait):
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        gen = torch.Generator(device="cuda").manual_seed(5)
        dtype = (torch.float32, torch.bfloat16)[i % 2]
        x, dy = (torch.randn(2, 24, 24, 2048, device="cuda", generator=gen).to(dtype) for _ in range(2))
        q, k, v, g = (torch.randn(1, 16, 16, 2, 64, device="cuda", generator=gen).to(dtype) for _ in range(4))
        new = lambda t: torch.zeros_like(t)
        y, dx, out, dq, dk, dv, z = new(x), new(x), new(q), new(q), new(q), new(q), new(q)
        mean, rstd = (torch.zeros(2, 2048, device="cuda") for _ in range(2))
        dgamma, dbeta = (torch.zeros(2048, device="cuda") for _ in range(2))
        lse, idx, rng = torch.zeros(1, 16, 16, 2, device="cuda"), torch.zeros(1, 2, 16, 3, device="cuda", dtype=torch.int32), torch.tensor([1, 2], device="cuda")
        stream.synchronize()
        if wait:
            gate.wait()
        sa.slide_attn_group_norm_forward(x, None, None, 2048, 1e-5, sa.ACT_SILU, y, mean, rstd)
        sa.slide_attn_group_norm_backward(x, None, None, 2048, sa.ACT_SILU, mean, rstd, dy, dx, dgamma, dbeta)
        sa.slide_attn_select_blocks(q, k, (4, 4), idx)
        sa.slide_attn_sparse_forward(q, k, v, idx, (4, 4), out, lse)
        sa.slide_attn_sparse_backward(q, k, v, idx, (4, 4), out, lse, g, dq, dk, dv)
        sa.slide_attn_dropout_forward(out, q, 0.3, sa.DROP_ELEMENTS, rng, z)
        stream.synchronize()
    results[i] = [t.clone() for t in (y, mean, rstd, dx, dgamma, dbeta, idx, out, lse, dq, dk, dv, z)]

first, later = [None] * N, [None] * N
threads = [threading.Thread(target=work, args=(i, first, True)) for i in range(N)]
[t.start() for t in threads]
[t.join() for t in threads]
torch.cuda.synchronize()
for i in range(N):
    work(i, later, False)
torch.cuda.synchronize()
assert all(torch.equal(a, b) for i in range(N) for a, b in zip(first[i], later[i]))
print("same")
"""


def test_first_calls_by_several_host_threads():
    """In a process of its own, where nothing has been called before: what a kernel asks for on its first call on a device is asked for by all of them."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", THREADS], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip().endswith("same"), r.stderr[-2000:]


@pytest.mark.parametrize("d", [16, 32])
def test_lists_that_mostly_name_the_same_blocks(d):
    """bf16, several heads: every list of a head names one block, most name a few, some none: more lists than a table of the keys' kernel holds (512)."""
    from test_gpu_sparse import call as attend, check as compare, inputs
    B, H, W, heads, block, top = 2, 48, 50, 3, (2, 2), 4
    q, k, v, g = inputs((B, H, W, heads, d), "bf16", seed=d)
    R = 24 * 25
    r = np.random.default_rng(d)
    idx = np.minimum(r.zipf(1.3, size=(B, heads, R, top)) - 1, R - 1).astype(np.int32)
    idx[:, :, :, 0] = 100 + np.arange(heads)[None, :, None]
    idx[:, :, ::11] = -1
    idx = torch.from_numpy(idx).cuda()
    got = attend(q, k, v, idx, block, g)
    compare(got, ops.sparse(back(q), back(k), back(v), idx.cpu().numpy(), block, back(g), back(got["out"])), "bf16")
