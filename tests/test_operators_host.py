"""What the operators' entry points refuse, checked without a GPU: every call here is turned down before anything is launched."""
import ctypes

import pytest
import torch

import paper_2304_04237_b200 as sa
from paper_2304_04237_b200 import binding

A, B2, C2, D2, E2, F2, G2, H2, I2, J2, K2 = (i << 32 for i in range(1, 12))     # addresses that nothing reads
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    from paper_2304_04237_b200 import build
    build.build()
    return binding.load()


def norm(lib, x=A, gamma=B2, beta=C2, y=D2, mean=E2, rstd=F2, B=2, H=40, W=40, C=32, groups=4, eps=1e-5, act=0, dtype=0,
         ws=G2, size=BIG):
    return lib.slide_attn_group_norm_forward(x, gamma, beta, y, mean, rstd, B, H, W, C, groups, eps, act, dtype, ws, size, None)


def norm_back(lib, x=A, gamma=B2, beta=C2, mean=D2, rstd=E2, dy=F2, dx=G2, dgamma=H2, dbeta=I2, B=2, H=4, W=4, C=32, groups=4, act=0, dtype=0, ws=J2,
              size=BIG):
    return lib.slide_attn_group_norm_backward(x, gamma, beta, mean, rstd, dy, dx, dgamma, dbeta, B, H, W, C, groups, act, dtype, ws, size, None)


def drop(lib, x=A, residual=B2, y=C2, images=2, per_image=10, p=0.5, unit=0, rng=D2, dtype=0):
    return lib.slide_attn_dropout_forward(x, residual, y, images, per_image, p, unit, rng, dtype, None)


def select(lib, q=A, k=B2, idx=C2, B=2, H=8, W=8, heads=2, d=32, bh=4, bw=4, top=2, dtype=0, ws=D2, size=BIG):
    return lib.slide_attn_select_blocks(q, k, idx, B, H, W, heads, d, bh, bw, top, dtype, ws, size, None)


def sparse(lib, q=A, k=B2, v=C2, idx=D2, out=E2, lse=F2, B=2, H=8, W=8, heads=2, d=32, bh=4, bw=4, top=2, dtype=0):
    return lib.slide_attn_sparse_forward(q, k, v, idx, out, lse, B, H, W, heads, d, bh, bw, top, dtype, None)


def sparse_back(lib, q=A, k=B2, v=C2, idx=D2, out=E2, lse=F2, dout=G2, dq=H2, dk=I2, dv=J2, B=2, H=8, W=8, heads=2, d=32, bh=4, bw=4, top=2, dtype=0,
                ws=K2, size=BIG):
    return lib.slide_attn_sparse_backward(q, k, v, idx, out, lse, dout, dq, dk, dv, B, H, W, heads, d, bh, bw, top, dtype, ws, size, None)


ARG, UNS, ALIGN = sa.ERR_INVALID_ARG, sa.ERR_UNSUPPORTED, sa.ERR_ALIGNMENT
NAN, INF = float("nan"), float("inf")
MAP = [dict(B=0), dict(H=0), dict(W=-1), dict(dtype=2)]
SPARSE = [(c, ARG) for c in MAP + [dict(heads=0), dict(bh=0), dict(bw=-4), dict(top=0)]] + [
    (dict(d=8), UNS), (dict(d=48), UNS), (dict(d=128), UNS), (dict(bh=33), UNS), (dict(bw=64), UNS), (dict(top=65), UNS),
    (dict(H=64, W=64, bh=1, bw=2), UNS), (dict(H=1 << 30, W=1 << 30), UNS), (dict(B=1 << 30, heads=64), UNS),
    (dict(B=1, heads=1 << 25), UNS)]

CASES = {
    norm: [(c, ARG) for c in MAP + [dict(C=0), dict(groups=0), dict(x=None), dict(y=None), dict(mean=None), dict(rstd=None), dict(eps=-1.0), dict(eps=NAN),
                                    dict(eps=INF), dict(act=3), dict(act=-1), dict(y=A), dict(y=B2), dict(mean=A), dict(mean=F2), dict(rstd=D2), dict(ws=None), dict(size=8),
                                    dict(ws=A), dict(ws=D2)]] +
          [(dict(C=36), UNS), (dict(groups=3), UNS), (dict(C=20, groups=5), UNS), (dict(C=8192, groups=1), UNS), (dict(C=4096, groups=1), UNS),
           (dict(C=8192, groups=1, dtype=1), UNS), (dict(H=1 << 16, W=1 << 16), UNS), (dict(B=1 << 30, H=1 << 10, W=1 << 10), UNS),
           (dict(x=A + 8), ALIGN), (dict(gamma=B2 + 4), ALIGN), (dict(y=D2 + 2), ALIGN), (dict(mean=E2 + 4), ALIGN), (dict(ws=G2 + 8), ALIGN)],
    norm_back: [(c, ARG) for c in MAP + [dict(x=None), dict(mean=None), dict(rstd=None), dict(dy=None), dict(dx=None), dict(dgamma=None), dict(dbeta=None),
                                         dict(ws=None), dict(size=2 * 4 * 8 + 2 * 2 * 32 * 4 - 1), dict(act=7), dict(dx=A), dict(dx=F2), dict(dgamma=I2),
                                         dict(dgamma=G2), dict(ws=A), dict(ws=I2)]] +
               [(dict(groups=5), UNS), (dict(C=12, groups=1), UNS), (dict(ws=J2 + 4), ALIGN), (dict(dx=G2 + 8), ALIGN), (dict(dbeta=I2 + 4), ALIGN)],
    drop: [(c, ARG) for c in [dict(x=None), dict(y=None), dict(rng=None), dict(images=0), dict(per_image=0), dict(dtype=5), dict(unit=2), dict(p=-0.1),
                              dict(p=1.01), dict(p=NAN), dict(y=D2)]] +
          [(dict(images=1 << 40, per_image=2), UNS), (dict(images=1 << 31, per_image=8, unit=1), UNS),
           (dict(x=A + 4), ALIGN), (dict(residual=B2 + 8), ALIGN), (dict(y=C2 + 2), ALIGN), (dict(rng=D2 + 4), ALIGN)],
    select: SPARSE + [(dict(B=1 << 20, heads=200, d=64), UNS)] + [(c, ARG) for c in [dict(q=None), dict(k=None), dict(idx=None), dict(ws=None), dict(top=5), dict(size=2 * 8 * 2 * 2 * 4 * 32 - 1),
                                         dict(idx=A), dict(ws=B2), dict(ws=C2)]] + [(dict(q=A + 8), ALIGN), (dict(idx=C2 + 4), ALIGN), (dict(ws=D2 + 8), ALIGN)],
    sparse: SPARSE + [(c, ARG) for c in [dict(q=None), dict(k=None), dict(v=None), dict(idx=None), dict(out=None), dict(lse=None), dict(out=A), dict(out=F2),
                                         dict(lse=C2)]] + [(dict(v=C2 + 8), ALIGN), (dict(lse=F2 + 4), ALIGN)],
    sparse_back: SPARSE + [(c, ARG) for c in [dict(q=None), dict(out=None), dict(lse=None), dict(dout=None), dict(dq=None), dict(dk=None), dict(dv=None),
                                              dict(ws=None), dict(size=2 * 4 * 2 * 64 * 2 + 4 * (1 + 4 * (5 + 8)) - 1), dict(dq=A), dict(dk=G2), dict(dv=I2), dict(dq=J2), dict(ws=F2),
                                              dict(ws=H2)]] + [(dict(dk=I2 + 8), ALIGN), (dict(ws=K2 + 4), ALIGN)],
}


# Outputs that share a part of their memory with another tensor: the last 16 bytes of one, or a place inside it.  Bytes of a tensor of `norm`, ...
NORM, BACK, DROP, SPARSE_MAP = 2 * 40 * 40 * 32 * 4, 2 * 4 * 4 * 32 * 4, 2 * 12 * 4, 2 * 8 * 8 * 2 * 32 * 4
PARTS = [(norm, dict(y=A + NORM - 16)), (norm, dict(mean=D2 + 64)), (norm, dict(rstd=E2 + 16)), (norm, dict(ws=F2 + 16)), (norm, dict(y=C2 - NORM + 16)),
         (norm_back, dict(dx=F2 + BACK - 16)), (norm_back, dict(dgamma=I2 + 64)), (norm_back, dict(dx=J2 - 16)), (norm_back, dict(ws=E2 + 16)),
         (drop, dict(per_image=12, y=A + DROP - 16)), (drop, dict(per_image=12, y=A, residual=A + 16)), (drop, dict(per_image=12, y=B2 - 16)),
         (drop, dict(per_image=12, rng=C2 + 8)), (drop, dict(per_image=12, y=D2 - DROP + 16)),
         (select, dict(idx=A + SPARSE_MAP - 16)), (select, dict(ws=B2 + 16)), (select, dict(idx=D2 + 64)),
         (sparse, dict(out=C2 - 16)), (sparse, dict(lse=E2 + SPARSE_MAP - 16)), (sparse, dict(out=D2 - 16)),
         (sparse_back, dict(dk=H2 + 16)), (sparse_back, dict(dv=G2 + SPARSE_MAP - 16)), (sparse_back, dict(ws=F2 - 16)), (sparse_back, dict(ws=J2 + 16)),
         (sparse_back, dict(dq=D2 - 16))]


@pytest.mark.parametrize("call,change", PARTS, ids=lambda v: getattr(v, "__name__", None) or str(v))
def test_outputs_that_share_memory(lib, call, change):
    assert call(lib, **change) == ARG


def test_neighbours_share_nothing(lib):
    """Outputs that begin where an input ends, and the other way round, are fine."""
    if torch.cuda.is_available():
        pytest.skip("a device is present")
    fine = (sa.ERR_CUDA, sa.ERR_ARCH)
    assert norm(lib, y=A + NORM) in fine and norm(lib, y=C2 - NORM) in fine
    assert drop(lib, per_image=12, y=A + DROP) in fine and drop(lib, per_image=12, rng=C2 + DROP) in fine
    assert sparse(lib, out=C2 + SPARSE_MAP) in fine and sparse_back(lib, dk=H2 + SPARSE_MAP, dv=H2 - SPARSE_MAP) in fine


@pytest.mark.parametrize("call,change,status", [(f, c, s) for f, cases in CASES.items() for c, s in cases],
                         ids=lambda v: getattr(v, "__name__", None) or str(v))
def test_refusals(lib, call, change, status):
    assert call(lib, **change) == status


def test_accepted_arguments_reach_the_device_check(lib):
    """The calls that the refusals change one argument of are themselves fine: without a device they get as far as looking for it."""
    if torch.cuda.is_available():
        pytest.skip("a device is present")
    for call in CASES:
        assert call(lib) in (sa.ERR_CUDA, sa.ERR_ARCH)
    assert norm(lib, H=4, W=4, ws=None, size=0) in (sa.ERR_CUDA, sa.ERR_ARCH)
    assert norm(lib, gamma=None, beta=None) in (sa.ERR_CUDA, sa.ERR_ARCH)
    assert norm_back(lib, dgamma=None, dbeta=None) in (sa.ERR_CUDA, sa.ERR_ARCH)
    for same in (dict(y=A), dict(y=B2), dict(residual=None, y=A)):
        assert drop(lib, **same) in (sa.ERR_CUDA, sa.ERR_ARCH)


def test_workspace_sizes(lib):
    n = ctypes.c_size_t()
    assert lib.slide_attn_group_norm_workspace(3, 5, 7, 48, 6, 1, 0, ctypes.byref(n)) == sa.OK and n.value == 0
    assert lib.slide_attn_group_norm_workspace(3, 5, 7, 48, 6, 1, 1, ctypes.byref(n)) == sa.OK and n.value == 8 * 3 * 6 + 2 * 4 * 3 * 48
    assert lib.slide_attn_select_workspace(3, 9, 7, 2, 16, 4, 4, ctypes.byref(n)) == sa.OK and n.value == 2 * 8 * 3 * 2 * 6 * 16
    assert lib.slide_attn_sparse_workspace(3, 9, 7, 2, 16, 4, 4, 3, ctypes.byref(n)) == sa.OK and n.value == 2 * 4 * 3 * 63 * 2 + 4 * (1 + 6 * (7 + 18))
    assert lib.slide_attn_group_norm_workspace(3, 5, 7, 48, 7, 1, 0, ctypes.byref(n)) == sa.ERR_UNSUPPORTED
    assert lib.slide_attn_select_workspace(3, 9, 7, 2, 8, 4, 4, ctypes.byref(n)) == sa.ERR_UNSUPPORTED
    assert lib.slide_attn_sparse_workspace(3, 9, 7, 2, 16, 4, 4, 3, None) == sa.ERR_INVALID_ARG
    assert lib.slide_attn_sparse_workspace(3, 9, 7, 2, 16, 4, 4, 65, ctypes.byref(n)) == sa.ERR_UNSUPPORTED


def test_binding_refuses_what_it_can_see(lib):
    x = torch.zeros(1, 4, 4, 32)
    s, rng = torch.zeros(1, 4), torch.zeros(2, dtype=torch.int64)
    with pytest.raises(ValueError):                                  # host tensors
        sa.slide_attn_group_norm_forward(x, None, None, 4, 1e-5, sa.ACT_NONE, torch.zeros_like(x), s, s.clone())
    with pytest.raises(ValueError):
        sa.slide_attn_group_norm_forward(x.half(), None, None, 4, 1e-5, sa.ACT_NONE, x.half(), s, s)
    with pytest.raises(ValueError):                                  # mean of another shape
        sa.slide_attn_group_norm_forward(x, None, None, 8, 1e-5, sa.ACT_NONE, torch.zeros_like(x), s, s.clone())
    with pytest.raises(ValueError):
        sa.slide_attn_dropout_forward(x, None, 0.5, sa.DROP_ELEMENTS, torch.zeros(3, dtype=torch.int64), x)
    with pytest.raises(ValueError):
        sa.slide_attn_dropout_forward(x, torch.zeros(1, 4, 4, 31), 0.5, sa.DROP_ELEMENTS, rng, x)
    with pytest.raises(ValueError):
        sa.slide_attn_dropout_backward(x[:0], 0.5, sa.DROP_ELEMENTS, rng, x[:0])
    q = torch.zeros(1, 8, 8, 2, 16)
    for idx in (torch.zeros(1, 2, 3, 2, dtype=torch.int32), torch.zeros(1, 2, 4, 2, dtype=torch.int64)):
        with pytest.raises(ValueError):
            sa.slide_attn_select_blocks(q, q, (4, 4), idx)
        with pytest.raises(ValueError):
            sa.slide_attn_sparse_forward(q, q, q, idx, (4, 4), torch.zeros_like(q), torch.zeros(1, 8, 8, 2))
