"""The operators as they are used together: a residual block with a norm ahead of its projections, attention over chosen blocks (or the
local attention) and dropout behind them; forward, backward, captured, on other streams."""
import numpy as np
import pytest
import torch

import paper_2304_04237_b200 as sa
from oracle import operators as ops

pytestmark = pytest.mark.gpu

B, H, W, HEADS, D, GROUPS, BLOCK, TOP, P = 2, 21, 27, 2, 32, 16, (7, 9), 3, 0.2
C = HEADS * D


def back(t):
    return t.double().cpu().numpy()


class Net:
    """y = x + dropout(attention(norm(x) W_qkv) W_o) with bf16 maps, and the gradients down to what the norm gives."""

    def __init__(self, seed):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        normal = lambda *s: torch.randn(*s, device="cuda", generator=gen)  # noqa: E731
        self.ctx = sa.slide_attn_create(B, H, W, HEADS, D, 3, torch.bfloat16, False)
        self.x, self.dy = (normal(B, H, W, C).bfloat16() for _ in range(2))
        self.gamma, self.beta = 1 + 0.1 * normal(C), 0.1 * normal(C)
        self.w_qkv, self.w_o = normal(3, C, C) / C ** 0.5, normal(1, C, C) / C ** 0.5
        self.state = torch.tensor([seed, 17], dtype=torch.int64, device="cuda")
        empty = lambda *s, t=torch.bfloat16: torch.full(s, float("nan"), device="cuda", dtype=t)  # noqa: E731
        self.n, self.o, self.y, self.do, self.dn, self.dx = (empty(B, H, W, C) for _ in range(6))
        self.mean, self.rstd = (empty(B, GROUPS, t=torch.float32) for _ in range(2))
        self.q, self.k, self.v, self.z, self.dz, self.dq, self.dk, self.dv = (empty(B, H, W, HEADS, D) for _ in range(8))
        self.lse = empty(B, H, W, HEADS, t=torch.float32)
        self.idx = torch.full((B, HEADS, 9, TOP), -1, device="cuda", dtype=torch.int32)
        self.dgamma, self.dbeta = (empty(C, t=torch.float32) for _ in range(2))

    def run(self, stream=None):
        sa.slide_attn_group_norm_forward(self.x, self.gamma, self.beta, GROUPS, 1e-5, sa.ACT_SILU, self.n, self.mean, self.rstd, stream=stream)
        sa.slide_attn_project(self.ctx, self.n, self.w_qkv, [self.q, self.k, self.v], stream=stream)
        sa.slide_attn_select_blocks(self.q, self.k, BLOCK, self.idx, stream=stream)
        sa.slide_attn_sparse_forward(self.q, self.k, self.v, self.idx, BLOCK, self.z, self.lse, stream=stream)
        sa.slide_attn_project(self.ctx, self.z, self.w_o, [self.o], stream=stream)
        sa.slide_attn_dropout_forward(self.o, self.x, P, sa.DROP_ELEMENTS, self.state, self.y, stream=stream)
        # backward; a projection's gradient of its input is a projection with the transposed weights
        sa.slide_attn_dropout_backward(self.dy, P, sa.DROP_ELEMENTS, self.state, self.do, stream=stream)
        sa.slide_attn_project(self.ctx, self.do, self.w_o_t, [self.dz], stream=stream)
        sa.slide_attn_sparse_backward(self.q, self.k, self.v, self.idx, BLOCK, self.z, self.lse, self.dz, self.dq, self.dk, self.dv, stream=stream)
        sa.slide_attn_project(self.ctx, self.dq, self.w_q_t, [self.dn], stream=stream)
        sa.slide_attn_group_norm_backward(self.x, self.gamma, self.beta, GROUPS, sa.ACT_SILU, self.mean, self.rstd, self.dn, self.dx, self.dgamma,
                                          self.dbeta, stream=stream)

    @property
    def results(self):
        return [self.n, self.mean, self.rstd, self.idx, self.z, self.lse, self.y, self.do, self.dq, self.dk, self.dv, self.dx, self.dgamma, self.dbeta]

    def transposes(self):
        self.w_o_t, self.w_q_t = self.w_o.transpose(1, 2).contiguous(), self.w_qkv[:1].transpose(1, 2).contiguous()
        return self


def test_each_stage_against_its_definition():
    net = Net(1).transposes()
    net.run()
    torch.cuda.synchronize()
    bf = 2.0 ** -8
    ref = ops.group_norm(back(net.x), back(net.gamma), back(net.beta), GROUPS, 1e-5, "silu", back(net.dn))
    assert (np.abs(back(net.n) - ref["y"]) <= bf * np.abs(ref["y"]) + 2e-5 * np.maximum(1, np.abs(ref["y"]))).all()
    assert (np.abs(back(net.dx) - ref["dx"]) <= bf * np.abs(ref["dx"]) + 2e-5 * ref["rstd"].max() * np.maximum(1, np.abs(ref["dx"]))).all()
    assert (np.abs(back(net.dgamma) - ref["dgamma"]) <= 2e-5 * ref["dgamma_abs"] + 1e-6).all()
    assert (net.idx.cpu().numpy() == ops.select(back(net.q), back(net.k), BLOCK, TOP)).all()
    at = ops.sparse(back(net.q), back(net.k), back(net.v), net.idx.cpu().numpy(), BLOCK, back(net.dz), back(net.z))
    for name, t in (("out", net.z), ("dq", net.dq), ("dk", net.dk), ("dv", net.dv)):
        assert (np.abs(back(t) - at[name]) <= (bf + 2e-5) * at[name + "_abs"] + bf * np.abs(at[name])).all(), name
    y = ops.dropout(back(net.o), back(net.x), P, False, 1, 17)
    assert (np.abs(back(net.y) - y) <= (bf + 1e-6) * (np.abs(back(net.o)) / (1 - P) + np.abs(back(net.x)))).all()
    assert sa.slide_attn_query_status(net.ctx) == sa.OK
    sa.slide_attn_destroy(net.ctx)


def test_beside_the_local_attention_and_its_block():
    """A norm ahead of slide_attn_block_forward and stochastic depth behind it: the kernels of both follow one another without waiting on the host."""
    net = Net(2).transposes()
    k2 = 9
    wk, wv = (torch.eye(k2, device="cuda").repeat(C, 1, 1).contiguous() for _ in range(2))
    want = []
    for wait in (True, False):
        for t in (net.n, net.o, net.y):
            t.fill_(float("nan"))
        for _ in range(3):
            sa.slide_attn_group_norm_forward(net.x, net.gamma, net.beta, GROUPS, 1e-5, sa.ACT_NONE, net.n, net.mean, net.rstd)
            if wait:
                torch.cuda.synchronize()
            sa.slide_attn_block_forward(net.ctx, net.n, net.w_qkv, net.w_o[0], wk, wv, None, net.o)
            if wait:
                torch.cuda.synchronize()
            sa.slide_attn_dropout_forward(net.o, net.x, 0.5, sa.DROP_IMAGES, net.state, net.y)
        torch.cuda.synchronize()
        want.append([t.clone() for t in (net.n, net.o, net.y)])
    assert all(torch.equal(a, b) and torch.isfinite(a).all() for a, b in zip(*want))
    sa.slide_attn_destroy(net.ctx)


def test_capture_replay_and_streams():
    nets = [Net(3).transposes(), Net(4).transposes()]
    want = []
    for net in nets:
        net.run()
        torch.cuda.synchronize()
        want.append([t.clone() for t in net.results])
    # captured: both nets' graphs replayed side by side on two streams
    graphs = []
    for net in nets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            net.run()
            net.run()
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in nets]
    for how in ("graph", "current", "given", "handle"):
        for net in nets:
            for t in net.results:
                t.fill_(-1)
        torch.cuda.synchronize()
        for _ in range(10):
            for net, g, s in zip(nets, graphs, streams):
                if how == "given":
                    net.run(s)
                elif how == "handle":
                    net.run(s.cuda_stream)
                else:
                    with torch.cuda.stream(s):
                        g.replay() if how == "graph" else net.run()
        torch.cuda.synchronize()
        for net, w in zip(nets, want):
            assert all(torch.equal(a, b) for a, b in zip(net.results, w)), how
    del graphs
    for net in nets:
        sa.slide_attn_destroy(net.ctx)


def test_workspaces_of_the_callers():
    net = Net(5).transposes()
    net.run()
    torch.cuda.synchronize()
    want = [t.clone() for t in (net.idx, net.dq, net.dk, net.dv, net.dgamma)]
    room = torch.full((2 * 8 * B * HEADS * 9 * D // 8 + 64,), float("nan"), device="cuda", dtype=torch.float64)
    sa.slide_attn_select_blocks(net.q, net.k, BLOCK, net.idx, workspace=room)
    assert torch.isnan(room[-64:]).all() and not torch.isnan(room[:-64]).any()
    sa.slide_attn_sparse_backward(net.q, net.k, net.v, net.idx, BLOCK, net.z, net.lse, net.dz, net.dq, net.dk, net.dv, workspace=room)
    sa.slide_attn_group_norm_backward(net.x, net.gamma, net.beta, GROUPS, sa.ACT_SILU, net.mean, net.rstd, net.dn, net.dx, net.dgamma, net.dbeta,
                                      workspace=room)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (net.idx, net.dq, net.dk, net.dv, net.dgamma)))
    for f in (lambda w: sa.slide_attn_select_blocks(net.q, net.k, BLOCK, net.idx, workspace=w),
              lambda w: sa.slide_attn_sparse_backward(net.q, net.k, net.v, net.idx, BLOCK, net.z, net.lse, net.dz, net.dq, net.dk, net.dv, workspace=w)):
        with pytest.raises(sa.SlideAttnError) as e:
            f(room[:16])
        assert e.value.status == sa.ERR_INVALID_ARG
    sa.slide_attn_destroy(net.ctx)


def test_tensors_that_are_refused():
    x = torch.zeros(1, 4, 8, 32, device="cuda")
    s = torch.zeros(1, 4, device="cuda")
    with pytest.raises(ValueError):                                  # not contiguous
        sa.slide_attn_group_norm_forward(x.transpose(1, 2), None, None, 4, 1e-5, sa.ACT_NONE, torch.empty_like(x).transpose(1, 2), s, s.clone())
    with pytest.raises(sa.SlideAttnError) as e:                      # 4 bytes past a 16-byte boundary
        flat = torch.zeros(1 * 4 * 8 * 32 + 1, device="cuda")
        sa.slide_attn_group_norm_forward(flat[1:].view(1, 4, 8, 32), None, None, 4, 1e-5, sa.ACT_NONE, torch.empty_like(x), s, s.clone())
    assert e.value.status == sa.ERR_ALIGNMENT
    with pytest.raises(sa.SlideAttnError) as e:
        sa.slide_attn_group_norm_forward(x, None, None, 4, 1e-5, sa.ACT_NONE, x, s, s.clone())
    assert e.value.status == sa.ERR_INVALID_ARG
