"""Block-sparse attention, backward, with keys of -infinity that mask themselves."""
import pytest
import torch

from test_gpu_sparse import call, check, inputs
from test_gpu_norm import back
from oracle import operators as ops

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [16, 32, 64])
def test_a_masked_key_reaches_one_component_of_dq_only(d, dtype):
    """Key (1, 1) of block 0 holds -infinity in its first component: its weights are 0; all else is as if the key were not there."""
    B, H, W, heads, block = 1, 8, 12, 2, (4, 4)
    q, k, v, g = inputs((B, H, W, heads, d), dtype, seed=d)
    q[..., 0] = q[..., 0].abs() + 0.1
    idx = torch.tensor([[0, 1], [1, 2], [0, 3], [3, 3], [2, 5], [4, 0]], device="cuda", dtype=torch.int32).expand(B, heads, 6, 2).contiguous()
    k[0, 1, 1, :, 0] = float("-inf")
    got = call(q, k, v, idx, block, g)
    sees = torch.zeros(H, W, dtype=torch.bool, device="cuda")
    sees[:4, :4] = sees[:4, 8:] = sees[4:, 8:] = True                # blocks 0, 2 and 5
    assert torch.isnan(got["dq"][0][sees][..., 0]).all() and torch.isfinite(got["dq"][0][~sees]).all() and torch.isfinite(got["dq"][..., 1:]).all()
    for n in ("out", "lse", "dk", "dv"):
        assert torch.isfinite(got[n]).all()
    assert (got["dk"][0, 1, 1] == 0).all() and (got["dv"][0, 1, 1] == 0).all()
    far = k.clone()
    far[0, 1, 1, :, 0] = -1e4 * d                                    # as good as masked: weights below 2^-150
    check({n: got[n] for n in ("out", "lse", "dk", "dv")}, ops.sparse(back(q), back(far), back(v), idx.cpu().numpy(), block, back(g), back(got["out"])), dtype)
