"""GPU: the weighted sum onto the rows that it adds to, over several pieces per thread."""
import pytest
import torch

from blocks_ref import gen
from paper_2505_14638_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,N,k", [(1, 16, 1), (33, 272, 3), (9000, 2064, 5)])
@pytest.mark.parametrize("y_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_sum_in_place(M, N, k, y_dtype, dtype):
    g = gen(M + N)
    y = torch.randn((M, N), generator=g, device="cuda").to(y_dtype)
    slots = torch.randint(0, M, (M, k), generator=g, device="cuda").to(torch.int32)
    weights = torch.rand((M, k), generator=g, device="cuda")
    wide = torch.randn((M, N + 16), generator=g, device="cuda").to(dtype)
    want = binding.combine_experts(y, slots, weights, add=wide[:, :N], out=torch.empty((M, N), dtype=dtype, device="cuda"))
    same = wide.clone()
    binding.combine_experts(y, slots, weights, add=same[:, :N], out=same[:, :N])
    torch.cuda.synchronize()
    assert binding.query_device_status() == 0
    assert torch.equal(same[:, :N], want) and torch.equal(same[:, N:], wide[:, N:])
