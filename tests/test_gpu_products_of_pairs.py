"""Products of two blocks on one tile, each holding half of its operands: whatever the second
block's copies are slowed by, the first multiplies what they brought."""
import pytest
import torch

from paper_2607_23115_gb300 import fp8

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


@pytest.mark.parametrize("m,n,k", [(2560, 2304, 128), (4096, 4096, 512), (8192, 4864, 640)])
def test_products_beside_copies_agree_with_products_alone(m, n, k):
    """Another stream's copies through L2 and memory make the blocks' copies land unevenly."""
    torch.manual_seed(m)
    xs = [torch.randn(m, k, device=DEV).to(torch.bfloat16) for _ in range(4)]
    w = fp8.quantize_weight(0.02 * torch.randn(n, k, device=DEV), grad=True)
    want = [fp8.linear(x, w) for x in xs]
    back = [fp8.linear_grad(y, x, w) for x, y in zip(xs, want)]
    a, b = (torch.empty(96 << 20, dtype=torch.uint8, device=DEV) for _ in range(2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    differ = torch.zeros((), dtype=torch.int64, device=DEV)
    for i in range(60):
        with torch.cuda.stream(side):
            b.copy_(a)
        differ += (fp8.linear(xs[i % 4], w) != want[i % 4]).sum()
        if i % 3 == 0:
            dx, dw = fp8.linear_grad(want[i % 4], xs[i % 4], w)
            differ += (dx != back[i % 4][0]).sum() + (dw != back[i % 4][1]).sum()
    torch.cuda.synchronize()
    assert differ.item() == 0
