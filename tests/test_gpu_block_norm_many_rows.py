"""Block norm on the GPU with more rows than one axis of a launch has threads for: rows of eight channels, 1.1 GB each tensor."""
import pytest
import torch

import paper_2509_25401_amd as pkg

pytestmark = pytest.mark.gpu


def test_seventy_million_rows():
    rows, C = 70_000_000, 8
    print(f"[case] block_norm many rows {rows} {C}", flush=True)
    first = torch.randn(1000, C, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    x = first.repeat(rows // 1000, 1)
    h = torch.full_like(x, 7.0)
    want = torch.empty_like(first)
    pkg.sparse_block_norm(first, None, want, norm="layer")
    pkg.sparse_block_norm(x, None, h, norm="layer")
    assert torch.equal(h.view(-1, 1000, C), want.expand(rows // 1000, 1000, C))
    dx, dx1, grad = torch.full_like(x, 7.0), torch.empty_like(first), torch.ones_like(x)
    pkg.sparse_block_norm_backward(grad[:1000], None, first, None, dx1, norm="layer")
    pkg.sparse_block_norm_backward(grad, None, x, None, dx, norm="layer")
    assert torch.equal(dx.view(-1, 1000, C), dx1.expand(rows // 1000, 1000, C))
