"""After one call of the largest sizes on a stream, smaller ones can be captured there, whatever route they take."""
import pytest
import torch

import paper_2509_25401_amd as pkg

pytestmark = pytest.mark.gpu
E4M3, U8 = torch.float8_e4m3fn, torch.uint8


def _weight(N, K, seed):
    w = torch.randn(N, K, generator=torch.Generator().manual_seed(seed)).bfloat16().cuda()
    q, s = torch.zeros(N, K, dtype=E4M3, device="cuda"), torch.zeros(-(-N // 128), -(-K // 128), dtype=U8, device="cuda")
    pkg.sparse_fp8_quantize(w, q, s, block=True)
    return q, s


def _replayed(side, call, out):
    """Captures the call on a stream that has seen the largest sizes; every replay has to give the eager result."""
    call()
    torch.cuda.synchronize()
    want = out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        call()
    for _ in range(3):
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


@pytest.mark.parametrize("rows", [1, 40, 128, 300])
def test_products_of_fewer_rows(rows):
    print(f"[case] capture product {rows}", flush=True)
    M, N, K = 400, 3072, 12288
    q, s = _weight(N, K, 1)
    x = torch.randn(M, K, generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
    a, sa = torch.zeros(M, K, dtype=E4M3, device="cuda"), torch.zeros(M, K // 128, dtype=U8, device="cuda")
    pkg.sparse_fp8_quantize(x, a, sa)
    big, out = (torch.zeros(n, N, dtype=torch.bfloat16, device="cuda") for n in (M, rows))
    for call in (lambda x, a, sa, o: pkg.sparse_fp8_linear(x, q, s, None, o), lambda x, a, sa, o: pkg.sparse_fp8_gemm(a, sa, q, s, None, o)):
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call(x, a, sa, big)
        torch.cuda.synchronize()
        _replayed(side, lambda: call(x[:rows], a[:rows], sa[:rows], out), out)
        assert torch.equal(out, big[:rows]) or (out.float() - big[:rows].float()).abs().max() <= 2.0 ** -7 * big.float().abs().max()
        pkg.sparse_attn_release_scratch(side)


def test_rotary_gradients_of_fewer_tokens():
    H, D, axes = 24, 128, (16, 56, 56)
    g = torch.Generator().manual_seed(3)
    L, small = 8192, 8176                 # 512 token groups, and 511, which are dealt to twice as many workgroups
    qkv = torch.randn(1, L, 3 * H * D, generator=g).bfloat16().cuda()
    pos = torch.randint(0, 99, (L, 3), generator=g, dtype=torch.int32).cuda()
    grads = [torch.randn(1, H, L, D, generator=g).bfloat16().cuda() for _ in range(3)]
    w = torch.ones(D, dtype=torch.bfloat16, device="cuda")
    dqkv, dq, dk = torch.zeros_like(qkv), torch.zeros(D, device="cuda"), torch.zeros(D, device="cuda")

    def call(n):
        pkg.sparse_rotary_heads_backward(*(t[:, :, :n] for t in grads), qkv[:, :n], pos[:n], dqkv[:, :n], axes=axes, q_weight=w, k_weight=w, dq_weight=dq,
                                         dk_weight=dk)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(L)
    torch.cuda.synchronize()
    _replayed(side, lambda: call(small), dq)
    pkg.sparse_attn_release_scratch(side)
