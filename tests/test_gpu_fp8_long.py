"""8-bit products over long reductions on the GPU: more groups than have their scales in LDS at a time, and reductions that are
split, with sums that divide by no eight and results at any alignment.  Tolerances are those of test_gpu_fp8.  Which route a size
takes is held by test_host_routes."""
import pytest
import torch

import paper_2509_25401_amd as pkg
from test_gpu_fp8 import E4M3, U8, _check_product, _form, _matrix

pytestmark = pytest.mark.gpu

# more than 32 groups in one piece, in one more than 64
LONG = [(9, 4100, 4240), (1, 18432, 4608), (3, 9456, 6656), (1, 50, 4160), (1100, 1000, 8336), (4631, 65, 5760)]
# split: an odd number of results, one with four and one with eight left over, few rows, few columns
SPLIT = [(33, 301, 9008), (35, 71, 9008), (12, 67, 5008), (1, 16, 4592), (8, 200, 6000), (1, 2285, 16928), (4229, 17, 5840)]
# too large to be brought to 8 bits on the CPU: made of 8-bit values; split, also into parts of more than 32 groups
LARGE = [(1, 4355, 19424), (4345, 19, 19824), (65, 2451, 16384), (65, 4158, 20096), (2419, 66, 18656)]


def _everywhere(forms, a, b, bias, M, N):
    """Both types of result, with and without a bias, on 16 bytes and off them."""
    for dtype in (torch.bfloat16, torch.float32):
        held = torch.full((M * N + 64,), 7.0, dtype=dtype, device="cuda")
        out = held[:M * N].view(M, N)
        pkg.sparse_fp8_gemm(*forms, bias.cuda(), out)
        assert (held[M * N:] == 7.0).all(), "written past the end"
        _check_product(out, a, b, bias, f"{dtype}")
        other = torch.full((M * N + 64,), 7.0, dtype=dtype, device="cuda")
        shifted = other[1:1 + M * N].view(M, N)
        pkg.sparse_fp8_gemm(*forms, bias.cuda(), shifted)
        assert torch.equal(shifted, out), "another result at another alignment"
        assert other[0] == 7.0 and (other[1 + M * N:] == 7.0).all(), "written outside"
    plain = torch.empty(M, N, dtype=torch.float32, device="cuda")
    pkg.sparse_fp8_gemm(*forms, None, plain)
    _check_product(plain, a, b, None, "no bias")


@pytest.mark.parametrize("M,N,K", LONG + SPLIT)
@pytest.mark.parametrize("b_block", [True, False])
def test_long_reductions(M, N, K, b_block):
    print(f"[case] fp8_gemm long {M} {N} {K} {b_block}", flush=True)
    a, b, bias = _matrix(M + K, M, K), _matrix(N + 2 * K, N, K), _matrix(3, 1, N)[0]
    forms = []
    for m, n in ((a, 1), (b, 128 if b_block else 1)):
        q, s = torch.zeros(m.shape, dtype=E4M3, device="cuda"), torch.zeros(-(-m.shape[0] // n), -(-K // 128), dtype=U8, device="cuda")
        pkg.sparse_fp8_quantize(m.cuda(), q, s, block=n > 1)
        forms += [q, s]
    _everywhere(forms, _form(a), _form(b, 128 if b_block else 1), bias, M, N)


@pytest.mark.parametrize("M,N,K", LARGE)
def test_long_reductions_of_8_bit_values(M, N, K):
    print(f"[case] fp8_gemm large {M} {N} {K}", flush=True)
    forms, given = [], []
    for seed, rows in enumerate((M, N)):
        g = torch.Generator(device="cuda").manual_seed(seed)
        q = (torch.randn(rows, K, generator=g, device="cuda") * 16).clamp(-448, 448).to(E4M3)
        e = torch.randint(-4, 5, (rows, -(-K // 128)), generator=g, device="cuda")
        forms += [q, (e + 127).to(U8)]
        given.append((q.float().cpu().double(), e.cpu().int()))
    _everywhere(forms, *given, _matrix(3, 1, N)[0], M, N)
