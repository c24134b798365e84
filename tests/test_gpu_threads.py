"""Two host threads with calls on one stream of the GPU: operands and partial sums in the stream's scratch memory stay those of their
call."""
import threading

import pytest
import torch

import paper_2509_25401_amd as pkg

pytestmark = pytest.mark.gpu


def test_two_threads_on_one_stream():
    N, K, sizes = 384, 1024, (64, 700)
    g = torch.Generator().manual_seed(1)
    w = torch.randn(N, K, generator=g).bfloat16().cuda()
    q, s = torch.zeros(N, K, dtype=torch.float8_e4m3fn, device="cuda"), torch.zeros(3, 8, dtype=torch.uint8, device="cuda")
    pkg.sparse_fp8_quantize(w, q, s, block=True)
    stream = torch.cuda.Stream()
    xs = [[torch.randn(M, K, generator=g).bfloat16().cuda() for _ in range(4)] for M in sizes]
    want = [[torch.empty(M, N, dtype=torch.bfloat16, device="cuda") for _ in range(4)] for M in sizes]
    for x, o in zip(sum(xs, []), sum(want, [])):
        pkg.sparse_fp8_linear(x, q, s, None, o)
    torch.cuda.synchronize()
    got = [[torch.zeros(20, *o.shape, dtype=o.dtype, device="cuda") for o in os] for os in want]
    torch.cuda.synchronize()
    start, failed = threading.Barrier(2), []

    def work(t):
        try:
            start.wait()
            for i in range(20):
                for x, o in zip(xs[t], got[t]):
                    pkg.sparse_fp8_linear(x, q, s, None, o[i], stream=stream)
        except Exception as e:              # noqa: BLE001 -- reported below
            failed.append(e)

    team = [threading.Thread(target=work, args=(t,)) for t in range(2)]
    [t.start() for t in team]
    [t.join() for t in team]
    torch.cuda.synchronize()
    assert not failed
    for os, ws in zip(got, want):
        for o, v in zip(os, ws):
            assert torch.equal(o, v.expand_as(o))
