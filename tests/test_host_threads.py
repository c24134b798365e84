"""Calls from several threads on one stream.  Those that keep operands or partial sums in the stream's scratch memory enqueue a row
of kernels that belong together: nothing of another call may come between them, and the memory may not be replaced before the last."""
import pytest

from host_calls import run

CALLS = [("linear", [[200, 512, 256], [64, 512, 256]]), ("linear", [[8, 384, 256], [3000, 384, 1024]]), ("gemm", [[40, 70, 9008], [20, 64, 20000]]),
         ("gemm", [[4608, 9216, 512], [4096, 9216, 512]]), ("linear_backward", [[300, 256, 384], [5000, 512, 384]]),
         ("norm_backward", [[640, 64, 1160], [64, 64, 256]]), ("norm_backward", [[9001, 9001, 256], [33024, 2064, 3072]]),
         ("rotary_backward", [[1, 300, 4, 4, 64], [2, 9001, 24, 8, 128]]), ("attention", [[1, 24, 33024, 128], [1, 24, 20000, 128]]),
         ("symbols", [[1, 24, 8192, 128], [1, 2, 4096, 64]])]


@pytest.mark.parametrize("kind,sizes", CALLS)
def test_calls_of_two_threads_do_not_mix(kind, sizes):
    alone, both = run("threads", kind, sizes)
    rows = [[entry[1:] for entry in record if entry[1] == "launch"] for record in alone]
    assert all(len(r) > 1 for r in rows) and rows[0] != rows[1], "the case does not show anything"
    launches = [(e[0], e[1:]) for e in both if e[1] == "launch"]
    assert len(launches) == 6 * sum(map(len, rows))
    i, ends = 0, set()
    while i < len(launches):
        row = next((r for r in rows if launches[i][1] == r[0] and [e for _, e in launches[i:i + len(r)]] == r), None)
        assert row, f"kernels of two calls are mixed: {launches[i:i + 4]}"
        assert len({thread for thread, _ in launches[i:i + len(row)]}) == 1
        i += len(row)
        ends.add(i)
    seen = 0
    for e in both:
        seen += e[1] == "launch"
        assert e[1] != "free" or seen in ends | {0}, "the memory is replaced under a call"
