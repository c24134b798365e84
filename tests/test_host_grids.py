"""A launch has fewer than 2^32 threads along an axis, however many rows there are."""
import random

from host_calls import run


def _fits(record):
    names = [e for e in record if e[0] == "launch"]
    return names and all(x * threads < 1 << 32 and y <= 65535 and z <= 65535 for _, _, x, y, z, threads, *_ in names)


def test_norms_of_many_rows():
    most = (1 << 31) - 1
    rng = random.Random(2)
    sizes = [(most, most, 8), (most, 1, 8), (70_000_000, 70_000_000, 8), (5_000_000, 5_000_000, 8192), (most, 7, 16384), (8_000_000, 1, 4104)]
    sizes += [(int(2 ** rng.uniform(20, 31)) - 1, int(2 ** rng.uniform(0, 31)), rng.randint(1, 16384)) for _ in range(60)]
    calls = [[kind, [rows, per, C], {}] for rows, per, C in sizes for kind in ("norm", "norm_backward")]
    for call, (rc, message, record) in zip(calls, run("calls", calls)):
        assert rc == 0, (call, message)
        assert _fits(record), (call, record)


def test_rotary_heads_of_many_tokens():
    calls = [[kind, [B, L, 1, 1, D], {}] for B, L, D in ((1, (1 << 31) - 1, 32), (1, 100_000_000, 256), (64, 1 << 24, 128), (1 << 20, 1 << 11, 32))
             for kind in ("rotary", "rotary_backward")]
    for call, (rc, message, record) in zip(calls, run("calls", calls)):
        assert (rc == 0 and _fits(record)) or (rc == -2 and "too many tokens" in message), (call, rc, message, record)


def test_products():
    rng = random.Random(3)
    sizes = [(1 << 22, 32768, 16), (1 << 22, 1 << 14, 512), (32768, 1 << 22, 128), (1 << 22, 1, 16), (1, 1 << 22, 400)]
    sizes += [(int(2 ** rng.uniform(10, 22)), int(2 ** rng.uniform(0, 15)), 16 * rng.randint(1, 64)) for _ in range(100)]
    calls = [["gemm", list(s), {}] for s in sizes] + [["gemm", [1 << 22, 1 << 22, 16], {}]]
    got = run("calls", calls)
    for call, (rc, message, record) in zip(calls[:-1], got):
        M, N, _ = call[1]
        assert (rc == 0 and _fits(record)) or (M * N >= 1 << 37 and rc == -2 and "results" in message), (call, rc, message, record)
    assert got[-1][0] == -2 and "results" in got[-1][1]
