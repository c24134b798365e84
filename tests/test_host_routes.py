"""The products' tests reach every route that a product can take.  Which one a size takes follows from measured times; where these
change, the sizes of the tests have to follow."""
import itertools
import re

import test_gpu_fp8
import test_gpu_fp8_long
from host_calls import run


def routes(sizes):
    """{(M, N, K, float32 result): route}"""
    calls = [["gemm", [M, N, K], {"f32": f}] for M, N, K in sizes for f in (0, 1)]
    found = {}
    for (_, (M, N, K), kw), (rc, message, record) in zip(calls, run("calls", calls)):
        assert rc == 0, message
        f32, groups = kw["f32"], -(-K // 128)
        past = N * (4 if f32 else 2) % 64 == 0                    # every row of the result starts on 64 bytes
        names = [e for e in record if e[0] == "launch"]
        for _, name, x, y, z, *_ in names:
            big = re.search(r"fp8_gemm_big_kernelILi(\d)ELb(\d)", name)
            tile = re.search(r"fp8_gemm_kernelILi(\d+)ELi(\d+)", name)
            if big:
                assert int(big[2]) == f32
                found[M, N, K, f32] = ("rows", 32 * int(big[1]), f32, past)
            elif tile:
                order = "by rows" if not past and N * K <= 2 << 20 else "by columns"
                found[M, N, K, f32] = ("tile", int(tile[1]), order, "split" if z > 1 else "past" if past else "whole", -(-groups // z) > 32)
    assert len(found) == len(calls)
    return found


def test_every_route_has_a_test():
    found = routes(test_gpu_fp8.MNK + test_gpu_fp8.ROUTES + test_gpu_fp8_long.LONG + test_gpu_fp8_long.SPLIT + test_gpu_fp8_long.LARGE)
    wanted = set(itertools.product(["rows"], [128, 160, 192, 224, 256], [0, 1], [False, True]))
    for tile, long_ in ((128, False), (64, False), (32, False), (64, True), (32, True)):
        wanted |= {("tile", tile, "by columns", "past", long_), ("tile", tile, "by rows", "whole", long_)}
    wanted |= {("tile", t, "by columns", "whole", False) for t in (128, 64, 32)} | {("tile", 32, "by columns", "whole", True)}
    wanted |= {("tile", t, o, "split", False) for t in (128, 64, 32) for o in ("by rows", "by columns")}
    wanted |= {("tile", 128, "by columns", "split", True), ("tile", 64, "by columns", "split", True), ("tile", 64, "by rows", "split", True)}
    assert wanted <= set(found.values()), sorted(wanted - set(found.values()), key=str)


def test_long_and_split_cases_are_what_they_say():
    assert all(r[4] for r in routes(test_gpu_fp8_long.LONG).values())
    assert all(r[3] == "split" for r in routes(test_gpu_fp8_long.SPLIT + test_gpu_fp8_long.LARGE).values())
