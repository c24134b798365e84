"""What the calls take of the stream's scratch memory."""
import random

import pytest

from host_calls import run

SUMS = ("dweight", "dscale", "dshift", "dgate", "dpost_weight")


def _taken(cases):
    """Bytes that each call asks for, in a process that has given the memory back before it."""
    return [sum(e[1] for e in run("calls", [case])[0][2] if e[0] == "malloc") for case in cases]


def test_sums_of_a_vector_for_each_token_are_kept_where_they_belong():
    rows, C = 33024, 3072
    *alone, both, all_ = _taken([["norm_backward", [rows, 1, C], {"sums": s}] for s in (("dshift",), ("dscale",), ("dgate",), ("dscale", "dshift", "dgate"), SUMS)])
    assert alone + [both] == [0, 0, 0, 0]
    assert all_ <= 1.5 * 2 * rows * C * 4


def test_only_the_sums_that_are_wanted_take_memory():
    one, three, weights = _taken([["norm_backward", [33024, 2064, 3072], {"sums": s}] for s in (("dshift",), ("dscale", "dshift", "dgate"), ("dweight",))])
    assert 0 < one <= three / 3
    assert weights <= one + 1.5 * 16 * 3072 * 4


def _sizes(rng, kind):
    def size(most):
        return int(2 ** rng.uniform(0, most))
    if kind == "rotary_backward":
        return [size(3), size(15), size(6), size(5), rng.choice((32, 64, 128, 256))]
    return [size(14), 16 * size(9), 16 * size(9)]


def _smaller(rng, kind, sizes):
    if kind == "rotary_backward":
        return [rng.randint(1, n) for n in sizes[:4]] + [rng.choice([d for d in (32, 64, 128, 256) if d <= sizes[4]])]
    return [rng.randint(1, sizes[0])] + [16 * rng.randint(1, n // 16) for n in sizes[1:]]


@pytest.mark.parametrize("kind", ["gemm", "linear", "linear_backward", "rotary_backward"])
def test_no_smaller_call_takes_more(kind):
    """A capture may follow a call of the largest sizes: whatever is smaller then allocates nothing."""
    rng = random.Random(len(kind))
    known = {"gemm": [[[400, 3072, 12288], [1, 3072, 12288]], [[4608, 3072, 8192], [16, 48, 8192]]],
             "linear": [[[400, 3072, 12288], [128, 3072, 12288]], [[33024, 512, 512], [1000, 512, 512]]],
             "linear_backward": [[[400, 12288, 3072], [128, 12288, 3072]], [[33024, 512, 512], [20000, 512, 512]]],
             "rotary_backward": [[[1, 8192, 24, 24, 128], [1, 8176, 24, 24, 128]], [[1, 33024, 24, 24, 128], [1, 4608, 24, 8, 128]]]}[kind]
    pairs = known + [[s, _smaller(rng, kind, s)] for s in (_sizes(rng, kind) for _ in range(400))]
    got = run("calls", [c for large, small in pairs for c in ([kind, large, {}], [kind, small, {}], ["release", [], {}])])
    for (large, small), first, second in zip(pairs, got[::3], got[1::3]):
        assert first[0] == second[0] == 0, (first, second)
        assert all(e[0] == "launch" for e in second[2]), f"{kind} {small} allocates after {large}"


def test_a_call_with_fewer_results_takes_no_more():
    for want in ({"dx": False}, {"dw": False}, {"db": False}, {"dx": False, "dw": False}):
        got = run("calls", [["linear_backward", [9001, 512, 768], {}], ["linear_backward", [9001, 512, 768], want]])
        assert all(e[0] == "launch" for e in got[1][2])


def test_products_stay_inside_what_they_take():
    """What is launched fits the memory: split sums of M x N floats, packed scales of 2 x 128 bytes for each tile and pair of groups."""
    rng = random.Random(7)
    sizes = [_sizes(rng, "gemm") for _ in range(400)] + [[1, 3072, 12288], [40, 64, 9008], [128, 65536, 400], [256, 32768, 3072]]
    got = run("calls", [c for s in sizes for c in (["gemm", s, {}], ["release", [], {}])])[::2]
    seen = set()
    for (M, N, K), (_, _, record) in zip(sizes, got):
        room = sum(e[1] for e in record if e[0] == "malloc") / 1.5
        groups = -(-K // 128)
        for _, name, x, y, z, *_ in (e for e in record if e[0] == "launch"):
            if "pack_scales" in name:
                assert x * 2048 - 2048 < room and groups >= 3
                seen.add("scales")
            elif "fp8_gemm_kernel" in name and z > 1:
                assert z * M * N * 4 <= room + 1
                seen.add("sums")
    assert seen == {"scales", "sums"}
