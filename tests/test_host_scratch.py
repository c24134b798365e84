"""What the calls take of the stream's scratch memory."""
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
