"""Sizes at the ends of their types: no sum of them may leave its type."""
import pytest

import paper_2509_25401_amd as pkg
from host_calls import run
from test_block_host import UNSUPPORTED, _rotary

ALL = (1 << 63) - 1


@pytest.mark.parametrize("many", [ALL, 1 << 32, (1 << 31) + 5])
def test_all_rows_share_a_vector_however_many_that_may_be(many):
    for kind in ("norm", "norm_backward"):
        want, got = run("calls", [[kind, [40, 40, 256], {}], [kind, [40, many, 256], {}]])
        assert want[0] == got[0] == 0
        launches = [[e for e in r if e[0] == "launch"] for r in (want[2], got[2])]
        assert launches[0] == launches[1] and launches[0]


@pytest.mark.parametrize("kw", [dict(heads_q=1 << 30, heads_kv=1 << 30), dict(heads_q=(1 << 31) - 1, heads_kv=1), dict(heads_q=1, heads_kv=1 << 30)])
@pytest.mark.parametrize("backward", [False, True])
def test_more_heads_than_are_counted(kw, backward):
    assert _rotary(backward, **kw) == UNSUPPORTED
    assert "heads" in pkg.sparse_attn_last_error()


def test_frequencies_of_a_negative_axis():
    with pytest.raises(ValueError):
        pkg.sparse_rotary_frequencies((-4, 8))
