"""Every tensor of the norm and the gradients of the rotary weights have to be aligned to their elements, whatever type these are."""
import pytest

import paper_2509_25401_amd as pkg
from test_block_host import INVALID, _at, _back, _norm, _rotary

F32 = dict(x_dtype=1, vector_dtype=1)


def _refused(code):
    assert code == INVALID and "aligned to their elements" in pkg.sparse_attn_last_error()


@pytest.mark.parametrize("name", ["x", "x_out", "scale", "shift", "gate", "weight", "post_weight"])
def test_float32_tensors_of_the_norm(name):
    _refused(_norm(**F32, **{name: _at(20) + 2}))


@pytest.mark.parametrize("name", ["y", "h"])
def test_bf16_tensors_of_the_norm(name):
    _refused(_norm(**F32, **{name: _at(20) + 1}))


@pytest.mark.parametrize("name", ["dx_out", "x_out", "dx", "scale", "gate", "weight", "post_weight", "dscale", "dshift", "dgate", "dweight", "dpost_weight"])
def test_float32_tensors_of_its_gradients(name):
    _refused(_back(**F32, **{name: _at(20) + 2}))


@pytest.mark.parametrize("name", ["dh", "y", "dy"])
def test_bf16_tensors_of_its_gradients(name):
    _refused(_back(**{name: _at(20) + 1}))


@pytest.mark.parametrize("name", ["dscale", "dpost_weight"])
def test_sums_beside_bf16_tensors(name):
    _refused(_back(**{name: _at(20) + 2}))


@pytest.mark.parametrize("name", ["dq", "dk"])
def test_gradients_of_the_rotary_weights(name):
    _refused(_rotary(True, q_weight=_at(8), k_weight=_at(9), extra={name: _at(10) + 2}))
