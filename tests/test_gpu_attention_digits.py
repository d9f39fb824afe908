"""The attention calls where the tests of test_gpu_attention.py do not reach: more digits than the sums of rotations add up before they
fold (4) and than the kernel for many rotations of one decomposition holds (8), ring 2^17, and splits with more rotations or groups
than a launch takes (32)."""
import pytest

import test_gpu_attention as attention
from ckks_inputs import make_params

pytestmark = pytest.mark.gpu

attention.PARAMS.update({
    "ring13_5_digits": lambda: make_params(13, 5, 50, 1, 60, 5),
    "ring13_9_digits": lambda: make_params(13, 9, 50, 1, 60, 9),
    "ring13_9_digits_int": lambda: make_params(13, 9, 60, 1, 60, 9),
})


@pytest.mark.parametrize("name,nl,B,npt,R", [
    ("ring13_5_digits", 5, 3, 3, 2), ("ring13_5_digits", 4, 1, 1, 2), ("ring13_5_digits", 5, 2, 1, 1), ("ring13_9_digits", 9, 2, 1, 2),
    ("ring13_9_digits", 8, 1, 1, 3), ("ring13_9_digits", 9, 1, 1, 1), ("ring13_9_digits_int", 9, 2, 2, 2)])
def test_rope_of_many_digits(name, nl, B, npt, R):
    attention.test_rope_matches_the_oracle(name, nl, B, npt, R)


@pytest.mark.parametrize("op,C,name,nl,B,n1,n2", [
    ("step", 1, "ring13_5_digits", 5, 1, 2, 2), ("chunk", 2, "ring13_5_digits", 5, 2, 3, 1), ("step", 1, "ring13_9_digits", 9, 2, 2, 2),
    ("chunk", 2, "ring13_9_digits", 9, 1, 2, 2), ("step", 1, "ring13_9_digits_int", 9, 1, 2, 1)])
def test_linear_attention_of_many_digits(op, C, name, nl, B, n1, n2):
    attention._run(op, name, nl, B, C, n1, n2, True, True)


@pytest.mark.parametrize("op,C,n1,n2", [("step", 1, 2, 2), ("chunk", 2, 2, 1)])
def test_linear_attention_at_2_to_17(op, C, n1, n2):
    attention._run(op, "ring17", 2, 1, C, n1, n2, True, True)


@pytest.mark.parametrize("op,C,n1,n2", [("step", 1, 1, 64), ("step", 1, 64, 1), ("chunk", 2, 2, 34)])
def test_more_rotations_than_a_launch_takes(op, C, n1, n2):
    attention._run(op, "ring10", 2, 1, C, n1, n2, True, False)
