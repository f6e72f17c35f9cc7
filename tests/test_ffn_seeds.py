"""Seeds and offsets of the dropout as a program has them, without a GPU."""
import numpy as np
import pytest

import paper_2602_21466_amd as lib


@pytest.mark.parametrize("kind", [int, np.int32, np.int64, np.uint64])
def test_whole_numbers_of_any_kind(kind):
    plan = lib.NormPlan(8, dropout=0.5)
    n = plan._norm(kind(5), kind(7))
    assert (n.seed, n.offset) == (5, 7)


def test_negative_and_large_seeds_are_taken_modulo_2_to_the_64():
    plan = lib.NormPlan(8, dropout=0.5)
    n = plan._norm(np.int64(-1), -2)
    assert (n.seed, n.offset) == (2 ** 64 - 1, 2 ** 64 - 2)
    n = plan._norm(2 ** 64 + 3, np.uint64(2 ** 64 - 1))
    assert (n.seed, n.offset) == (3, 2 ** 64 - 1)


def test_a_seed_that_is_no_whole_number():
    with pytest.raises(TypeError):
        lib.NormPlan(8, dropout=0.5)._norm(0.5, 0)
