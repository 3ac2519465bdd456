"""The expert-layer example at a row length of one whole scale group and a half."""
import os
import sys

import pytest

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                                "examples"))

pytestmark = pytest.mark.gpu


def test_eight_bit_rows_of_192_columns():
    import expert_alltoall

    got = expert_alltoall.main(tokens=256, dim=192, num_experts=32, k=2, steps=2, candidates=64,
                               say=lambda line: None)
    # e4m3 has 4 significant bits: rows are within 2^-4 of themselves
    assert 0 < got["off"] < 2.0 ** -4
