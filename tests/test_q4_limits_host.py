"""Limits that the calls on a 4-bit cache store keep to, checked on the host: runs without a GPU."""

import pytest

from tests.test_q4_host import INVALID, _tables


@pytest.mark.parametrize("limit", [-1, -(1 << 31)])
def test_rows_per_request_are_not_negative(limit):
    assert _tables(max_fresh=limit) == INVALID
