"""The serving example's check on pages of full width covers the keys that it reads back and turns back."""

import os
import sys

import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,bound", [("bf16", 2e-2), ("f32", 1e-5)])
def test_worst_error_covers_the_keys_read_back(dtype, bound):
    """A key is rounded to the cache's type (half a step: 2^-8 of an element of bf16, 2^-24 of fp32) after its turn and again
    after the turn back, a pair's turn adding up two such errors: below 2^-6 of the largest element in bf16.  In fp32 2^-22, and
    of each turn's sine, cosine, two products and their sum as much again: below 2^-20."""
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import paged_serving
    r = paged_serving.serve(requests=9, pages=30, batch=6, dtype=dtype, check=True, longest=400)
    assert 0 < r["worst_keys"] <= r["worst"] <= bound, r
    assert r["worst_keys"] <= (2.0 ** -6 if dtype == "bf16" else 2.0 ** -20), r
