"""What the serving example refuses before it touches a GPU."""

import os
import sys

import pytest

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_a_request_larger_than_the_pool_is_refused():
    import paged_serving
    with pytest.raises(ValueError):
        paged_serving.serve(requests=9, pages=3, longest=400)
