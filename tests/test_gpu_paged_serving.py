"""The serving example: eviction, prefix match and the paged cache's operators in one loop.  Every output is within the
rounding of its weights and of itself (bf16: 2^-8 of values up to about 5, twice, halved by averaging) of attention
without a cache over the keys and values that the cache holds; prefixes are reused and blocks evicted on the way."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("kv_type", [0, 2])
def test_serving_example(kv_type):
    import paged_serving
    r = paged_serving.main(kv_type, n_blocks=56, n_requests=24)
    assert r["matched"] > 0.2 and r["evicted"] > 0
    assert r["worst"] < 5 * 2.0 ** -7
