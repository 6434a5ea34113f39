"""What the operators around queries, keys and values do in large calls alone: workers with several tiles and several pairs."""
import pytest

from tests import kv4_cases as K
from tests import kv4_large as large
from tests.kv4_cases import same
from tests.test_gpu_kv4_attention import go

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2506_02850_amd import binding
    return binding


@pytest.mark.parametrize("name", sorted(large.CASES))
def test_attention_of_workers_with_several_tiles(B, name):
    """tests/test_qkv_boundary.py shows that they have them."""
    c = large.make(name)
    start = None if c["weight"] is None else c["weight"].clone()
    first = go(B, c)
    again = K.call(B, c if start is None else dict(c, weight=start))         # a row that is appended twice is the same row
    assert same(first["out"], again["out"]) and same(first["lse"], again["lse"]) and (start is None or same(start, c["weight"]))
