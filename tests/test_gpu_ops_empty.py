"""Attention where one side of every sequence is empty."""
import pytest

from tests.test_gpu_ops import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,heads,kv,dim", [
    (((1100, 0),), 2, 1, 64), (((600, 0), (20, 0)), 4, 2, 32), (((0, 1100),), 2, 1, 64), (((0, 40), (0, 0)), 2, 2, 64),
    (((1100, 0),), 2, 1, 4), (((40, 0),), 2, 2, 64)])
def test_no_keys_or_no_queries(dtype, lens, heads, kv, dim):
    """Queries without keys: results and gradients of zero; keys without queries: gradients of zero.  Rows that belong to
    no sequence lie around them."""
    for radius in (None, 9):
        check(dtype=dtype, lens=lens, heads=heads, kv_heads=kv, dim=dim, radius=radius, gap=2, seed=80)
