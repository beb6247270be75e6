"""Orders between the lanes of a wave in the attention's gradients, with bounds and statement of test_gpu_ops."""
import pytest

from tests.gpu_util import announce, torch_cuda
from tests.test_gpu_ops import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,heads,kv,dim", [
    (((300, 300), (257, 129)), 4, 2, 64), (((300, 300),), 2, 2, 128), (((40, 700), (33, 64)), 2, 2, 32),
    (((128, 128), (97, 65)), 3, 3, 64), (((64, 64), (64, 40)), 3, 3, 32)])
def test_bias_gradient_of_every_distance(dtype, lens, heads, kv, dim):
    """A bucket for each distance and no dropout: neighbouring 32 x 32 tiles of scores add to the same distances one
    right after the other, from different lanes, in the tiled kernels (long or grouped) and the short one."""
    torch = torch_cuda()
    radius = 200
    announce(f"bias gradient by distance {dtype} {lens} {heads} {kv} {dim}")
    c = Case(dtype=dtype, lens=lens, heads=heads, kv_heads=kv, dim=dim, radius=radius, n_buckets=2 * radius + 1, seed=60)
    c.bucket.copy_(torch.arange(2 * radius + 1))
    c.run()
    c.verify()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,heads,kv,dim,radius", [
    (((300, 300), (129, 257)), 4, 2, 64, None), (((260, 300),), 2, 1, 128, 30), (((700, 40), (33, 31)), 2, 1, 32, None)])
def test_dropped_probabilities_tile_after_tile(dtype, lens, heads, kv, dim, radius):
    """The key kernel turns each tile's keep bits through the same words of LDS, one tile right after the other: half of
    the probabilities dropped, so that bits of a neighbouring tile would show in every gradient."""
    announce(f"dropout tile after tile {dtype} {lens} {heads} {kv} {dim} {radius}")
    c = Case(dtype=dtype, lens=lens, heads=heads, kv_heads=kv, dim=dim, radius=radius, p=0.5, seed=61)
    c.run()
    c.verify()
