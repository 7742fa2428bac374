"""Many rows on packed weights in 32 bits: the product of three parts with
narrow factors in each of its tiles and in parts of the summed index."""
import pytest

from paper_1706_05544_amd import native as nv
from test_gpu_packed import check, gen, rnd

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,k,n", [
    # tiles of 128 x 256, steps of 32 inputs whole and cut
    (16384, 2048, 2048), (8000, 1000, 2000), (16385, 1001, 2047),
    # of 128 x 128 and of 64 x 64
    (4000, 500, 1000), (1100, 300, 900), (2000, 65, 130),
    # the summed index in parts
    (1100, 20000, 130), (1030, 9001, 200)])
def test_tiles(m, k, n):
    g = gen(m + k)
    X, W = rnd(g, m, k), rnd(g, n, k, by=k ** -0.5)
    b, R = rnd(g, n), rnd(g, m, n)
    check(X, nv.svm_pack_weights(W, 64), b, R, "gelu", "f32")
