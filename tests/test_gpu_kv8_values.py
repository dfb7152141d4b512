"""Probabilities of the many-row attention over 8-bit codes: sums of exactly what is multiplied, and blocks whose values'
scales lie far apart, down to elements that only the smaller ones are not 0 in."""
import numpy as np
import pytest
import torch

from tests import kv8_util as K8
from tests import test_gpu_kv8 as kv8

pytestmark = pytest.mark.gpu

SHAPES = [kv8.LARGE[i] for i in (0, 1, 6, 10, 11)]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def batch(shape, **kw):
    hq, hkv, d, lens, tile, split = SHAPES[shape]
    b = kv8.Batch(lens, hq, hkv, d, torch.bfloat16, **kw)
    assert kv8.tile_of(b) == (tile, split)
    return b


@pytest.mark.parametrize("code", kv8.CODES)
@pytest.mark.parametrize("shape", [1, 3, 4])
def test_rows_of_one_value(shape, code):
    """Where all values that a row sees are one number, the output is that number: the sum of a row is of the probabilities that
    are multiplied.  A token that sees only itself gives its own values."""
    b = batch(shape, code=code, seed=7)
    v = b.v_codes.copy()
    v[:] = v[:1, :, :1]       # the same row of values everywhere, of one scale
    scale = b.scale.copy()
    scale[..., 1] = 2.0 ** -3
    b.set_pool(b.k_codes, v, scale)
    g = b.hq // b.hkv
    want = np.repeat(K8.decode(v[0, :, 0], code) * 2.0 ** -3, g, 0)
    assert (kv8.f64(b.run()) == want).all()
    if b.lens[0][0] == 0:
        c = batch(shape, code=code, seed=8)
        at = c.table[0, 0]
        want = np.repeat(K8.decode(c.v_codes[at, :, 0], code) * c.scale[at, :, 1:].astype(np.float64), g, 0)
        assert (kv8.f64(c.run())[0] == want).all()


@pytest.mark.parametrize("code", kv8.CODES)
@pytest.mark.parametrize("shape", range(len(SHAPES)))
@pytest.mark.parametrize("apart", [4, 14, 60, "zeros"])
def test_values_of_scales_apart(shape, code, apart):
    """Blocks of values 2^apart times the others', or of zeros between values of 2^40: every row's sum still counts every key."""
    b = batch(shape, code=code, seed=shape + 3, prerotated=shape % 2)
    scale = b.scale.copy()
    some = b.rng.random(scale.shape[:2]) < 0.5
    v = b.v_codes.copy()
    if apart == "zeros":      # (as pic_kv8_write stores them: the least scale)
        scale[..., 1] = np.where(some, 2.0 ** 40, 2.0 ** -126)
        v[~some] = 0
    else:
        scale[..., 1] = np.where(some, 1.0, 2.0 ** -apart)
    b.set_pool(b.k_codes, v, scale)
    b.check(b.run(), f"{apart}")


@pytest.mark.parametrize("code", kv8.CODES)
@pytest.mark.parametrize("shape", [1, 2])
def test_rows_that_see_small_values_alone(shape, code):
    """Values grow from block to block by 2^10: the first tokens see only small ones, the last ones all."""
    b = batch(shape, code=code, seed=shape + 5)
    scale = b.scale.copy()
    for r in range(len(b.lens)):
        n = -(-sum(b.lens[r][:2]) // 16)
        scale[b.table[r, :n], :, 1] = np.exp2(np.minimum(10 * np.arange(n), 150) - 80)[:, None]
    b.set_pool(b.k_codes, b.v_codes, scale)
    b.check(b.run(), "growing")
