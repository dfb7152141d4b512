"""Where the decode over 8-bit codes rounds queries: once, as they turn by their distance from a block."""
import math

import numpy as np
import pytest
import torch

from tests import test_gpu_kv8 as kv8
from tests import tree_util as T
from tests import kv8_util as K8
from tests.gpu_util import say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("style", [0, 1])
@pytest.mark.parametrize("code", kv8.CODES)
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 4, 64), (20, 1, 128)])
def test_queries_whole_revolutions_from_a_block(hq, hkv, d, code, style):
    """Every pair turns by a multiple of 1/16 of a revolution a position, and positions begin at 5: the query, the first
    token of its block, is whole revolutions away from every block's first key, though neither is a whole number of them
    from position 0.  Keys other than a block's first are 0.  Nothing that a score is made of has to be rounded then
    (numbers of bf16 and codes are exact in float16), but the sums of its products in 32 bits (d 2^-24 of |q| |k|); the
    probabilities have 16 bits, the outputs 8."""
    n = 400
    freq = np.random.default_rng(d).integers(1, 16, d // 2) * (2 * math.pi / 16)
    b = kv8.Batch([(n, 1), (16, 1), (n // 2 // 16 * 16, 1)], hq, hkv, d, torch.bfloat16, code, style, decode=True, inv_freq=freq, softmax=1.0,
                  seed=hq, positions=lambda rng, total: np.concatenate([5 + np.arange(m + 1) for m in (n, 16, n // 2 // 16 * 16)]))
    k = b.k_codes.copy()
    k[:, :, 1:] = 0
    # a block's largest element near 1, so that scores are a few units apart
    b.set_pool(k, b.v_codes, b.scale * np.float32(0.25))
    got = kv8.f64(b.run())
    kk, vv = (K8.decode(c, code) * b.scale[..., i].astype(np.float64)[:, :, None, None] for i, c in enumerate((b.k_codes, b.v_codes)))
    q = kv8.f64(b.q)
    worst = 0.0
    for r, (ctx, _, _) in enumerate(b.lens):
        j = np.arange(ctx + 1)
        keys, values = (p[b.table[r, j // 16], :, j % 16] for p in (kk, vv))
        o, spread = T.attention(q[r:r + 1], keys, values, np.ones((1, ctx + 1), bool), 1.0)   # (turned as far as the keys that are not 0)
        ds = np.linalg.norm(q[r], axis=-1).max() * np.linalg.norm(keys, axis=-1).max() * d * 2.0 ** -24
        e = np.expm1(ds) + 2.0 ** -16 + 2.0 ** -20
        tol = e / (1 - e) * spread + (2.0 ** -8 * 1.01 + (2 * ctx + 18) * 2.0 ** -24) * (np.abs(o) + e / (1 - e) * spread) + (2 * ctx + 18) * 2.0 ** -24 * spread
        off = np.abs(got[r:r + 1] - o)
        worst = max(worst, float((off / tol).max()))
    say(f"  at most {worst:.2f} of the bound")
    assert worst <= 1.0
