"""How far the angles of keys are off late in a run of positions, where the many-row attention over 8-bit codes has advanced
them step by step."""
import math

import numpy as np
import pytest
import torch

from tests import kv8_util as K8
from tests import test_gpu_kv8 as kv8
from tests.gpu_util import say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("style", [0, 1])
@pytest.mark.parametrize("rounds", [1, 3, 300])
def test_angles_late_in_a_run(style, rounds, monkeypatch):
    """Pair i turns by m_i / 1984 revolutions a position, so that at position 1984, the first key's after 32 advances of
    64 positions, the sine is 0 again (positions go on until 2047, the end of its step).  Request i's queries are the x
    of pair i at position 0, its key 1984 the largest code in that pair's y, and all other keys 0: that key's score is
    448 S times the sine that the kernel has, which the outputs show: its value is 1 and the others 0, so that
    o = e^s / (n - 1 + e^s) for a row of n keys.

    The angle may be off by 2^-17.  The sine is rounded to 2^-25 at most and its product with the code to 11 bits, the
    probability and the output to 8 bits, which s shows as they are (o is below 1/400); the sums to less."""
    def zeros(rng, nb, hkv, d, code, powers):
        return np.zeros((nb, hkv, 16, d), np.uint8), np.zeros((nb, hkv, 16, d), np.uint8), np.ones((nb, hkv, 2))
    monkeypatch.setattr(kv8, "random_pool", zeros)
    heads, n, big = 8, 16, 448 * 64.0
    m = np.random.default_rng(rounds).integers(1, 1984 * rounds, 32)
    m[:4] = 1, 31, 62, 991
    b = kv8.Batch([(2048, n)] * 32, 16 * heads, heads, 64, torch.bfloat16, K8.E4M3, style, softmax=64.0, inv_freq=m * (2 * math.pi / 1984),
              positions=lambda rng, total: np.tile(np.concatenate([np.arange(2048), np.zeros(n, np.int64)]), 32))
    assert kv8.tile_of(b) == (256, False)
    k, v = b.k_codes, b.v_codes
    q = torch.zeros_like(b.q)
    for i in range(32):
        x, y = (i, i + 32) if style == 0 else (2 * i, 2 * i + 1)
        q[n * i:n * (i + 1), :, x] = 1.0
        k[b.table[i, 124], :, 0, y] = 0x7e    # 448
        v[b.table[i, 124], :, 0, :] = 0x38    # 1
    b.q = q
    b.set_pool(k, v, b.scale)
    o = kv8.f64(b.run()).reshape(32, n, -1)
    rows = 2048 + np.arange(n)[None, :, None] + 1
    s = np.log(o * (rows - 1) / (1 - o))
    sine = np.abs(s).max((1, 2)) / big
    say(f"  sines within 2^{math.log2(sine.max()):.2f}")
    angle = 2.0 ** -17 * (1 + 2.0 ** -8)     # (a frequency is 2 pi times a double: 2^-52 of 1984 m revolutions)
    assert (np.abs(s) <= big * (angle + 2.0 ** -25) * (1 + 2.0 ** -10) + 2.0 ** -7 * 1.05).all(), float(sine.max())
