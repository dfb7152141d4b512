"""pic_qk_norm of heads that hold what is no number."""
import numpy as np
import pytest
import torch

from tests import kv8_util as K8
from tests import tree_util as T
from tests.test_gpu_kv8 import DTYPES, cfg_of, dev, f64

pytestmark = pytest.mark.gpu

B = pytest.importorskip("paper_2606_13126_amd._binding")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d,style", [(128, 0), (64, 1)])
@pytest.mark.parametrize("rotate", [0, 1])
def test_norm_of_what_is_no_number(dtype, d, style, rotate):
    """A NaN makes its whole head NaN.  An infinity makes the root infinite: its own element is NaN (turned, its
    partner too, which takes a product with it), the others 0.  Other heads and rows keep their bits."""
    n, hq, hkv = 6, 6, 2
    g = torch.Generator(device="cuda").manual_seed(d)
    clean = torch.randn(n, hq + hkv, d, generator=g, device="cuda").to(dtype)
    x = clean.clone()
    odd = {(0, 0): (float("nan"), 3), (1, 4): (float("inf"), 0), (2, 2): (-float("inf"), d - 1), (3, hq): (float("nan"), d - 1),
           (4, hq + 1): (float("inf"), d // 2)}
    for (r, h), (v, i) in odd.items():
        x[r, h, i] = v
    w = torch.randn(2, d, generator=g, device="cuda").to(dtype)
    pos = np.arange(1, n + 1, dtype=np.int32) * 1001
    cfg = cfg_of(hq, hkv, d, dtype, style, prerotated=rotate)

    def run(t):
        out = torch.zeros_like(t)
        B.pic_qk_norm(cfg, t[:, :hq], t[:, hq:], w[0], w[1], 1e-6, dev(pos), q_out=out[:, :hq], k_out=out[:, hq:])
        return out
    got, want = run(x), run(clean)
    for r in range(n):
        for h in range(hq + hkv):
            if (r, h) not in odd:
                assert torch.equal(got[r, h], want[r, h]), (r, h)
    with np.errstate(invalid="ignore"):
        for r, h in odd:
            ref = K8.norm(f64(x[r:r + 1, h:h + 1]), f64(w[int(h >= hq)]), 1e-6)
            if rotate:
                ref = T.rotate(ref, pos[r:r + 1], d, 1e4, style)
            out = f64(got[r, h])
            assert np.array_equal(np.isnan(out), np.isnan(ref[0, 0])) and (out[~np.isnan(out)] == 0).all(), (r, h, out)


def test_a_row_of_nan_does_not_reach_the_cache():
    """... nor does it move a scale: a key that holds one NaN is stored as zeros, and the block's other rows keep their codes."""
    cfg = cfg_of(1, 1, 64, torch.bfloat16)
    pool = B.Kv8Pool(torch.zeros(1, 1, 16, 64, dtype=torch.uint8, device="cuda"), torch.zeros(1, 1, 16, 64, dtype=torch.uint8, device="cuda"),
                     torch.zeros(1, 1, 2, device="cuda"), K8.INT8)
    k = torch.randn(5, 1, 64, generator=torch.Generator().manual_seed(0)).bfloat16().cuda()
    B.pic_qk_norm(cfg, None, k, None, None, 1e-6)
    B.pic_kv8_write(cfg, pool, k, k, dev(np.arange(5, dtype=np.int32)))
    codes, scale = pool.k.clone(), pool.scale.clone()
    bad = torch.ones(1, 1, 64, dtype=torch.bfloat16, device="cuda")
    bad[0, 0, 7] = float("nan")
    B.pic_qk_norm(cfg, None, bad, None, None, 1e-6)
    B.pic_kv8_write(cfg, pool, bad, bad, dev(np.array([5], np.int32)))
    assert torch.equal(pool.k, codes) and torch.equal(pool.scale, scale)
