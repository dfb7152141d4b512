"""How exact pic_attn_tree is beyond the bound of the other tests, in both directions: probabilities
of calls with few rows, and agreement with prefill and decode."""
import numpy as np
import pytest
import torch

from tests import test_gpu_tree as G
from tests import tree_util as T
from tests.gpu_util import say

pytestmark = pytest.mark.gpu

B = pytest.importorskip("paper_2606_13126_amd._binding")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def two_part_bound(o, spread, nq, nk, d):
    """Without rotation q and k are exact, so that scores are off by their sums alone: D 2^-24 |q||k| scale.
    A probability in two bf16 parts is off by 2^-15: the upper part cut leaves less than 2^-7 of it, which
    the lower one's rounding changes by 2^-8.  (exp2 and the row sum in 32 bits: 2^-20.)  Then the output's
    own rounding.  With one bf16 part, 2^-8, outputs near 0 of rows that see few keys lie far outside."""
    e = np.expm1(nq * nk * d ** -0.5 * d * 2.0 ** -24) + 2.0 ** -15 + 2.0 ** -20
    return e / (1 - e) * spread + (2.0 ** -8 * 1.01 + 2.0 ** -20) * np.abs(o) + 2.0 ** -8 * e * spread + 1e-30


def worst_of(b, got, bound):
    """Largest error of `got` over the bound."""
    kp, vp, q = G.f64(b.k_pool), G.f64(b.v_pool), G.f64(b.q)
    row, worst = 0, 0.0
    for r, (ctx, n, w) in enumerate(b.lens):
        j = np.arange(w, ctx + n)
        k, v = (p[b.table[r, j // 16], :, j % 16] for p in (kp, vp))
        see = np.concatenate([np.ones((n, ctx - w), bool), b.see[r]], 1)
        o, spread = T.attention(q[row:row + n], k, v, see, b.d ** -0.5)
        nq, nk = np.linalg.norm(q[row:row + n], axis=-1).max(), np.linalg.norm(k, axis=-1).max()
        d = np.abs(got[row:row + n] - o)
        assert np.isfinite(d).all()
        worst = max(worst, float((d / bound(o, spread, nq, nk, b.d)).max()))
        row += n
    return worst


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens", [[(0, 3), (5, 7)], [(2, 12), (0, 20)], [(40, 4), (16, 16)]])
def test_probabilities_of_few_rows_keep_16_bits(d, lens):
    b = G.Drafts(lens, 8, 2, d, prerotated=1, seed=len(lens) + d)
    items = B.pic_tree_plan_debug(b.cfg, b.host)
    assert (items[:, 3] - items[:, 2]).max() <= 32   # row tiles of 16 or 32
    worst = worst_of(b, G.f64(b.run()), two_part_bound)
    say(f"  {lens} D {d}: at most {worst:.2f} of the bound")
    assert worst <= 1


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_chain_agrees_with_prefill_and_one_token_with_decode(dtype):
    """Both signs.  Two bf16 results of one row differ by their roundings, 2^-8 of each, and by what
    roundings of rotated q, k and cos/sin to 8 bits do to a score: a sum of 128 errors of up to 2^-8 q k
    each, 5e-3 at its standard deviation, which moves an output by no more of its values' spread."""
    most = 5e-2 if dtype == torch.bfloat16 else 1e-4
    for n in (1, 9, 50):
        b = G.Drafts([(210, n), (35, n)], 8, 2, 128, dtype, see=lambda rng, m: np.tril(np.ones((m, m), bool)),
                     positions=lambda rng, m: np.arange(m), seed=n + 100)
        tree, o = G.f64(b.run()), torch.empty_like(b.q)
        for decode in (False, True) if n == 1 else (False,):
            ws = torch.empty(max(1, B.pic_workspace_size(b.cfg, b.host, decode)), dtype=torch.uint8, device="cuda")
            (B.pic_attn_decode if decode else B.pic_attn_prefill)(b.cfg, b.host, b.block_tables, b.positions, b.q, o, b.k_pool,
                                                                  b.v_pool, workspace=ws)
            off = float(np.abs(tree - G.f64(o)).max())
            say(f"  {n} tokens, {'decode' if decode else 'prefill'}: {off:.2e}")
            assert off < most   # (a NaN is no less)
