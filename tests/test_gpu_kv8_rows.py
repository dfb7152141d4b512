"""pic_kv8_write takes a block's rows from anywhere in a call: padding and rows of other blocks among them, in any
order, few rows and more than one workgroup looks through."""
import numpy as np
import pytest
import torch

from tests import kv8_util as K8
from tests.test_gpu_kv8 import CODES, DTYPES, Store, dev, f64

pytestmark = pytest.mark.gpu

B = pytest.importorskip("paper_2606_13126_amd._binding")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def by_blocks(slots, nb):
    """The last row of every slot that a call stores, block by block, padding left out: an order in which the rows of a
    block follow one another."""
    last = {int(s): i for i, s in enumerate(slots) if 0 <= s < nb * 16}
    return np.array([last[s] for s in sorted(last)], np.int64)


def put(st, slots, kv):
    """Store.put with the model's rows sorted by blocks."""
    slots = np.asarray(slots, np.int32)
    B.pic_kv8_write(st.cfg, st.pool, kv[0].cuda(), kv[1].cuda(), dev(slots))
    order = by_blocks(slots, st.nb)
    for i in range(2):
        K8.write(st.codes[i], st.scale[..., i], f64(kv[i])[order], slots[order], st.code)
    st.same()
    assert not torch.signbit(st.pool.scale).any()


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("hkv,d", [(1, 64), (5, 128)])
def test_rows_between_rows_of_a_block(code, dtype, hkv, d):
    """Padding, and rows of other blocks, between two rows of one; blocks that start and blocks that grow."""
    for what in ([3, -1, 4], [3, 20, 4], [1, -1, 0], [17, 0, -1, 18, 1, 16, 2], [5, 25, 5, 26, 5], [33, -5, 9999, 34, 40, -1, 33]):
        for size in (1.0, 30.0):
            st = Store(4, hkv, d, code, dtype, seed=len(what), scale=2.0 ** -5)
            put(st, what, st.rows(len(what), size))
            put(st, what[::-1], st.rows(len(what), 4 * size))


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("n", [64, 65, 200, 1024, 1025, 3000, 12000])
def test_rows_in_any_order(code, n):
    """Tokens of many requests, token by token; shuffled; shuffled within a block's reach; twice, with padding."""
    hkv, d, dtype = {1025: (5, 64, torch.float32), 3000: (3, 128, torch.bfloat16), 12000: (1, 64, torch.bfloat16)}.get(n, (2, 64, torch.bfloat16))
    nb = n // 8 + 8
    rng = np.random.default_rng(n)
    blocks = rng.permutation(nb)
    reqs = max(1, n // 24)
    per = -(-n // reqs)
    first = rng.integers(0, 16, reqs)
    need = -(-(first + per) // 16)
    base = np.concatenate([[0], np.cumsum(need)[:-1]])
    assert need.sum() <= nb
    slot = lambda r, t: blocks[base[r] + (first[r] + t) // 16] * 16 + (first[r] + t) % 16   # noqa: E731
    by_token = np.array([slot(r, t) for t in range(per) for r in range(reqs)])[:n]
    any_order = rng.permutation(by_token)
    near = np.sort(by_token)
    for i in range(0, n, 40):
        near[i:i + 40] = rng.permutation(near[i:i + 40])
    twice = rng.choice(by_token, n)
    twice[::7] = -1
    for slots in (by_token, any_order, near, twice) if n < 2000 else (by_token, twice):
        st = Store(nb, hkv, d, code, dtype, seed=n, scale=2.0 ** -6)
        kv = st.rows(n, 2.0)
        put(st, slots, kv)
        if n < 2000 or slots is twice:
            put(st, rng.permutation(slots), [x * 3 for x in kv])


@pytest.mark.parametrize("n", [100, 9000])
def test_scales_of_unused_memory(n):
    """Blocks that start need no scale: NaN and negative numbers, as fresh memory holds them."""
    nb = -(-n // 16)
    st = Store(nb, 2, 64, K8.INT8, torch.bfloat16, seed=n)
    st.pool.scale.copy_(torch.where(torch.rand_like(st.pool.scale) < 0.5, -3.0, float("nan")))
    kv = st.rows(nb * 16)
    put(st, np.random.default_rng(n).permutation(nb * 16), kv)


def test_captured_and_replayed():
    """More rows than a workgroup looks through, in any order: every replay is what an eager call gives."""
    n, nb = 9000, 700
    rng = np.random.default_rng(1)
    slots = dev(rng.permutation(nb * 16)[:n].astype(np.int32))
    a, b = (Store(nb, 1, 64, K8.E4M3, torch.bfloat16, seed=2, scale=2.0 ** -6) for _ in range(2))
    rows = [x.cuda() for x in a.rows(n)]
    buf = [x.clone() for x in rows]
    B.pic_kv8_write(a.cfg, a.pool, *buf, slots)
    B.pic_kv8_write(b.cfg, b.pool, *buf, slots)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.pic_kv8_write(a.cfg, a.pool, *buf, slots, stream=torch.cuda.current_stream())
    for i in range(4):
        for x, y in zip(buf, rows):
            x.copy_(y * 2.0 ** i)
        graph.replay()
        B.pic_kv8_write(b.cfg, b.pool, *buf, slots)
        torch.cuda.synchronize()
        assert torch.equal(a.pool.k, b.pool.k) and torch.equal(a.pool.v, b.pool.v) and torch.equal(a.pool.scale, b.pool.scale)
        assert (a.pool.scale > 0).all()
