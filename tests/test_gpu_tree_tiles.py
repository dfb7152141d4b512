"""pic_attn_tree in bf16 at its row tiles of 32, 128 and 256 query rows against float64.  The tile is
chosen for a whole call, by its cost, and small calls take 16 rows: here the trees that a test is
about stand in a call beside others that make it take the tile that the test names, which the plan
then has to show."""
import numpy as np
import pytest
import torch

from tests import test_gpu_tree as G
from tests import tree_util as T
from tests.gpu_util import say

pytestmark = pytest.mark.gpu

B = pytest.importorskip("paper_2606_13126_amd._binding")
TILES = [32, 128, 256]
FEW = 8   # spans that the short kernel arguments hold


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def host_batch(lens):
    seq, cu, start, flags, win = [], [0], [], [], []
    for ctx, n, w in lens:
        if ctx:
            start.append(0), flags.append(B.PIC_PDEP), win.append(-1)
        start.append(ctx), flags.append(B.PIC_PDEP | B.PIC_QUERY), win.append(w)
        seq.append(ctx + n)
        cu.append(len(start))
    return B.HostBatch(seq, cu, start, flags, win)


def plan_of(hq, hkv, d, lens):
    """Row tile of the call (None where no tree is longer than one), and the requests with key splits."""
    items = B.pic_tree_plan_debug(B.make_config(hq, hkv, d), host_batch(lens))
    first = np.unique(items[:, 2])
    return (int(first[1]) if len(first) > 1 else None), set(items[items[:, 7] >= 0, 0].tolist())


def beside(edges, tile, split, hq, hkv, d, most=1000):
    """Trees with which the call of `edges` takes `tile`, and splits the keys of the first edge or no keys
    at all (None: either); at most `most` in all."""
    g = hq // hkv
    found = []
    for reqs in (1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64, 96, 128):
        for rows in (48, 320, 513, 1030, 2050, 4100, 8200, 16400):
            for ctx in (20, 100, 300):
                n = rows // g + 1
                if reqs * n * hq <= 140000 and reqs + len(edges) <= most:
                    found.append((reqs * n * hq * (ctx + n), reqs, n, ctx))
    for _, reqs, n, ctx in sorted(found):
        lens = edges + [(ctx, n, 0)] * reqs
        got, splits = plan_of(hq, hkv, d, lens)
        if got == tile and (split is None or (0 in splits if split else not splits)):
            return lens[len(edges):]
    raise AssertionError(f"none of these calls takes row tiles of {tile}")


class Tiled(G.Drafts):
    def __init__(self, edges, tile, split=False, hq=8, hkv=2, d=128, most=1000, **kw):
        edges = [(e + (0,))[:3] for e in edges]
        lens = edges + beside(edges, tile, split, hq, hkv, d, most)
        self.edges = len(edges)
        super().__init__(lens, hq, hkv, d, **kw)
        assert plan_of(hq, hkv, d, lens)[0] == tile

    def rows_of(self, r):
        """Query rows of request r."""
        at = sum(n for _, n, _ in self.lens[:r])
        return slice(at, at + self.lens[r][1])

    def check(self, got, what=""):
        """As Drafts.check (its comment derives the bound): every output of the edges, some of two others."""
        rot, scale, worst = self.rot or self.d, self.d ** -0.5, 0.0
        each = 0.0 if self.prerotated else 2.0 ** -11 + G.ANGLE_ADVANCED
        row, off = 0, 0
        for r, (ctx, n, w) in enumerate(self.lens):
            L = ctx + n
            if self.edges <= r < len(self.lens) - 2:
                row, off = row + n, off + L
                continue
            pick = np.arange(n) if r < self.edges else np.unique(np.r_[0, n // 3, max(0, n - 2), n - 1])
            j = torch.arange(w, L, device="cuda")
            blk = torch.from_numpy(self.table[r].astype(np.int64)).cuda()[j // 16]
            k, v = (G.f64(p[blk, :, j % 16]) for p in (self.k_pool, self.v_pool))
            q = G.f64(self.q[row:row + n])[pick]
            if not self.prerotated:
                k = T.rotate(k, self.pos[off + w:off + L], rot, self.theta, self.style, self.inv_freq)
                q = T.rotate(q, self.pos[off + ctx:off + L][pick], rot, self.theta, self.style, self.inv_freq)
            see = G.dev(np.concatenate([np.ones((len(pick), ctx - w), bool), self.see[r][pick]], 1))
            nq, nk = np.linalg.norm(q, axis=-1).max(), np.linalg.norm(k, axis=-1).max()
            ds = nq * nk * scale * (2 * each + each * each + self.d * 2.0 ** -24)
            e = np.expm1(ds) + 2.0 ** -8 + 2.0 ** -20
            assert e < 0.5, "inputs too large for the bound"
            q, k, v = G.dev(q), G.dev(k), G.dev(v)
            g = self.hq // self.hkv
            for h in range(self.hq):
                s = torch.where(see, (q[:, h] @ k[:, h // g].T.contiguous()) * scale, -torch.inf)
                p = torch.exp(s - s.amax(-1, keepdim=True))
                p = torch.where(see.any(-1, keepdim=True), p / p.sum(-1, keepdim=True), 0.0)
                vv = v[:, h // g].contiguous()
                o = p @ vv
                spread = torch.cat([(p[i:i + 32, :, None] * (vv - o[i:i + 32, None]).abs()).sum(1) for i in range(0, len(o), 32)])
                tol = e / (1 - e) * spread + (2.0 ** -8 * 1.01 + 2.0 ** -20) * (o.abs() + spread) + 1e-30
                x = got[row + G.dev(pick), h].double()
                assert torch.isfinite(x).all(), (what, r, h)
                ratio = float(((x - o).abs() / tol).max())
                worst = max(worst, ratio)
                assert ratio <= 1, (what, r, h, self.lens[r], ratio)
            row, off = row + n, off + L
        say(f"  {what}: {len(self.lens)} trees, at most {worst:.2f} of the bound")


def edge_nodes(g):
    """Tokens whose rows are one, fill or underfill a wave's rows, a tile, and spill over it."""
    return sorted({1, 2, max(1, 16 // g), 16 // g + 1, 32 // g + 1, max(1, 96 // g), 128 // g + 1, 256 // g + 1})


@pytest.mark.parametrize("tile", TILES)
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 4, 64), (16, 1, 128), (7, 1, 64)])
def test_lengths(tile, hq, hkv, d):
    nodes = edge_nodes(hq // hkv)
    for i, ctx in enumerate((0, 1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 700)):
        b = Tiled([(ctx, n) for n in nodes], tile, None, hq, hkv, d, style=i % 2, seed=ctx)
        b.check(b.run(), f"tile {tile} ctx {ctx}")


@pytest.mark.parametrize("tile", [None] + TILES)
@pytest.mark.parametrize("hq,hkv,d", [(8, 8, 64), (24, 8, 128), (32, 16, 64), (5, 1, 128), (128, 1, 64), (12, 12, 128)])
def test_heads(tile, hq, hkv, d):
    """Every way of laying a span's workgroups out over the dies (8 KV heads, 8 key splits, neither)."""
    g = hq // hkv
    edges = [(2500, 40 // g + 1), (130, 1), (700, 130 // g + 1), (3000, max(1, 16 // g), 1001), (0, 2)]
    if tile is not None:
        b = Tiled(edges, tile, None, hq, hkv, d, seed=hq)
        b.check(b.run(), f"tile {tile}")
        return
    for dtype in (torch.bfloat16, torch.float32):   # (as the call itself chooses)
        for lens in (edges, edges[:1]):
            b = G.Drafts(lens, hq, hkv, d, dtype, seed=hq)
            b.check(b.run(), str(dtype))


@pytest.mark.parametrize("tile", TILES)
def test_few_spans(tile):
    for hq, hkv, d in ((8, 2, 64), (4, 4, 128), (16, 1, 128)):
        g = hq // hkv
        for ctx, nodes in ((0, (1, 32 // g + 1)), (31, (96 // g, 16 // g + 1)), (700, (256 // g + 1, 2))):
            b = Tiled([(ctx, n) for n in nodes], tile, None, hq, hkv, d, FEW, seed=ctx)
            assert len(b.lens) <= FEW
            b.check(b.run(), f"tile {tile} ctx {ctx}")


@pytest.mark.parametrize("tile", TILES)
def test_more_spans_than_the_arguments_hold(tile):
    for hq, hkv, d in ((8, 2, 64), (16, 1, 128)):
        edges = [(c, n) for c in (0, 1, 16, 33, 64, 100, 129, 333) for n in edge_nodes(hq // hkv)[:5 if tile == 32 else None]] + [(50 + i, 1 + i % 9) for i in range(40)]
        b = Tiled(edges, tile, None, hq, hkv, d, seed=hq)
        assert len(b.lens) > 64
        b.check(b.run(), f"tile {tile}, {len(b.lens)} spans")


@pytest.mark.parametrize("tile", TILES)
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 4, 64), (16, 1, 64)])
def test_key_splits(tile, hq, hkv, d):
    g = hq // hkv
    for ctx in (4999, 9000):
        b = Tiled([(ctx, 40 // g + 1), (ctx, 1), (ctx - 63, 140 // g), (3000, 300 // g, 1001), (7, 2)], tile, True, hq, hkv, d, seed=ctx)
        b.check(b.run(), f"tile {tile} ctx {ctx}")


@pytest.mark.parametrize("tile", TILES)
@pytest.mark.parametrize("style,rot,prerotated", [(0, 0, 0), (1, 0, 0), (0, 32, 0), (0, 16, 0), (1, 34, 0), (1, 2, 0), (0, 0, 1), (0, 64, 1)])
@pytest.mark.parametrize("d", [64, 128])
def test_rotations(tile, style, rot, prerotated, d):
    b = Tiled([(150, 5), (150, 40), (150, 70), (290, 3), (16, 1)], tile, False, 8, 2, d, style=style, rot=rot, prerotated=prerotated, seed=d)
    o = b.run()
    b.check(o, f"tile {tile}")
    if not prerotated:
        assert torch.equal(b.run(table=b.rope_table(100)), o)   # (a table is not read in bf16)
    freq = 5e5 ** (-2.0 * np.arange(d // 4) / (d // 2)) / np.linspace(1, 8, d // 4)
    b = Tiled([(200, 4), (200, 50)], tile, False, 8, 2, d, style=style, rot=d // 2, prerotated=prerotated, inv_freq=freq, seed=rot)
    b.check(b.run(), f"tile {tile}, frequencies")


@pytest.mark.parametrize("tile", TILES)
@pytest.mark.parametrize("kind", ["far", "negative", "scattered", "jumps", "least", "around"])
def test_positions(tile, kind):
    """Logical positions of any kind; 5,000 keys, so that a lane's angles are renewed on the way."""
    def positions(rng, n):
        p = np.arange(n)
        if kind == "scattered":
            return rng.integers(-(1 << 31), 1 << 31, n)
        if kind == "around":   # past the type's end to its start
            return (p + (1 << 32) - 700) % (1 << 32) - (1 << 31)
        return {"far": p + (1 << 30), "negative": p - 5000, "least": p - (1 << 31), "jumps": p + 1000 * (p // 150)}[kind]
    for style, d in ((0, 128), (1, 64)):
        b = Tiled([(5000, 6), (5000, 60), (333, 33)], tile, True, 8, 2, d, style=style, positions=positions, seed=3)
        b.check(b.run(), f"tile {tile} {kind}")


@pytest.mark.parametrize("tile", TILES)
@pytest.mark.parametrize("d", [64, 128])
def test_windows(tile, d):
    edges = [(333, n, w) for w in (0, 1, 15, 16, 100, 333) for n in (3, 33)] + [(400, 2, 399)]
    b = Tiled(edges, tile, False, 8, 2, d, seed=d)
    b.check(b.run(), f"tile {tile}")
    # what lies outside the window is not read
    for r, (ctx, n, w) in enumerate(b.lens[:b.edges]):
        for j in range(w):
            G.poison(b, r, j, (float("nan"), float("nan")))
    b.check(b.run(), f"tile {tile}, NaN outside the windows")


@pytest.mark.parametrize("tile", TILES)
@pytest.mark.parametrize("d", [64, 128])
def test_any_mask(tile, d):
    """Rows that see nothing, later tokens, not themselves; bits past the span are ignored."""
    def see(rng, n):
        s = rng.random((n, n)) < 0.3
        s[::3] = False
        return s
    edges = [(c, n) for c in (0, 40) for n in (1, 5, 20, 70)]
    b = Tiled(edges, tile, False, 8, 2, d, see=see, seed=d)
    clean = b.run()
    b.check(clean, f"tile {tile}")
    words = b.mask.cpu().numpy().view(np.uint64).copy()
    row = 0
    for c, n, w in b.lens:
        for j in range(n, b.words * 64):
            words[row:row + n, j // 64] |= np.uint64(1) << np.uint64(j % 64)
        row += n
    b.mask = G.dev(words.view(np.int64))
    o = b.run()
    assert torch.equal(o, clean)
    for r, (c, n, w) in enumerate(b.lens[:b.edges]):
        nothing = ~b.see[r].any(1)
        if c == 0:
            assert nothing.any() and (G.f64(o[b.rows_of(r)])[nothing] == 0).all()


@pytest.mark.parametrize("tile", TILES)
@pytest.mark.parametrize("d,prerotated,split", [(128, 0, False), (64, 1, False), (64, 0, False), (128, 1, False), (128, 0, True), (64, 0, True)])
def test_unseen_tokens_do_not_matter(tile, d, prerotated, split):
    """Infinities and NaN in keys and values of tokens that a row does not see leave it bit for bit;
    infinities that it sees arrive in their own dimensions."""
    edges = [(5000 if split else 77, 30), (77, 3), (300, 7), (300, 70), (0, 40), (50, 130)]
    b = Tiled(edges, tile, split, 8, 2, d, prerotated=prerotated, seed=d)
    bad = [n // 2 for _, n in edges]
    sees = torch.zeros(len(b.q), dtype=torch.bool, device="cuda")

    def poison(kv):
        for r in range(b.edges):
            G.poison(b, r, edges[r][0] + bad[r], kv)
    for r in range(b.edges):
        sees[b.rows_of(r)] = G.dev(b.see[r][:, bad[r]])
    poison((0.0, 0.0))
    ref = b.run()
    assert torch.isfinite(ref).all()
    for kv in ((float("nan"), float("inf")), (float("inf"), float("nan")), (None, -float("inf")), (float("nan"), None)):
        poison(kv)
        o = b.run()
        assert torch.equal(o[~sees], ref[~sees])
        assert not torch.isfinite(o[sees].flatten(1)).all(1).any()
    v = torch.ones(d, device="cuda", dtype=torch.bfloat16)
    v[::4], v[1::4], v[2::4] = float("inf"), -float("inf"), float("nan")
    poison((0.0, v))
    o = b.run()
    assert torch.equal(o[~sees], ref[~sees])
    o = G.f64(o[sees])
    assert (o[..., ::4] == np.inf).all() and (o[..., 1::4] == -np.inf).all() and np.isnan(o[..., 2::4]).all() and np.isfinite(o[..., 3::4]).all()


@pytest.mark.parametrize("tile", TILES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("split", [False, True])
def test_infinities_of_the_context(tile, d, split):
    """Infinities in values that every row sees, of one sign or both, arrive as they are."""
    edges = [(5000 if split else 300, 20), (300, 3), (90, 7), (500, 70), (75, 70), (110, 40)]
    b = Tiled(edges, tile, split, 8, 2, d, seed=d)
    v = torch.ones(d, device="cuda", dtype=torch.bfloat16)
    v[::4], v[1::4], v[2::4] = float("inf"), -float("inf"), float("nan")
    w, x = v.clone(), v.clone()
    w[0] = x[0] = 1
    x[4] = -float("inf")
    for r in range(b.edges):
        for j, value in ((5, v), (70, w), (71, x)):
            G.poison(b, r, j, (None, value))
    got = b.run()
    for r in range(b.edges):
        o = G.f64(got[b.rows_of(r)])
        assert (o[..., 0] == np.inf).all() and np.isnan(o[..., 4]).all() and (o[..., 8::4] == np.inf).all(), r
        assert (o[..., 1::4] == -np.inf).all() and np.isnan(o[..., 2::4]).all() and np.isfinite(o[..., 3::4]).all(), r
    rest = got[sum(n for _, n in edges):]
    assert torch.isfinite(rest).all()


@pytest.mark.parametrize("tile", TILES)
@pytest.mark.parametrize("power", [-124, -60, -20, 17, 60, 124])
def test_large_and_small_keys(tile, power):
    """Keys far from 1, queries as far the other way: float16 holds them by powers of two."""
    for style, d in ((0, 128), (1, 128), (0, 64)):
        b = Tiled([(130, 5), (130, 40), (0, 70)], tile, False, 8, 2, d, style=style, seed=5, kscale=2.0 ** power, qscale=2.0 ** -power)
        b.check(b.run(), f"tile {tile} 2^{power}")


@pytest.mark.parametrize("tile", TILES)
def test_keys_of_mixed_sizes(tile):
    b = Tiled([(130, 40), (200, 7)], tile, False, 8, 2, 128, seed=7, qscale=2.0 ** -20)
    for j in (3, 64, 100, 131):
        G.poison_key(b, j, 2.0 ** 20)
    for j in (1, 65):
        G.poison_key(b, j, 2.0 ** -20)
    b.check(b.run(), f"tile {tile}")
    b = Tiled([(130, 40), (200, 7)], tile, False, 8, 2, 128, seed=3)
    for dim in range(128):
        if dim % 64 == 0:   # the pair that the queries do not have
            b.q[..., dim] = 0
            b.k_pool[..., dim] = 2.0 ** -7
        else:
            b.q[..., dim] *= 2.0 ** 14
            b.k_pool[..., dim] /= 2.0 ** 14
    b.check(b.run(), f"tile {tile}, small beside large")


@pytest.mark.parametrize("tile", TILES)
def test_writes_its_rows_only(tile):
    for split in (False, True):
        b = Tiled([(5000 if split else 500, 40), (64, 3)], tile, split, 8, 2, 128, seed=tile)
        pools = [b.k_pool.clone(), b.v_pool.clone()]
        o = b.run()
        guarded = torch.full((len(b.q) + 2, 8, 128), 7.0, dtype=torch.bfloat16, device="cuda")
        ws = torch.full((b.ws.numel() + 512,), 255, dtype=torch.uint8, device="cuda")
        b.run(o=guarded[1:-1], ws=ws[:b.ws.numel()])
        assert (guarded[0] == 7).all() and (guarded[-1] == 7).all() and (ws[b.ws.numel():] == 255).all()
        assert torch.equal(b.k_pool, pools[0]) and torch.equal(b.v_pool, pools[1])
        assert torch.equal(guarded[1:-1], o)


@pytest.mark.parametrize("tile", TILES)
def test_captured_and_replayed(tile):
    b = Tiled([(5000, 40), (64, 3)], tile, True, 8, 2, 128, seed=tile)
    ref = b.run()
    torch.cuda.synchronize()
    o = torch.zeros_like(ref)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.run(o=o, stream=torch.cuda.current_stream())
    for i in range(4):
        o.zero_()
        b.ws.fill_(255)
        b.q.copy_(b.q.flip(0))   # other queries in the same place
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, b.run())
    assert torch.equal(o, ref)   # an even number of times over
