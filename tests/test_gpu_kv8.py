"""The cache held in 8 bits on the GPU against plain float64: norms, the store, reading back and
attention, at the sizes, masks and values where they can go wrong, and a step of all of them."""
import numpy as np
import pytest
import torch

from tests import kv8_util as K8
from tests import tree_util as T
from tests.gpu_util import say

pytestmark = pytest.mark.gpu

B = pytest.importorskip("paper_2606_13126_amd._binding")
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}   # of a rounding, relative
# cos/sin in float32: the phase rounded to 24 bits (pi 2^-24), the sine of it to a few units, and in
# the bf16 attention 32 advances of at most 2^-22 each
ANGLE, ANGLE_ADVANCED = 2.0 ** -21, 2.0 ** -17
DTYPES = [torch.bfloat16, torch.float32]
CODES = [K8.E4M3, K8.INT8]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def cfg_of(hq, hkv, d, dtype, style=0, rot=0, prerotated=0, theta=1e4, scale=0.0, inv_freq=None):
    return B.make_config(hq, hkv, d, dtype=B.PIC_F32 if dtype == torch.float32 else B.PIC_BF16, rope_theta=theta, rope_style=style,
                         rotary_dim=rot, k_prerotated=prerotated, softmax_scale=scale, inv_freq=inv_freq)


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def f64(t):
    return t.detach().double().cpu().numpy()


def pool_of(codes_k, codes_v, scale, code):
    """A pool of host bytes [blocks][H][16][D] and scales [blocks][H][2]."""
    return B.Kv8Pool(dev(codes_k), dev(codes_v), dev(np.asarray(scale, np.float32)), code)


def random_pool(rng, nb, hkv, d, code, powers=True):
    """Full blocks of normally distributed rows, the sizes of whose blocks differ."""
    out, scale = [], np.zeros((nb, hkv, 2), np.float32)
    for i in range(2):
        x = rng.standard_normal((nb, hkv, 16, d)) * np.exp2(rng.integers(-2, 3, (nb, hkv)))[:, :, None, None]
        size = np.abs(x).max((2, 3))
        s = np.vectorize(lambda m: K8.scale_of(m, code))(size) if powers else (size / K8.MOST[code]).astype(np.float32).astype(np.float64)
        scale[..., i] = s
        out.append(K8.encode(x / s[:, :, None, None], code))
    return out[0], out[1], scale


# ------------------------------------------------------------------------------------
# pic_qk_norm
# ------------------------------------------------------------------------------------

def check_norm(got, x, w, pos, cfg_kw, rotate, eps, what):
    """A head's sum of D squares is off by D 2^-24 of itself, so its root by half of that; root, division, product with
    the weight and the turn round a few times more; angles are within ANGLE of a pair's size; the result rounds once."""
    d = x.shape[-1]
    ref = K8.norm(f64(x), None if w is None else f64(w), eps)
    size = np.abs(ref)
    if rotate:
        rot = cfg_kw.get("rot") or d
        style = cfg_kw.get("style", 0)
        half = rot // 2
        a, b = (ref[..., :half], ref[..., half:rot]) if style == 0 else (ref[..., 0:rot:2], ref[..., 1:rot:2])
        pair = np.hypot(a, b)
        size = np.abs(ref).copy()
        if style == 0:
            size[..., :half] = size[..., half:rot] = pair
        else:
            size[..., 0:rot:2] = size[..., 1:rot:2] = pair
        ref = T.rotate(ref, pos, rot, 1e4, style)
    tol = size * ((d / 2 + 12) * 2.0 ** -24 + (ANGLE if rotate else 0)) + HALF_STEP[got.dtype] * np.abs(ref) * 1.001
    off = np.abs(f64(got) - ref)
    assert (off <= tol + 1e-38).all(), (what, float((off / (tol + 1e-38)).max()))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d,style,rot", [(128, 0, 0), (64, 0, 0), (128, 1, 0), (64, 1, 34), (128, 0, 32), (64, 0, 16), (64, 1, 2)])
@pytest.mark.parametrize("rotate", [0, 1])
def test_qk_norm(dtype, d, style, rot, rotate):
    for n, hq, hkv in ((1, 1, 1), (7, 8, 2), (33, 28, 4), (5, 64, 8)):
        g = torch.Generator(device="cuda").manual_seed(n)
        qkv = torch.randn(n, hq + 2 * hkv, d, generator=g, device="cuda")
        qkv *= torch.exp2(torch.randint(-12, 12, (n, hq + 2 * hkv, 1), generator=g, device="cuda").float())
        qkv = qkv.to(dtype)
        before = qkv.clone()
        q, k = qkv[:, :hq], qkv[:, hq:hq + hkv]
        wq, wk = (torch.randn(d, generator=g, device="cuda").to(dtype) for _ in range(2))
        pos = dev(np.random.default_rng(n).integers(-2**31, 2**31 - 1, n).astype(np.int32))
        cfg = cfg_of(hq, hkv, d, dtype, style, rot, prerotated=rotate)
        qo, ko = torch.full_like(q.contiguous(), float("nan")), torch.full_like(k.contiguous(), float("nan"))
        B.pic_qk_norm(cfg, q, k, wq, wk, 1e-6, pos if rotate else None, q_out=qo, k_out=ko)
        assert torch.equal(qkv, before)
        kw = dict(style=style, rot=rot)
        check_norm(qo, q, wq, f64(pos), kw, rotate, 1e-6, "q")
        check_norm(ko, k, wk, f64(pos), kw, rotate, 1e-6, "k")
        # in place inside the fused rows, without weights, and one of the two alone: the same bits
        B.pic_qk_norm(cfg, q, k, wq, wk, 1e-6, pos if rotate else None)
        assert torch.equal(q, qo) and torch.equal(k, ko) and torch.equal(qkv[:, hq + hkv:], before[:, hq + hkv:])
        alone = torch.empty_like(ko)
        B.pic_qk_norm(cfg, None, before[:, hq:hq + hkv], None, wk, 1e-6, pos, k_out=alone)
        assert torch.equal(alone, ko)
        plain = torch.empty_like(qo)
        B.pic_qk_norm(cfg, before[:, :hq], None, None, None, 0.5, pos, q_out=plain)
        check_norm(plain, before[:, :hq], None, f64(pos), kw, rotate, 0.5, "no weight")


def test_qk_norm_of_zeros_and_large_rows():
    cfg = cfg_of(2, 1, 64, torch.float32)
    q = torch.zeros(2, 2, 64, device="cuda")
    q[1] = 2.0 ** 59
    k = torch.full((2, 1, 64), 2.0 ** -70, device="cuda")
    B.pic_qk_norm(cfg, q, k, None, None, 1e-6)
    assert torch.equal(q[0], torch.zeros(2, 64, device="cuda"))
    assert (q[1] - 1).abs().max() < 1e-5
    assert torch.allclose(k.double(), torch.full_like(k, 2.0 ** -70).double() * 1e3, rtol=1e-5)   # 1 / sqrt(eps)


# ------------------------------------------------------------------------------------
# pic_kv8_write, pic_kv8_read
# ------------------------------------------------------------------------------------

class Store:
    """A pool on the device beside its model on the host."""

    def __init__(self, nb, hkv, d, code, dtype, seed=0, scale=0.0):
        self.rng = np.random.default_rng(seed)
        self.nb, self.hkv, self.d, self.code, self.dtype = nb, hkv, d, code, dtype
        self.cfg = cfg_of(hkv, hkv, d, dtype)
        self.codes = [self.rng.integers(0, 127, (nb, hkv, 16, d)).astype(np.uint8) for _ in range(2)]
        self.scale = np.full((nb, hkv, 2), scale, np.float64)
        self.pool = pool_of(self.codes[0], self.codes[1], self.scale, code)

    def rows(self, n, size=1.0):
        return [torch.from_numpy(self.rng.standard_normal((n, self.hkv, self.d)) * size).to(self.dtype) for _ in range(2)]

    def put(self, slots, kv, fused=False):
        slots = np.asarray(slots, np.int32)
        n = len(slots)
        on = [t.cuda() for t in kv]
        if fused:   # slices of one projection behind a query
            all_ = torch.cat([torch.full((n, 1, self.d), float("nan"), dtype=self.dtype, device="cuda"), *on], 1)
            on = [all_[:, 1:1 + self.hkv], all_[:, 1 + self.hkv:]]
        B.pic_kv8_write(self.cfg, self.pool, on[0], on[1], dev(slots))
        for i in range(2):
            s = self.scale[..., i]
            K8.write(self.codes[i], s, f64(kv[i]), slots, self.code)
        self.same()

    def same(self):
        torch.cuda.synchronize()
        assert np.array_equal(self.pool.scale.cpu().numpy().astype(np.float64), self.scale)
        for t, c in zip((self.pool.k, self.pool.v), self.codes):
            got = t.cpu().numpy()
            if not np.array_equal(got, c):
                at = np.argwhere(got != c)[0]
                raise AssertionError((at, got[tuple(at)], c[tuple(at)], int((got != c).sum())))

    def check_read(self, slots):
        slots = np.asarray(slots, np.int32)
        out = [torch.full((len(slots), self.hkv, self.d), 7.0, dtype=self.dtype, device="cuda") for _ in range(2)]
        B.pic_kv8_read(self.cfg, self.pool, dev(slots), out[0], out[1])
        for i in range(2):
            x = K8.decode(self.codes[i], self.code) * self.scale[..., i][:, :, None, None]
            ref = np.full((len(slots), self.hkv, self.d), 7.0)
            for r, s in enumerate(slots):
                if 0 <= s < self.nb * 16:
                    ref[r] = x[s // 16, :, s % 16]
            want = torch.from_numpy(ref).to(torch.float32).to(self.dtype)   # (exact in float32)
            assert torch.equal(out[i].cpu(), want)


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("hkv,d", [(1, 64), (2, 128), (5, 128), (12, 64)])
def test_write_blocks_that_start(code, dtype, hkv, d):
    st = Store(9, hkv, d, code, dtype, seed=hkv)
    for i, n in enumerate((1, 2, 15, 16)):
        st.put(16 * i + np.arange(n), st.rows(n, 2.0 ** (3 * i)), fused=i % 2 == 1)
    st.put(64 + np.arange(63), st.rows(63))   # several blocks, the last of them not full
    st.check_read([0, 1, 33, 64, 126, 143, -1, 144, 70, 70])


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("hkv,d", [(3, 64), (2, 128)])
def test_write_token_by_token(code, dtype, hkv, d):
    """Every token behind the others: scales grow, and the rows kept are rounded to them."""
    st = Store(6, hkv, d, code, dtype, seed=d)
    order = st.rng.permutation(6)
    slots = np.concatenate([order[b] * 16 + np.arange(16) for b in range(6)])
    size = np.exp2(st.rng.integers(-6, 7, len(slots)))
    for i, s in enumerate(slots[:70]):
        st.put([s], st.rows(1, size[i]), fused=i % 3 == 0)
    st.put(slots[70:], st.rows(len(slots) - 70, 100.0))
    st.check_read(slots)


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", DTYPES)
def test_write_a_step_of_many_requests(code, dtype):
    """One token each, blocks in any order, padding rows among them; some start their block."""
    st = Store(80, 4, 128, code, dtype, seed=3, scale=2.0 ** -5)
    blocks = st.rng.permutation(80)[:70]
    slots = blocks * 16 + st.rng.integers(0, 16, 70)
    slots[::9] = -1
    slots[5] = 80 * 16
    slots[6] = 2**31 - 1
    slots[7] = -2**31
    st.put(slots, st.rows(70, 3.0))
    st.check_read(slots)


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("hkv,d", [(1, 128), (2, 64)])
def test_write_long_prompts(code, hkv, d):
    """More rows than one workgroup looks through, from the middle of blocks on, and padding."""
    st = Store(160, hkv, d, code, torch.bfloat16, seed=5, scale=0.25)
    order = st.rng.permutation(160)
    flat = np.concatenate([order[b] * 16 + np.arange(16) for b in range(160)])
    slots = np.concatenate([flat[5:1100], [-1, -1, -1], flat[1100 + 4:2400], [-7]])
    st.put(slots, st.rows(len(slots), 2.0))
    st.check_read(flat)


@pytest.mark.parametrize("n", [256, 257, 512, 513, 1024, 1025, 2048, 2049])
def test_write_rows_and_their_workgroups(n):
    """The numbers of rows around which a workgroup looks through twice as many: runs of 1 to 40 tokens, padding between."""
    st = Store(n // 4 + 400, 2, 64, K8.INT8 if n % 2 else K8.E4M3, torch.bfloat16, seed=n, scale=2.0 ** -6)
    blocks = iter(st.rng.permutation(st.nb))
    slots = []
    while len(slots) < n:
        run, first = int(st.rng.integers(1, 41)) if st.rng.random() < 0.4 else 1, int(st.rng.integers(0, 16))
        table = [next(blocks) for _ in range((first + run - 1) // 16 + 1)]
        slots += [table[(first + i) // 16] * 16 + (first + i) % 16 for i in range(run)] + [-1] * int(st.rng.integers(0, 2))
    st.put(np.array(slots[:n]), st.rows(n, 5.0))


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", DTYPES)
def test_write_what_is_no_number(code, dtype):
    """Infinities saturate, NaN is 0, and neither moves a scale; a block of zeros has the smallest."""
    st = Store(4, 2, 64, code, dtype, seed=1)
    k, v = st.rows(20)
    k[3, 0, 5], k[3, 0, 6], k[4, 1, 7] = float("inf"), -float("inf"), float("nan")
    v[:, 1] = float("nan")
    v[0, 0] = float("inf")
    k[16:] = 0.0
    st.put(np.arange(20), [k, v])
    st.check_read(np.arange(32))
    st.put([20], st.rows(1, 1e-3))


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", DTYPES)
def test_write_at_the_ends_of_the_type(code, dtype):
    big = float(torch.finfo(dtype).max)
    st = Store(8, 1, 64, code, dtype, seed=2)
    for i, s in enumerate((big, 2.0 ** 120, 448.0, 127.0, 2.0 ** -120, 2.0 ** -126, 1e-39)):
        k, v = st.rows(3)
        k = (k.double() / k.double().abs().max() * s).to(dtype)
        v = torch.full_like(v, s)
        st.put(16 * i + np.arange(3), [k, v])
        assert torch.isfinite(st.pool.scale).all()
    st.check_read(np.arange(8 * 16)[:100])


@pytest.mark.parametrize("code", CODES)
def test_write_ties_go_to_even(code):
    """Halfway between two codes, with a scale of 1 and with a smaller one."""
    st = Store(4, 1, 128, code, torch.float32)
    vals = K8.E4M3_VALUES if code == K8.E4M3 else np.arange(128.0)
    mid = (vals[1:] + vals[:-1]) / 2
    row = np.zeros(128)
    row[:len(mid)] = mid * np.where(np.arange(len(mid)) % 2, 1, -1)
    row[127] = K8.MOST[code]
    for b, s in enumerate((1.0, 2.0 ** -7)):
        x = torch.from_numpy(row * s).float().view(1, 1, 128)
        st.put([16 * b], [x, -x])
    assert st.scale[0, 0, 0] == 1.0 and st.scale[1, 0, 1] == 2.0 ** -7


def test_write_of_a_slot_twice():
    """Of rows that follow one another in one slot the last counts (also of more than a wave looks at)."""
    for n in (2, 5, 64, 65, 200):
        st = Store(2, 2, 64, K8.INT8, torch.bfloat16, scale=1.0)
        kv = st.rows(n + 2)
        st.put(np.concatenate([[17], np.full(n, 18), [19]]), kv)


def test_write_keeps_a_scale_that_is_no_power_of_two():
    """Scales of another program: a call that does not pass them keeps them and the codes."""
    st = Store(1, 1, 64, K8.INT8, torch.float32, scale=0.3)
    before = st.pool.k.clone()
    k, v = st.rows(1)
    B.pic_kv8_write(st.cfg, st.pool, k.cuda(), v.cuda(), dev(np.array([5], np.int32)))
    assert (st.pool.scale == np.float32(0.3)).all()
    other = [o for o in range(16) if o != 5]
    assert torch.equal(st.pool.k[:, :, other], before[:, :, other])
    got = st.pool.k[0, 0, 5].cpu().numpy().view(np.int8)
    assert (np.abs(got * np.float64(np.float32(0.3)) - f64(k)[0, 0]) <= 0.15 * (1 + 1e-5)).all()
    # ... and a larger row replaces them: half a step of rounding for the row, and one more for those kept
    B.pic_kv8_write(st.cfg, st.pool, k.cuda() * 1000, v.cuda() * 1000, dev(np.array([6], np.int32)))
    s = float(st.pool.scale[0, 0, 0])
    assert s == K8.scale_of(float(k.abs().max() * 1000), K8.INT8)
    kept = st.pool.k[0, 0, 5].cpu().numpy().view(np.int8) * s
    assert (np.abs(kept - got * 0.3) <= s / 2 * (1 + 1e-5)).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n", [1, 3, 65, 517, 4000])
def test_read_and_write_stay_in_their_rows(dtype, n):
    """Outputs inside a larger buffer, and a pool between two others: what lies around them keeps its bits."""
    nb = -(-n // 16)
    st = Store(nb, 2, 64, K8.INT8, dtype, seed=n)
    around = torch.full((3, nb, 2, 16, 64), 77, dtype=torch.uint8, device="cuda")
    st.pool = B.Kv8Pool(around[1], torch.zeros_like(around[1]), st.pool.scale, K8.INT8)
    k, v = (x.cuda() for x in st.rows(n))
    slots = dev(np.arange(n, dtype=np.int32))
    B.pic_kv8_write(st.cfg, st.pool, k, v, slots)
    assert (around[0] == 77).all() and (around[2] == 77).all()
    out = torch.full((3 * n + 128, 2, 64), 7.0, dtype=dtype, device="cuda")
    B.pic_kv8_read(st.cfg, st.pool, slots, out[:n], out[n:2 * n])
    assert (out[2 * n:] == 7.0).all()
    size = st.pool.scale[slots.long() // 16]
    for got, x, i in ((out[:n], k, 0), (out[n:2 * n], v, 1)):
        assert (got.float() - x.float()).abs().sub(size[..., i, None] * 0.5 * (1 + 2.0 ** -7)).max() <= 0


# ------------------------------------------------------------------------------------
# attention
# ------------------------------------------------------------------------------------

class Batch:
    """Requests of (cached tokens, new tokens, window start) over a pool of blocks in random order.  Decode: one new
    token each."""

    def __init__(self, lens, hq=8, hkv=2, d=128, dtype=torch.bfloat16, code=K8.E4M3, style=0, rot=0, prerotated=0, seed=0, positions=None,
                 inv_freq=None, theta=1e4, powers=True, qscale=1.0, decode=False, flags=None, softmax=0.0):
        rng = self.rng = np.random.default_rng(seed)
        self.lens = [(l + (0,))[:3] for l in lens]
        self.hq, self.hkv, self.d, self.dtype, self.code, self.style, self.rot = hq, hkv, d, dtype, code, style, rot
        self.prerotated, self.inv_freq, self.theta, self.decode, self.softmax = prerotated, inv_freq, theta, decode, softmax
        self.cfg = cfg_of(hq, hkv, d, dtype, style, rot, prerotated, theta, softmax, inv_freq)
        seq, cu, start, fl, win = [], [0], [], [], []
        for ctx, n, w in self.lens:
            if ctx:
                start.append(0), fl.append(B.PIC_PDEP), win.append(-1)
            start.append(ctx), fl.append(B.PIC_PDEP | B.PIC_QUERY), win.append(w)
            seq.append(ctx + n)
            cu.append(len(start))
        self.host = B.HostBatch(seq, cu, start, fl, win)
        need = [-(-s // 16) for s in seq]
        self.nb = sum(need) + 2
        table = np.full((len(seq), max(need) + 1), 2**30, np.int32)   # (past a request's blocks: never read)
        ids = rng.permutation(self.nb)
        for r, k in enumerate(need):
            table[r, :k], ids = ids[:k], ids[k:]
        self.table, self.spare = table, ids
        self.pos = (np.concatenate([np.arange(s) + rng.integers(0, 3000) for s in seq]) if positions is None
                    else positions(rng, sum(seq))).astype(np.int32)
        rows = sum(n for _, n, _ in self.lens)
        self.q = torch.from_numpy(rng.standard_normal((rows, hq, d)) * qscale).to(dtype).cuda()
        self.set_pool(*random_pool(rng, self.nb, hkv, d, code, powers))
        self.block_tables, self.positions = dev(table), dev(self.pos)
        self.ws = torch.empty(max(1, B.pic_attn8_workspace_size(self.cfg, self.host, decode)), dtype=torch.uint8, device="cuda")

    def set_pool(self, k, v, scale):
        self.k_codes, self.v_codes, self.scale = k, v, np.asarray(scale, np.float32)
        self.pool = pool_of(k, v, self.scale, self.code)

    def run(self, o=None, stream=None, ws=None, pool=None):
        o = torch.full_like(self.q, float("nan")) if o is None else o
        call = B.pic_attn8_decode if self.decode else B.pic_attn8_prefill
        call(self.cfg, self.host, self.block_tables, self.positions, self.q, o, pool or self.pool, workspace=self.ws if ws is None else ws,
             stream=stream)
        return o

    def check(self, got, what=""):
        """Every output within what its roundings can do.

        A score q.k is off by at most |q||k| scale times the relative errors of q and k as vectors, and by D 2^-24 of
        the same for its sum.  float32: angles, and one rounding each.  bf16 with rotation: q rounds once to 11
        bits.  A pair (x, y) of codes, of size n, is turned in 11-bit arithmetic as x c - (y s), y c + (x s): c and s round,
        the second product rounds, the result rounds: with u = 2^-11 the errors are at most u (|x c| + 2 |y s|) and u (|y c|
        + 2 |x s|), a vector of at most u n (|c| + 2 |s|) <= sqrt(5) u n, and u n for the results; what rounds below
        2^-14 (a cos or sin, 2^-25 times 634 at most) less than 2^-15 steps of the code, which is at least 2^-9: the term
        `low` beside n.  Row tiles of 16 and 32 turn a block's keys by their place in it and the rounded queries back by the
        block's position, in the same arithmetic: (sqrt(5) + 1) u for them too, and what rounds below 2^-14 (queries
        are within 1 there) less than 2^-25 four times.  Without rotation q and codes are exact.
        A relative error e of every probability moves an output by at most e / (1 - e) sum p |v - o|.  Probabilities
        are rounded to 8 bits at least, outputs to their type.  Both sums over n keys are in 32 bits: n additions, each
        rounding at most sum p |v| <= |o| + sum p |v - o| to 24 bits; exp2 and joins a few roundings more."""
        rot = self.rot or self.d
        k_all, v_all = (K8.decode(c, self.code) * self.scale[..., i].astype(np.float64)[:, :, None, None]
                        for i, c in enumerate((self.k_codes, self.v_codes)))
        q, got = f64(self.q), f64(got)
        row, off, worst, err, norm = 0, 0, 0.0, 0.0, 0.0
        scale = self.softmax or self.d ** -0.5
        bf = self.dtype == torch.bfloat16
        for r, (ctx, n, w) in enumerate(self.lens):
            L = ctx + n
            j = np.arange(w, L)
            k, v = (p[self.table[r, j // 16], :, j % 16] for p in (k_all, v_all))
            ks = self.scale[self.table[r, j // 16], :, 0].astype(np.float64)
            qq = q[row:row + n]
            if not self.prerotated:
                k = T.rotate(k, self.pos[off + w:off + L], rot, self.theta, self.style, self.inv_freq)
                qq = T.rotate(qq, self.pos[off + ctx:off + L], rot, self.theta, self.style, self.inv_freq)
            see = j <= np.arange(ctx, L)[:, None]
            o, spread = T.attention(qq, k, v, see, scale)
            low = 0.0
            if self.prerotated:
                eq = ek = 0.0 if bf else 2.0 ** -24   # (float32: code times scale, q times the softmax scale)
            elif bf:
                eq = 2.0 ** -11 + self.d ** 0.5 * 2.0 ** -24 + ANGLE
                if tile_of(self)[0] <= 32:
                    eq += (5 ** 0.5 + 1) * 2.0 ** -11 + self.d ** 0.5 * 2.0 ** -22 + ANGLE
                ek = (5 ** 0.5 + 1) * 2.0 ** -11 + ANGLE_ADVANCED
                low = self.d ** 0.5 * 2.0 ** -15 * float(ks.max())
            else:
                eq = ek = 4 * 2.0 ** -24 + ANGLE
            nq, nk = np.linalg.norm(qq, axis=-1).max(), np.linalg.norm(k, axis=-1).max() + low
            ds = nq * nk * scale * (eq + ek + eq * ek + self.d * 2.0 ** -24) + nq * low * scale
            e = np.expm1(ds) + (2.0 ** -8 if bf else 0.0) + 2.0 ** -20
            assert e < 0.5, "inputs too large for the bound"
            sums = (2 * len(j) + 16) * 2.0 ** -24
            tol = e / (1 - e) * spread + (HALF_STEP[self.dtype] * 1.01 + sums) * (np.abs(o) + spread) + 1e-30
            d = np.abs(got[row:row + n] - o)
            assert np.isfinite(got[row:row + n]).all(), (what, r)
            worst = max(worst, float((d / tol).max()))
            assert (d <= tol).all(), (what, r, float((d / tol).max()), float(d.max()))
            err, norm = err + float((d * d).sum()), norm + float((o * o).sum())
            row, off = row + n, off + L
        rel = (err / norm) ** 0.5
        say(f"  {what}: at most {worst:.2f} of the bound, {rel:.2e} of the norm")
        return rel


LENGTHS = [0, 1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 700]


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 4, 64), (16, 1, 128), (7, 1, 64)])
@pytest.mark.parametrize("ctx", LENGTHS)
def test_prefill_lengths(hq, hkv, d, dtype, code, ctx):
    g = hq // hkv
    # rows that fill, overfill and underfill every size of row tile
    nodes = sorted({1, 2, max(1, 16 // g), 16 // g + 1, max(1, 32 // g), 32 // g + 1, max(1, 128 // g), 128 // g + 1})
    for n in nodes:
        b = Batch([(ctx, n)], hq, hkv, d, dtype, code, style=n % 2, seed=ctx * 131 + n)
        b.check(b.run(), f"ctx {ctx} new {n}")


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (4, 4, 64), (16, 1, 128), (28, 4, 128), (40, 1, 64), (17, 1, 128)])
def test_decode_lengths(hq, hkv, d, dtype, code):
    for ctx in LENGTHS + [3000]:
        b = Batch([(ctx, 1)], hq, hkv, d, dtype, code, style=ctx % 2, seed=ctx + 7, decode=True)
        b.check(b.run(), f"ctx {ctx}")


@pytest.mark.parametrize("decode", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("style,rot,prerotated", [(0, 0, 0), (1, 0, 0), (0, 32, 0), (0, 16, 0), (1, 34, 0), (1, 2, 0), (0, 0, 1), (0, 64, 1)])
@pytest.mark.parametrize("d,nodes", [(128, 5), (128, 40), (64, 9), (64, 70)])
def test_rotations(dtype, style, rot, prerotated, d, nodes, decode):
    n = (1, 1, 1) if decode else (nodes, 3, 1)
    b = Batch([(150, n[0]), (290, n[1]), (16, n[2])], 8, 2, d, dtype, K8.E4M3 if nodes % 2 else K8.INT8, style, rot, prerotated, seed=nodes,
              decode=decode)
    b.check(b.run(), "rotation")


@pytest.mark.parametrize("decode", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("code", CODES)
def test_ragged_batches_with_windows(dtype, code, decode):
    rng = np.random.default_rng(9)
    for many in (3, 20, 70):   # more spans than the short and the long arguments hold
        lens = []
        for _ in range(many):
            ctx, n = int(rng.integers(0, 400)), 1 if decode else int(rng.integers(1, 90))
            lens.append((ctx, n, int(rng.integers(0, ctx + 1)) if rng.random() < 0.5 else 0))
        b = Batch(lens, 12, 4, 64, dtype, code, style=1, seed=many, decode=decode)
        b.check(b.run(), f"{many} requests")


@pytest.mark.parametrize("decode", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
def test_positions_anywhere(dtype, decode):
    n = 1 if decode else 40
    far = lambda rng, m: np.arange(m) + 2**31 - 1 - m   # noqa: E731
    for what, positions in (("random", lambda rng, m: rng.integers(-2**31, 2**31, m)), ("far", far), ("negative", lambda rng, m: -np.arange(m)),
                            ("jumps", lambda rng, m: np.arange(m) // 48 * 1000 + np.arange(m)), ("one", lambda rng, m: np.full(m, 5)),
                            ("around", lambda rng, m: np.where(np.arange(m) < 300, 2**31 - 300 + np.arange(m), np.arange(m) - 300 - 2**31))):
        for d, style in ((128, 0), (64, 1)):
            b = Batch([(600, n), (128, n)], 8, 2, d, dtype, K8.INT8, style, seed=3, positions=positions, decode=decode)
            b.check(b.run(), what)


@pytest.mark.parametrize("decode", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("code", CODES)
def test_scales_of_another_program(dtype, code, decode):
    """Scales that are no powers of two, zeros among them, and blocks of very different sizes."""
    n = 1 if decode else 50
    b = Batch([(260, n), (33, n)], 8, 2, 128, dtype, code, seed=4, powers=False, decode=decode)
    b.check(b.run(), "any scale")
    scale = b.scale.copy()
    scale[::3] = 0.0
    b.set_pool(b.k_codes, b.v_codes, scale)
    b.check(b.run(), "zero scales")
    scale = np.exp2(b.rng.integers(-100, -6, scale.shape)).astype(np.float32)
    scale[..., 1] = np.exp2(b.rng.integers(-40, 40, scale.shape[:2]))
    b.set_pool(b.k_codes, b.v_codes, scale)
    b.check(b.run(), "sizes apart")


@pytest.mark.parametrize("decode", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128])
def test_nothing_else_is_read(dtype, d, decode):
    """What lies outside the windows holds NaN, in codes and scales, and rows behind a request's last token too."""
    n = 1 if decode else 45
    lens = [(200, n, 70), (37, n, 0), (96, n, 96), (500, n, 333)]
    b = Batch(lens, 8, 2, d, dtype, K8.E4M3, seed=8, decode=decode)
    want = b.run()
    b.check(want, "clean")
    k, v, scale = b.k_codes.copy(), b.v_codes.copy(), b.scale.copy()
    used = np.zeros((b.nb, 16), bool)
    for r, (ctx, m, w) in enumerate(lens):
        j = np.arange(w, ctx + m)
        used[b.table[r, j // 16], j % 16] = True
    for c in (k, v):
        c.swapaxes(1, 2)[~used] = 0x7f
    scale[~used.any(1)] = np.nan
    got = b.run(pool=pool_of(k, v, scale, b.code))
    assert torch.equal(got, want)


def test_long_context_and_splits():
    for hq, hkv, n, decode in ((8, 1, 1, True), (32, 8, 1, True), (8, 1, 3, False), (16, 2, 40, False)):
        b = Batch([(20000, n)], hq, hkv, 128, torch.bfloat16, K8.INT8, seed=n, decode=decode)
        b.check(b.run(), f"20,000 keys, {n} new")


def test_spread_of_a_large_softmax_scale():
    """Row maxima that move again and again."""
    for decode, n in ((True, 1), (False, 60)):
        b = Batch([(900, n)], 8, 2, 128, torch.float32, K8.INT8, seed=6, softmax=2.0, decode=decode, qscale=0.5)
        b.check(b.run(), "float32")
        b = Batch([(900, n)], 8, 2, 128, torch.bfloat16, K8.INT8, prerotated=1, seed=6, softmax=2.0, decode=decode, qscale=0.5)
        b.check(b.run(), "bf16")


@pytest.mark.parametrize("code", CODES)
def test_precision_of_normal_inputs(code):
    """How far outputs are from 64 bits, by independent roundings.  A rounding to b bits is off by 2^-b / sqrt(3) / 1.39 of a
    value in the mean square (evenly over half a step, and over mantissas).  The result's: r8 = 1.6e-3, with the spread of
    values within a binade at most 1.07 times that.  Probabilities of 8 bits: r8 once more.  Turned keys and queries, in
    11 bits: of a pair's element x c - (y s), with pairs of any angle, c, s, the product and the result give 1/4 + 1/4 + 1/4 +
    1/2 of the pair's square, 1.58 of an element's size; with a query's own rounding a score is off by sqrt(1.58^2 + 1) r11 =
    1.87 r11 of its standard deviation, which is 4 for the largest blocks here: each probability by 7.5 r11 = 0.93 r8, and
    outputs by no more than that.  Row tiles of 16 and 32 turn the queries in 11 bits too: sqrt(1.58^2 + 1.58^2 + 1) =
    2.45 r11, 1.22 r8.  1.05 for what a sample of 10,000 and more outputs may be off by."""
    r8 = 2.0 ** -8 / 3 ** 0.5 / 1.39
    for n, decode in ((1, True), (2, False), (60, False), (200, False)):
        for prerotated in (0, 1):
            b = Batch([(2000, n)], 16, 2, 128, torch.bfloat16, code, prerotated=prerotated, seed=n, decode=decode)
            items = B.pic_attn8_plan_debug(b.cfg, b.host, decode)
            many = (items[:, 3] - items[:, 2]).max() > 32
            bound = 1.05 * r8 * (1.07 ** 2 + (1.0 if many else 0.0) + (0.0 if prerotated else (0.93 if many else 1.22) ** 2)) ** 0.5
            got = b.check(b.run(), f"{n} tokens")
            assert got <= bound, (n, prerotated, got, bound)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128])
def test_spans_as_prefill_has_them(dtype, d):
    """Several query spans of a request, detached, inheriting and dependent ones, windows of their own: what
    pic_attn_prefill gives on a pool of the same numbers."""
    rng = np.random.default_rng(d)
    hq, hkv, code = 8, 2, K8.E4M3
    seq = [500, 61, 333]
    cu = [0, 5, 6, 9]
    start = [0, 100, 160, 300, 420, 0, 0, 128, 200]
    S, P, Q = B.PIC_SSEP, B.PIC_PDEP, B.PIC_QUERY
    flags = [S, S | Q, Q, S, P | Q, S | Q, S | Q, Q, P | Q]
    win = [-1, -1, -1, -1, -1, -1, -1, 60, -1]
    host = B.HostBatch(seq, cu, start, flags, win)
    need = [-(-s // 16) for s in seq]
    nb = sum(need)
    ids = rng.permutation(nb).astype(np.int32)
    table = np.zeros((3, max(need)), np.int32)
    for r, k in enumerate(need):
        table[r, :k], ids = ids[:k], ids[k:]
    codes_k, codes_v, scale = random_pool(rng, nb, hkv, d, code)
    pool = pool_of(codes_k, codes_v, scale, code)
    dense = [dev(K8.decode(c, code) * scale[..., i][:, :, None, None]).to(dtype) for i, c in enumerate((codes_k, codes_v))]
    cfg = cfg_of(hq, hkv, d, dtype)
    rows = 60 + 140 + 80 + 61 + 128 + 72 + 133
    q = torch.from_numpy(rng.standard_normal((rows, hq, d)) * 0.5).to(dtype).cuda()
    tables, pos = dev(table), dev(np.concatenate([np.arange(s) + 50 for s in seq]).astype(np.int32))
    o, ref = torch.full_like(q, float("nan")), torch.empty_like(q)
    ws8 = torch.empty(max(1, B.pic_attn8_workspace_size(cfg, host, False)), dtype=torch.uint8, device="cuda")
    ws = torch.empty(max(1, B.pic_workspace_size(cfg, host, False)), dtype=torch.uint8, device="cuda")
    B.pic_attn8_prefill(cfg, host, tables, pos, q, o, pool, workspace=ws8)
    B.pic_attn_prefill(cfg, host, tables, pos, q, ref, *dense, workspace=ws)
    # the pool's numbers are exact in either type; the prefill rounds turned keys and queries to 8 bits each where this one has 11,
    # and probabilities to 8 bits: a few times 2^-8 of the outputs' norm (float32: of 2^-24, times its sums' lengths)
    err = float((o.double() - ref.double()).norm() / ref.double().norm())
    say(f"  spans: {err:.2e}")
    assert err < (1.5e-2 if dtype == torch.bfloat16 else 5e-6)


class Step:
    """Decode steps of a few requests: a projection's rows are normalised, stored in 8 bits and attended."""

    def __init__(self, code, dtype, prerotated, seed=0):
        self.code, self.dtype = code, dtype
        self.hq, self.hkv, self.d, self.r, self.most = 8, 2, 64, 5, 90
        self.cfg = cfg_of(self.hq, self.hkv, self.d, dtype, prerotated=prerotated)
        self.rng = np.random.default_rng(seed)
        self.nb = self.r * 6
        self.table = self.rng.permutation(self.nb).reshape(self.r, 6).astype(np.int32)
        shape = (self.nb, self.hkv, 16, self.d)
        self.pool = B.Kv8Pool(torch.full(shape, 0x7f, dtype=torch.uint8, device="cuda"), torch.full(shape, 0x7f, dtype=torch.uint8, device="cuda"),
                              torch.full((self.nb, self.hkv, 2), float("nan"), device="cuda"), code)
        self.wq, self.wk = (1 + 0.1 * torch.randn(self.d, generator=torch.Generator().manual_seed(i)) for i in (1, 2))
        self.wq, self.wk = self.wq.to(dtype).cuda(), self.wk.to(dtype).cuda()
        self.tables = dev(self.table)
        self.keys = [[] for _ in range(self.r)]     # as normalised, float64
        self.values = [[] for _ in range(self.r)]

    def rows(self, n):
        return torch.from_numpy(self.rng.standard_normal((n, self.hq + 2 * self.hkv, self.d))).to(self.dtype).cuda()

    def put(self, qkv, at, stream=None):
        """Rows of (request, index): norms in place, the store."""
        q, k, v = qkv[:, :self.hq], qkv[:, self.hq:self.hq + self.hkv], qkv[:, self.hq + self.hkv:]
        pos = dev(np.array([i for _, i in at], np.int32))
        slots = dev(np.array([self.table[r, i // 16] * 16 + i % 16 for r, i in at], np.int32))
        B.pic_qk_norm(self.cfg, q, k, self.wq, self.wk, 1e-6, pos, stream=stream)
        B.pic_kv8_write(self.cfg, self.pool, k, v, slots, stream=stream)
        return q


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("prerotated", [0, 1])
def test_prefill_then_steps_of_all(code, dtype, prerotated):
    """Prompts of odd lengths, then tokens one by one into pools that held NaN: attention over the pool is attention over what
    pic_kv8_read returns from it, and that is within the codes' error of the rows stored."""
    s = Step(code, dtype, prerotated)
    lens = [1, 15, 16, 33, 60]
    qkv = s.rows(sum(lens))
    stored = [[], []]
    at = [(r, i) for r, n in enumerate(lens) for i in range(n)]
    q = s.put(qkv, at)
    stored = {x: qkv[j, s.hq:].double().cpu() for j, x in enumerate(at)}
    for step in range(20):
        host = B.HostBatch([n + step for n in lens], range(s.r + 1), [0] * s.r, [B.PIC_PDEP | (B.PIC_QUERY if step == 0 else 0)] * s.r)
        decode = step > 0
        if decode:
            new = s.rows(s.r)
            at = [(r, n + step - 1) for r, n in enumerate(lens)]
            q = s.put(new, at)
            stored.update({x: new[j, s.hq:].double().cpu() for j, x in enumerate(at)})
        q = q.contiguous()
        total = [n + step for n in lens]
        positions = dev(np.concatenate([np.arange(n) for n in total]).astype(np.int32))
        o = torch.full_like(q, float("nan"))
        ws = torch.empty(max(1, B.pic_attn8_workspace_size(s.cfg, host, decode)), dtype=torch.uint8, device="cuda")
        (B.pic_attn8_decode if decode else B.pic_attn8_prefill)(s.cfg, host, s.tables, positions, q, o, s.pool, workspace=ws)
        slots = dev(np.array([s.table[r, i // 16] * 16 + i % 16 for r, n in enumerate(total) for i in range(n)], np.int32))
        k, v = (torch.empty(len(slots), s.hkv, s.d, dtype=dtype, device="cuda") for _ in range(2))
        B.pic_kv8_read(s.cfg, s.pool, slots, k, v)
        # half a step of rounding as it is stored, and less than another half over the growths of a block's scale
        scale = s.pool.scale[slots.long() // 16].double().cpu()
        ref = torch.stack([stored[r, i] for r, n in enumerate(total) for i in range(n)])
        for i, (x, want) in enumerate(((k, ref[:, :s.hkv]), (v, ref[:, s.hkv:]))):
            sc = scale[..., i, None]
            unit = sc if code == K8.INT8 else torch.maximum(torch.exp2(torch.floor(torch.log2((want / sc).abs().clamp(min=2.0 ** -6))) - 3), torch.tensor(2.0 ** -9)) * sc
            assert ((x.double().cpu() - want).abs() <= unit).all(), (step, i)
        row, off = 0, 0
        kk, vv, qq = f64(k), f64(v), f64(q)
        for r, n in enumerate(total):
            m = n if not decode else 1
            kr, qr = kk[off:off + n], qq[row:row + m]
            if not prerotated:
                kr = T.rotate(kr, np.arange(n), s.d, 1e4, 0)
                qr = T.rotate(qr, np.arange(n - m, n), s.d, 1e4, 0)
            want, spread = T.attention(qr, kr, vv[off:off + n], np.arange(n) <= np.arange(n - m, n)[:, None], s.d ** -0.5)
            err = np.abs(f64(o[row:row + m]) - want)
            bound = (2.0 ** -6 if dtype == torch.bfloat16 else 2.0 ** -15) * (np.abs(want) + spread) + 1e-30
            assert (err <= bound).all(), (step, r, float((err / bound).max()))
            row, off = row + m, off + n


@pytest.mark.parametrize("code", CODES)
def test_step_captured_and_replayed(code):
    """A captured norm, store and attention give, on every replay, what eager ones give on the same inputs; two graphs share a
    workspace."""
    dtype = torch.bfloat16
    s, e = Step(code, dtype, 0, seed=3), Step(code, dtype, 0, seed=3)
    lens = [40, 3, 17, 64, 80]
    first = s.rows(sum(lens))
    at = [(r, i) for r, n in enumerate(lens) for i in range(n)]
    for x in (s, e):
        x.put(first.clone(), at)
    total = [n + 1 for n in lens]
    host = B.HostBatch(total, range(6), [0] * 5, [B.PIC_PDEP] * 5)
    new = s.rows(5)
    at = [(r, n) for r, n in enumerate(lens)]
    pos = dev(np.array([i for _, i in at], np.int32))
    slots = dev(np.array([s.table[r, i // 16] * 16 + i % 16 for r, i in at], np.int32))
    positions = dev(np.concatenate([np.arange(n) for n in total]).astype(np.int32))
    ws = torch.empty(max(1, B.pic_attn8_workspace_size(s.cfg, host, True)) + 4096, dtype=torch.uint8, device="cuda")
    buf, qo = torch.empty_like(new), torch.empty(5, s.hq, s.d, dtype=dtype, device="cuda")

    def run(x, buf, qo, o, stream=None):
        q, k, v = buf[:, :x.hq], buf[:, x.hq:x.hq + x.hkv], buf[:, x.hq + x.hkv:]
        B.pic_qk_norm(x.cfg, q, k, x.wq, x.wk, 1e-6, pos, q_out=qo, stream=stream)
        B.pic_kv8_write(x.cfg, x.pool, k, v, slots, stream=stream)
        B.pic_attn8_decode(x.cfg, host, x.tables, positions, qo, o, x.pool, workspace=ws, stream=stream)

    other = Batch([(700, 30), (20, 9)], 8, 2, 64, seed=5)
    ref = other.run()
    other_ws = torch.empty(max(ws.numel(), other.ws.numel()), dtype=torch.uint8, device="cuda")
    ws = other_ws
    o, eo, oo = torch.empty_like(qo), torch.empty_like(qo), torch.empty_like(ref)
    torch.cuda.synchronize()
    graph, second = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(s, buf, qo, o, stream=torch.cuda.current_stream())
    with torch.cuda.graph(second):
        other.run(o=oo, ws=other_ws, stream=torch.cuda.current_stream())
    for i in range(4):
        rows = new * (1 + i)   # (scales grow: a replay works on the pool as it is)
        buf.copy_(rows)
        ebuf = rows.clone()
        o.zero_(), oo.zero_()
        graph.replay()
        second.replay()
        run(e, ebuf, torch.empty_like(qo), eo)
        torch.cuda.synchronize()
        assert torch.equal(o, eo) and torch.equal(oo, ref)
        assert torch.equal(s.pool.k, e.pool.k) and torch.equal(s.pool.v, e.pool.v) and torch.equal(s.pool.scale.view(torch.int32), e.pool.scale.view(torch.int32))


def test_calls_on_two_streams_and_repeats_agree():
    """Calls that overlap on two streams, each with its own workspace, and repeats: bit for bit."""
    a, b = Batch([(3000, 1)] * 7, 8, 2, 128, seed=1, decode=True), Batch([(2000, 9), (700, 70)], 8, 2, 128, seed=2)
    ra, rb = a.run(), b.run()
    torch.cuda.synchronize()
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    outs = [(torch.empty_like(ra), torch.empty_like(rb)) for _ in range(5)]
    torch.cuda.synchronize()
    for oa, ob in outs:
        a.run(o=oa, stream=s)
        b.run(o=ob, stream=t)
    torch.cuda.synchronize()
    for oa, ob in outs:
        assert torch.equal(oa, ra) and torch.equal(ob, rb)


def test_many_requests_captured_and_replayed():
    """More spans than the kernel arguments hold: the captured call uploads its plan on every replay."""
    rng = np.random.default_rng(11)
    for decode in (False, True):
        b = Batch([(int(rng.integers(1, 300)), 1 if decode else int(rng.integers(1, 20))) for _ in range(80)], 8, 2, 64, seed=12, decode=decode)
        ref = b.run()
        torch.cuda.synchronize()
        o = torch.zeros_like(ref)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            b.run(o=o, stream=torch.cuda.current_stream())
        for _ in range(3):
            o.zero_()
            b.ws.fill_(255)
            graph.replay()
            junk = torch.randn(1 << 16, device="cuda")
            torch.cuda.synchronize()
            assert torch.equal(o, ref) and junk.numel()


def test_float32_in_a_small_workspace():
    """Without room for partial results float32 keys stay unsplit: the same sums in another order."""
    for lens, decode in (([(700, 5)], False), ([(900, 30), (64, 3)], False), ([(3000, 1)], True)):
        b = Batch(lens, 8, 2, 64, torch.float32, K8.INT8, seed=7, decode=decode)
        for ws in (torch.empty(0, dtype=torch.uint8, device="cuda"), torch.empty(256, dtype=torch.uint8, device="cuda")):
            assert b.ws.numel() > ws.numel()
            b.check(b.run(ws=ws), "small workspace")


def test_pool_past_4_gib():
    """The same blocks at the far end of a pool of 4.3 GiB of keys (and of values): bit for bit."""
    for dtype, n, decode in ((torch.bfloat16, 1, True), (torch.bfloat16, 40, False), (torch.float32, 3, False)):
        b = Batch([(130, n), (77, n)], 8, 8, 128, dtype, K8.INT8, seed=n, decode=decode)
        want = b.run()
        per = 8 * 16 * 128
        nb = ((43 << 30) // 10) // per
        k, v = (torch.empty(nb, 8, 16, 128, dtype=torch.uint8, device="cuda") for _ in range(2))
        scale = torch.empty(nb, 8, 2, device="cuda")
        far = nb - b.nb
        k[far:], v[far:], scale[far:] = b.pool.k, b.pool.v, b.pool.scale
        pool = B.Kv8Pool(k, v, scale, K8.INT8)
        tables = b.block_tables
        b.block_tables = torch.where(tables < b.nb, tables + far, tables)
        assert torch.equal(b.run(pool=pool), want)
        # rows stored and read there
        slots = (torch.arange(40, device="cuda", dtype=torch.int32) + far * 16).contiguous()
        rows = torch.randn(40, 8, 128, device="cuda").to(dtype)
        near = B.Kv8Pool(torch.zeros_like(b.pool.k), torch.zeros_like(b.pool.v), torch.zeros_like(b.pool.scale), K8.INT8)
        B.pic_kv8_write(b.cfg, pool, rows, rows * 2, slots)
        B.pic_kv8_write(b.cfg, near, rows, rows * 2, slots - far * 16)
        assert torch.equal(k[far:far + 3], near.k[:3]) and torch.equal(v[far:far + 3], near.v[:3]) and torch.equal(scale[far:far + 3], near.scale[:3])
        got, ref = ([torch.empty_like(rows), torch.empty_like(rows)] for _ in range(2))
        B.pic_kv8_read(b.cfg, pool, slots, *got)
        B.pic_kv8_read(b.cfg, near, slots - far * 16, *ref)
        assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])
        del k, v, scale, pool


def tile_of(b):
    """Row tile of a batch's plan, and whether its keys are split."""
    items = B.pic_attn8_plan_debug(b.cfg, b.host, b.decode)
    rows = (items[:, 3] - items[:, 2]).max()
    return min(t for t in (16, 32, 128, 256) if rows <= t), bool((items[:, 7] >= 0).any())


# what the plans of these batches are is asserted, so that every kernel, split and not, and every layout of heads over the
# dies (8 KV heads and multiples, and others) is among them
LARGE = [(32, 8, 128, [(1500, 100), (750, 91)], 128, True), (32, 8, 128, [(30, 600)], 128, False),
         (32, 8, 128, [(900, 70)] + [(450, 61)] * 7, 256, True), (32, 8, 128, [(300, 60)] + [(150, 51)] * 23, 256, False),
         (10, 5, 128, [(30, 600)], 128, True), (10, 5, 128, [(300, 60)] + [(150, 51)] * 23, 128, False),
         (12, 12, 64, [(2500, 130), (1250, 121), (1250, 121)], 256, True), (12, 12, 64, [(300, 60)] + [(150, 51)] * 23, 128, False),
         (64, 8, 128, [(30, 600)], 256, False), (6, 1, 64, [(700, 300), (350, 291)], 128, True), (6, 1, 64, [(0, 1000)], 256, True),
         (8, 2, 64, [(0, 1000)], 128, True)]


@pytest.mark.parametrize("case", range(len(LARGE)))
@pytest.mark.parametrize("code", CODES)
def test_large_row_tiles(case, code):
    hq, hkv, d, lens, tile, split = LARGE[case]
    b = Batch(lens, hq, hkv, d, torch.bfloat16, code, seed=case)
    assert tile_of(b) == (tile, split)
    b.check(b.run(), f"case {case}")


@pytest.mark.parametrize("style,rot,prerotated", [(1, 0, 0), (0, 32, 0), (0, 16, 0), (1, 34, 0), (1, 2, 0), (0, 0, 1)])
@pytest.mark.parametrize("case", [0, 1, 2, 3, 6, 7, 8])
def test_large_row_tiles_and_rotations(case, style, rot, prerotated):
    hq, hkv, d, lens, tile, split = LARGE[case]
    b = Batch(lens[:6], hq, hkv, d, torch.bfloat16, CODES[case % 2], style, rot, prerotated, seed=case)
    if len(lens) < 7:
        assert tile_of(b) == (tile, split)
    b.check(b.run(), f"case {case}")


@pytest.mark.parametrize("what", ["positions", "jumps", "scales", "zeros", "sizes", "windows", "outside"])
@pytest.mark.parametrize("case", [0, 1, 2, 5, 6, 11])
def test_large_row_tiles_and_values(case, what):
    hq, hkv, d, lens, tile, split = LARGE[case]
    rng = np.random.default_rng(case)
    kw = {"positions": dict(positions=lambda rng, m: rng.integers(-2**31, 2**31, m)),
          "jumps": dict(positions=lambda rng, m: np.arange(m) // 40 * 999 + np.arange(m)), "scales": dict(powers=False)}.get(what, {})
    if what == "windows":
        lens = [(ctx, n, int(rng.integers(0, ctx // 8 + 1))) for ctx, n in lens]
    b = Batch(lens, hq, hkv, d, torch.bfloat16, CODES[case % 2], seed=case, **kw)
    if what != "windows":
        assert tile_of(b) == (tile, split)
    assert tile_of(b)[0] >= 128
    scale = b.scale.copy()
    if what == "zeros":
        scale[::3] = 0.0
    if what == "sizes":
        scale = np.exp2(b.rng.integers(-100, -6, scale.shape)).astype(np.float32)
        scale[..., 1] = np.exp2(b.rng.integers(-40, 40, scale.shape[:2]))
    if what in ("zeros", "sizes"):
        b.set_pool(b.k_codes, b.v_codes, scale)
    o = b.run()
    b.check(o, what)
    if what == "outside":
        used = np.zeros((b.nb, 16), bool)
        for r, (ctx, m, w) in enumerate(b.lens):
            j = np.arange(w, ctx + m)
            used[b.table[r, j // 16], j % 16] = True
        k, v = b.k_codes.copy(), b.v_codes.copy()
        for c in (k, v):
            c.swapaxes(1, 2)[~used] = 0x7f
        scale[~used.any(1)] = np.nan
        assert torch.equal(b.run(pool=pool_of(k, v, scale, b.code)), o)


# calls of which many row tiles share the keys: these are turned once, into a copy in the workspace
COPIED = [(64, 1, 128, [(800, 400)], 128, False), (64, 1, 128, [(790, 230, 37), (33, 300, 16), (0, 250)], 128, False),
          (16, 2, 64, [(1500, 900)], 128, True), (32, 1, 128, [(300, 160)] * 12, 256, False),
          (64, 2, 64, [(700, 500, 5), (1201, 499, 37)], 256, False), (24, 12, 128, [(300, 900)], 128, False),
          (32, 8, 128, [(600, 900)], 256, True), (64, 2, 128, [(2500, 120)], 128, True)]


def copied_bytes(b):
    """Workspace that a batch's turned keys take."""
    turned = cfg_of(b.hq, b.hkv, b.d, b.dtype, prerotated=1)
    return B.pic_attn8_workspace_size(b.cfg, b.host, b.decode) - B.pic_attn8_workspace_size(turned, b.host, b.decode)


@pytest.mark.parametrize("case,style,rot", [(i, 0, 0) for i in range(len(COPIED))] +
                         [(i, *r) for i in (1, 2) for r in ((1, 0), (0, 32), (1, 34))])
def test_keys_turned_once(case, style, rot):
    """... with the copy, and in a workspace without room for it."""
    hq, hkv, d, lens, tile, split = COPIED[case]
    b = Batch(lens, hq, hkv, d, torch.bfloat16, CODES[(case + style) % 2], style, rot, seed=case)
    extra = copied_bytes(b)
    assert extra > 0 and tile_of(b) == (tile, split)
    got = b.run(ws=torch.full((b.ws.numel(),), 0xff, dtype=torch.uint8, device="cuda"))
    b.check(got, f"case {case}")
    small = b.run(ws=torch.zeros(max(1, b.ws.numel() - extra), dtype=torch.uint8, device="cuda"))
    if case in (1, 2, 7):
        b.check(small, f"case {case}, turned in the kernel")


@pytest.mark.parametrize("what", ["random", "jumps", "outside", "scales"])
@pytest.mark.parametrize("case", [1, 2])
def test_keys_turned_once_and_values(case, what):
    hq, hkv, d, lens, tile, split = COPIED[case]
    kw = {"random": dict(positions=lambda rng, m: rng.integers(-2**31, 2**31, m)),
          "jumps": dict(positions=lambda rng, m: np.arange(m) // 40 * 999 + np.arange(m)), "scales": dict(powers=False)}.get(what, {})
    b = Batch(lens, hq, hkv, d, torch.bfloat16, CODES[case % 2], seed=case, **kw)
    assert copied_bytes(b) > 0
    got = b.run()
    b.check(got, what)
    if what == "outside":
        k, v, scale = b.k_codes.copy(), b.v_codes.copy(), b.scale.copy()
        used = np.zeros((b.nb, 16), bool)
        for r, (ctx, m, w) in enumerate(b.lens):
            j = np.arange(w, ctx + m)
            used[b.table[r, j // 16], j % 16] = True
        for c in (k, v):
            c.swapaxes(1, 2)[~used] = 0x7f
        scale[~used.any(1)] = np.nan
        assert torch.equal(b.run(pool=pool_of(k, v, scale, b.code)), got)


def test_keys_turned_once_for_many_spans():
    """More query spans than the kernel arguments hold, of few requests: plan and copy in the workspace."""
    lens = [(600, 350, 0), (500, 350, 21)]
    b = Batch(lens, 64, 1, 128, torch.bfloat16, K8.INT8, seed=2)
    n, spans = 10, 35
    start, flags, win, cu = [], [], [], [0]
    for ctx, m, w in lens:
        start += [0, *range(ctx, ctx + m, n)]
        flags += [B.PIC_PDEP] + [B.PIC_PDEP | B.PIC_QUERY] * spans
        win += [-1] + [w] * spans
        cu.append(len(start))
    b.host = B.HostBatch([ctx + m for ctx, m, _ in lens], cu, start, flags, win)
    assert copied_bytes(b) > 0
    b.ws = torch.full((B.pic_attn8_workspace_size(b.cfg, b.host, False),), 0xff, dtype=torch.uint8, device="cuda")
    b.check(b.run(), "70 spans")


def test_keys_turned_once_captured_and_replayed():
    """The copy is made anew on every replay, from the pool as it is then; calls on a side stream between them."""
    hq, hkv, d, lens, _, _ = COPIED[1]
    b = Batch(lens, hq, hkv, d, torch.bfloat16, K8.INT8, seed=1)
    assert copied_bytes(b) > 0
    o = torch.zeros_like(b.q)
    b.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.run(o, stream=torch.cuda.current_stream())
    for i in range(3):
        b.pool.k.copy_(b.pool.k.roll(1, 0))
        b.pool.scale.copy_(b.pool.scale.roll(1, 0))
        o.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = o.clone()
        assert torch.equal(b.run(ws=torch.zeros_like(b.ws)), got), i
