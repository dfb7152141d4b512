"""The cache held in 8 bits without a GPU: arguments are refused before any HIP call, plans cover every
(row, key) pair once, and the plain model of the codes."""
import ctypes

import numpy as np
import pytest

P = pytest.importorskip("paper_2606_13126_amd")
from paper_2606_13126_amd import _binding as B  # noqa: E402
from tests import kv8_util as K8  # noqa: E402

OK = 4096   # an address that passes the alignment checks and is never used


def status(name, *args):
    rc = getattr(B.lib(), name)(*[ctypes.byref(a) if isinstance(a, ctypes.Structure) else a for a in args])
    return rc, B.lib().pic_last_error().decode()


def batch(lens, window=None, decode=False):
    """One request per (cached, new tokens); 0 new: no query span."""
    seq, cu, start, flags, win = [], [0], [], [], []
    for ctx, n in lens:
        if ctx:
            start.append(0), flags.append(B.PIC_PDEP), win.append(-1)
        if n:
            start.append(ctx), flags.append(B.PIC_PDEP | B.PIC_QUERY), win.append(-1 if window is None else min(window, ctx))
        seq.append(ctx + n)
        cu.append(len(start))
    return B.HostBatch(seq, cu, start, flags, win)


def pool(k=OK, v=OK, scale=OK, num_blocks=64, code=B.PIC_KV8_E4M3):
    return B.pic_kv8_pool(k, v, scale, num_blocks, code)


# ------------------------------------------------------------------------------------
# refusals
# ------------------------------------------------------------------------------------

NORM = dict(q=1 << 20, q_stride=256, q_out=1 << 22, q_out_stride=256, k=1 << 24, k_stride=64, k_out=1 << 25, k_out_stride=64, q_weight=OK,
            k_weight=OK, eps=1e-6, positions=OK, n=3)


def norm_call(cfg, **kw):
    return status("pic_qk_norm", cfg, *{**NORM, **kw}.values(), None)


@pytest.mark.parametrize("kw,what", [
    (dict(n=-1), ">= 0"), (dict(n=1 << 24), "2^24"), (dict(eps=0.0), "eps"), (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"),
    (dict(eps=float("inf")), "eps"), (dict(eps=1e-39), "eps"), (dict(q_out=None), "both"), (dict(q=None), "both"), (dict(k=None), "both"), (dict(k_out=None), "both"),
    (dict(q=None, q_out=None, k=None, k_out=None), "neither"), (dict(positions=None), "positions"), (dict(q_stride=248), "stride"),
    (dict(k_stride=56), "stride"), (dict(k_out_stride=-64), "stride"), (dict(q_out_stride=1 << 62), "stride"), (dict(q_stride=260), "aligned"),
    (dict(k_out_stride=68), "aligned"), (dict(q=OK + 8), "aligned"), (dict(k_out=OK + 8), "aligned"), (dict(q_weight=OK + 8), "aligned"),
    (dict(k_weight=OK + 4), "aligned"), (dict(positions=OK + 2), "aligned"),
    (dict(q_out=(1 << 20) + 512), "overlaps"), (dict(q_out=1 << 20, q_out_stride=512), "overlaps"), (dict(k_out=1 << 20), "overlaps"),
    (dict(q_out=1 << 24), "overlaps"), (dict(k_out=1 << 22), "overlaps"),
    # slices of one fused output [384]: queries at 0, keys at 256; an output that reaches into the other's slice
    (dict(q=1 << 20, q_stride=384, q_out=1 << 20, q_out_stride=384, k=(1 << 20) + 512, k_stride=384, k_out=(1 << 20) + 496, k_out_stride=384),
     "overlaps"),
])
def test_qk_norm_refuses(kw, what):
    rc, msg = norm_call(B.make_config(4, 1, 64, k_prerotated=1), **kw)
    assert rc == B.PIC_EINVAL and what in msg, (rc, msg)


WRITE = dict(k=1 << 20, k_stride=64, v=1 << 21, v_stride=64, slots=OK, n=3)


@pytest.mark.parametrize("kw,pl,what", [
    (dict(n=-1), {}, ">= 0"), (dict(n=1 << 24), {}, "2^24"), (dict(k=None), {}, "NULL"), (dict(v=None), {}, "NULL"),
    (dict(slots=None), {}, "NULL"), (dict(slots=OK + 2), {}, "aligned"), (dict(k_stride=56), {}, "stride"), (dict(v_stride=1 << 62), {}, "stride"),
    (dict(k_stride=68), {}, "aligned"), (dict(v=OK + 8), {}, "aligned"), ({}, dict(k=None), "NULL"), ({}, dict(scale=None), "NULL"),
    ({}, dict(num_blocks=0), "empty"), ({}, dict(num_blocks=-1), ">= 0"), ({}, dict(v=OK + 8), "aligned"), ({}, dict(scale=OK + 4), "aligned"),
    ({}, dict(k=(1 << 20) + 256), "overlap"), ({}, dict(v=(1 << 21) - 65520), "overlap"), ({}, dict(scale=(1 << 21) - 504), "overlap"),
    (dict(k_stride=1 << 20), dict(v=(1 << 20) + (1 << 22)), "overlap"),
])
def test_kv8_write_refuses(kw, pl, what):
    rc, msg = status("pic_kv8_write", B.make_config(4, 1, 64), pool(**pl), *{**WRITE, **kw}.values(), None)
    assert rc == B.PIC_EINVAL and what in msg, (rc, msg)


@pytest.mark.parametrize("slots,n,k_out,v_out,pl,what", [
    (OK, -1, 1 << 20, 1 << 21, {}, ">= 0"), (OK, 1 << 24, 1 << 20, 1 << 21, {}, "2^24"), (None, 3, 1 << 20, 1 << 21, {}, "NULL"),
    (OK, 3, None, 1 << 21, {}, "NULL"), (OK, 3, 1 << 20, None, {}, "NULL"), (OK + 1, 3, 1 << 20, 1 << 21, {}, "aligned"),
    (OK, 3, (1 << 20) + 8, 1 << 21, {}, "aligned"), (OK, 3, 1 << 20, (1 << 20) + 368, {}, "overlap"), (OK, 3, 1 << 28, 1 << 21, dict(k=1 << 28), "pool"),
    (OK, 3, 1 << 21, (1 << 28) + 16, dict(scale=1 << 28), "pool"), (OK, 3, 1 << 20, 1 << 21, dict(num_blocks=0), "empty"),
])
def test_kv8_read_refuses(slots, n, k_out, v_out, pl, what):
    rc, msg = status("pic_kv8_read", B.make_config(4, 1, 64), pool(**pl), slots, n, k_out, v_out, None)
    assert rc == B.PIC_EINVAL and what in msg, (rc, msg)


@pytest.mark.parametrize("call", ["pic_attn8_prefill", "pic_attn8_decode"])
@pytest.mark.parametrize("dtype", [B.PIC_BF16, B.PIC_F32])
def test_attention_refuses(call, dtype):
    cfg, hb = B.make_config(8, 1, 64, dtype=dtype), batch([(900, 70)])

    def go(hb=hb, max_blocks=64, q=OK, o=OK, ws=OK, ws_bytes=1 << 30, pl={}, tables=OK, positions=OK, cfg=cfg):
        return status(call, cfg, hb.c, B.pic_batch_dev(tables, max_blocks, positions), q, o, pool(**pl), ws, ws_bytes, None)

    for kw, what in ((dict(q=None), "q and o"), (dict(o=None), "q and o"), (dict(max_blocks=60), "max_blocks"), (dict(o=OK + 8), "aligned"),
                     (dict(tables=None), "NULL"), (dict(positions=None), "NULL"), (dict(positions=OK + 1), "aligned"),
                     (dict(ws=OK + 8), "aligned"), (dict(pl=dict(k=None)), "NULL"), (dict(pl=dict(scale=None)), "NULL"),
                     (dict(pl=dict(scale=OK + 4)), "aligned"), (dict(pl=dict(num_blocks=0)), "empty"), (dict(pl=dict(num_blocks=-3)), ">= 0"),
                     (dict(hb=B.HostBatch([0], [0, 1], [0], [B.PIC_PDEP])), "seq_lens")):
        rc, msg = go(**kw)
        assert rc == B.PIC_EINVAL and what in msg, (kw, rc, msg)
    rc, msg = go(pl=dict(code=2))
    assert rc == B.PIC_EUNSUPPORTED and "code" in msg
    rc, msg = go(cfg=B.make_config(8, 1, 96, dtype=dtype))
    assert rc == B.PIC_EUNSUPPORTED
    need = B.pic_attn8_workspace_size(cfg, hb, call.endswith("decode"))
    assert need > 0
    if dtype == B.PIC_BF16:
        assert go(ws_bytes=need - 1)[0] == B.PIC_EWORKSPACE
        assert go(ws=None, ws_bytes=0)[0] == B.PIC_EWORKSPACE


def test_null_structures():
    cfg, hb, dv = B.make_config(4, 1, 64), batch([(5, 1)]), B.pic_batch_dev(OK, 4, OK)
    for name, args in (("pic_kv8_write", (cfg, None, OK, 64, OK, 64, OK, 3)), ("pic_kv8_read", (cfg, None, OK, 3, OK, OK)),
                       ("pic_attn8_prefill", (cfg, hb.c, dv, OK, OK, None, None, 0)), ("pic_attn8_decode", (cfg, None, dv, OK, OK, pool(), None, 0)),
                       ("pic_attn8_decode", (None, hb.c, dv, OK, OK, pool(), None, 0)), ("pic_qk_norm", (None, *NORM.values()))):
        rc, msg = status(name, *args, None)
        assert rc == B.PIC_EINVAL and "NULL" in msg, (name, rc, msg)
    assert B.lib().pic_attn8_workspace_size(ctypes.byref(cfg), ctypes.byref(hb.c), 0, None) == B.PIC_EINVAL


def test_nothing_to_do_is_no_error():
    cfg, none = B.make_config(4, 1, 64), B.pic_kv8_pool(None, None, None, 0, 0)
    assert norm_call(cfg, n=0)[0] == B.PIC_OK
    assert status("pic_kv8_write", cfg, none, None, 0, None, 0, None, 0, None)[0] == B.PIC_OK
    assert status("pic_kv8_read", cfg, none, None, 0, None, None, None)[0] == B.PIC_OK
    assert status("pic_attn8_decode", cfg, B.HostBatch([], [0], [], []).c, B.pic_batch_dev(None, 0, None), None, None, none, None, 0, None)[0] == B.PIC_OK
    hb = batch([(5, 0), (1, 0)])   # no request has a query
    assert status("pic_attn8_prefill", cfg, hb.c, B.pic_batch_dev(OK, 4, OK), None, None, pool(), None, 0, None)[0] == B.PIC_OK
    assert B.pic_attn8_workspace_size(cfg, hb, False) == 0


def test_binding_refuses_pools_and_rows_of_another_shape():
    torch = pytest.importorskip("torch")
    k, s = torch.zeros(3, 2, 16, 64, dtype=torch.uint8), torch.zeros(3, 2, 2)
    B.Kv8Pool(k, k, s, 0)
    for bad in ((k, k[:2], s), (k, k, s[:, :, :1]), (k.float(), k, s), (k, k, s.double()), (k[:, :, :, ::2], k[:, :, :, ::2], s), (k[0], k[0], s)):
        with pytest.raises(ValueError):
            B.Kv8Pool(*bad, 0)
    cfg, ids = B.make_config(4, 1, 64), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):   # two heads in the pool, one in the config
        B.pic_kv8_write(cfg, B.Kv8Pool(k, k, s, 0), torch.zeros(3, 1, 64), torch.zeros(3, 1, 64), ids, stream=0)
    with pytest.raises(ValueError):
        B.pic_qk_norm(cfg, torch.zeros(3, 4, 64), torch.zeros(2, 1, 64), None, None, 1e-6, stream=0)
    with pytest.raises(ValueError):
        B.pic_qk_norm(cfg, torch.zeros(3, 4, 128)[:, :, ::2], None, None, None, 1e-6, stream=0)


# ------------------------------------------------------------------------------------
# plans
# ------------------------------------------------------------------------------------

@pytest.mark.parametrize("decode", [False, True])
@pytest.mark.parametrize("dtype", [B.PIC_BF16, B.PIC_F32])
@pytest.mark.parametrize("hq,hkv,d,lens,window", [
    (32, 8, 128, [(1537, 8)], None), (32, 8, 128, [(0, 1)], None), (8, 2, 64, [(700, 13), (0, 3), (15, 1), (4, 2), (1, 40)], None),
    (64, 8, 128, [(131072, 26)], None), (12, 12, 64, [(100 + 7 * i, 1 + i % 5) for i in range(90)], None),
    (28, 4, 128, [(333, 19), (5000, 64)], 300), (16, 1, 128, [(64, 17)], 64), (4, 4, 64, [(2000, 700)], None), (4, 1, 128, [(0, 5000)], None),
])
def test_plan_covers_every_pair_once(dtype, hq, hkv, d, lens, window, decode):
    if decode:
        lens = [(ctx + n - 1, 1) for ctx, n in lens]
    cfg, hb = B.make_config(hq, hkv, d, dtype=dtype), batch(lens, window)
    g = hq // hkv
    seen, slots = {}, set()
    for r, h, lo, hi, kl, kh, tok0, slot in B.pic_attn8_plan_debug(cfg, hb, decode).tolist():
        assert 0 <= lo < hi and kl < kh
        seen.setdefault((r, h), []).append((lo, hi, kl, kh, tok0))
        if slot >= 0:
            assert slot not in slots
            slots.add(slot)
    for r, (ctx, n) in enumerate(lens):
        w = 0 if window is None else min(window, ctx)
        for h in range(hkv):
            rows = {}
            for lo, hi, kl, kh, tok0 in seen[r, h]:
                assert tok0 == ctx and hi <= n * g
                rows.setdefault((lo, hi), []).append((kl, kh))
            at = 0
            for (lo, hi), ranges in sorted(rows.items()):
                assert lo == at
                at = hi
                k = w
                for kl, kh in sorted(ranges):
                    assert kl == k
                    k = kh
                assert k == ctx + (hi - 1) // g + 1   # a row tile runs to its last token
            assert at == n * g


def test_a_batch_near_2_31_keys_is_planned():
    # (no sum of the plan passes 31 bits)
    hb = batch([(2**31 - 2, 1)])
    for dtype in (B.PIC_BF16, B.PIC_F32):
        items = B.pic_attn8_plan_debug(B.make_config(1, 1, 64, dtype=dtype), hb, True)
        assert sorted(items[:, 4])[0] == 0 and sorted(items[:, 5])[-1] == 2**31 - 1
        assert (items[:, 5] > items[:, 4]).all()


# ------------------------------------------------------------------------------------
# the plain model
# ------------------------------------------------------------------------------------

def test_codes_are_the_nearest_numbers():
    rng = np.random.default_rng(0)
    x = rng.standard_normal(5000) * np.exp2(rng.integers(-12, 9, 5000))
    for code in (K8.E4M3, K8.INT8):
        vals = np.unique(K8.decode(np.arange(256, dtype=np.uint8), code))
        vals = vals[np.isfinite(vals) & (np.abs(vals) <= K8.MOST[code])]
        got = K8.decode(K8.encode(x, code), code)
        best = np.abs(np.clip(x, vals[0], vals[-1])[:, None] - vals).min(1)
        assert (np.abs(got - np.clip(x, vals[0], vals[-1])) <= best).all()
        assert np.array_equal(K8.decode(K8.encode(vals, code), code), vals)


def test_codes_against_torch():
    torch = pytest.importorskip("torch")
    rng = np.random.default_rng(1)
    x = np.clip(rng.standard_normal(100000) * np.exp2(rng.integers(-12, 9, 100000)), -448, 448).astype(np.float32)
    bits = torch.from_numpy(x).to(torch.float8_e4m3fn)
    assert np.array_equal(K8.encode(x, K8.E4M3), bits.view(torch.uint8).numpy())
    assert np.array_equal(K8.decode(bits.view(torch.uint8).numpy(), K8.E4M3), bits.double().numpy())


def test_growth_stays_below_a_step():
    """Rows kept over any number of growths are off by less than one step of the last scale."""
    rng = np.random.default_rng(2)
    for code in (K8.E4M3, K8.INT8):
        codes, scale = np.zeros((1, 1, 16, 64), np.uint8), np.zeros((1, 1))
        rows = rng.standard_normal((16, 1, 64)) * np.exp2(np.arange(16))[:, None, None]
        for i in range(16):
            K8.write(codes, scale, rows[i:i + 1], [i], code)
        got = K8.decode(codes[0, 0], code) * scale[0, 0]
        s = scale[0, 0]
        step = s if code == K8.INT8 else np.maximum(2.0 ** (np.floor(np.log2(np.maximum(np.abs(rows[:, 0]) / s, 2.0 ** -6))) - 3), 2.0 ** -9) * s
        assert (np.abs(got - rows[:, 0]) < step * 1.0001).all()
