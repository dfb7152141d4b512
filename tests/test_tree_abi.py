"""Speculative decoding without a GPU: arguments are refused before any HIP call, and the plan
of pic_attn_tree covers every (row, key) pair once."""
import ctypes

import numpy as np
import pytest

P = pytest.importorskip("paper_2606_13126_amd")
from paper_2606_13126_amd import _binding as B  # noqa: E402

OK = 4096   # an address that passes the alignment checks and is never used


def status(name, *args):
    rc = getattr(B.lib(), name)(*[ctypes.byref(a) if isinstance(a, ctypes.Structure) else a for a in args])
    return rc, B.lib().pic_last_error().decode()


def batch(lens, window=None):
    """One request per (context, drafted tokens); 0 drafted: no query span."""
    seq, cu, start, flags, win = [], [0], [], [], []
    for ctx, n in lens:
        if ctx:
            start.append(0), flags.append(B.PIC_PDEP), win.append(-1)
        if n:
            start.append(ctx), flags.append(B.PIC_PDEP | B.PIC_QUERY), win.append(-1 if window is None else min(window, ctx))
        seq.append(ctx + n)
        cu.append(len(start))
    return B.HostBatch(seq, cu, start, flags, win)


def append_args(cfg, **kw):
    a = dict(k_pool=OK, v_pool=OK, num_blocks=4, q=1 << 20, q_stride=256, q_out=1 << 22, k_new=1 << 24, k_stride=64, v_new=1 << 25,
             v_stride=64, positions=OK, slots=OK, n=3)
    a.update(kw)
    return ("pic_kv_append", cfg, a["k_pool"], a["v_pool"], a["num_blocks"], a["q"], a["q_stride"], a["q_out"], a["k_new"],
            a["k_stride"], a["v_new"], a["v_stride"], a["positions"], a["slots"], a["n"], None)


@pytest.mark.parametrize("kw,what", [
    (dict(n=-1), "n and num_blocks"), (dict(num_blocks=-1), "n and num_blocks"), (dict(num_blocks=0), "empty pool"),
    (dict(k_pool=None), "NULL"), (dict(v_new=None), "NULL"), (dict(slots=None), "NULL"), (dict(q_out=None), "both"),
    (dict(q=None), "both"), (dict(positions=None), "positions"), (dict(n=1 << 24), "2^24"),
    (dict(q_stride=248), "strides"), (dict(k_stride=56), "strides"), (dict(v_stride=-64), "strides"),
    (dict(k_stride=1 << 62), "strides"), (dict(q_stride=260), "aligned"), (dict(k_stride=68), "aligned"),
    (dict(k_pool=OK + 8), "aligned"), (dict(q=OK + 8), "aligned"), (dict(q_out=OK + 8), "aligned"),
    (dict(slots=OK + 2), "aligned"), (dict(positions=OK + 2), "aligned"),
    (dict(q_out=1 << 20, q_stride=512), "overlaps"),                      # in place needs dense rows
    (dict(q_out=(1 << 20) + 512), "overlaps"), (dict(q_out=1 << 24), "overlaps"), (dict(q_out=(1 << 25) - 16), "overlaps"),
])
def test_kv_append_refuses(kw, what):
    cfg = B.make_config(4, 1, 64, k_prerotated=1)
    rc, msg = status(*append_args(cfg, **kw))
    assert rc == B.PIC_EINVAL and what in msg, (rc, msg)


def test_nothing_to_do_is_no_error():
    cfg = B.make_config(4, 1, 64, k_prerotated=1)
    assert status(*append_args(cfg, n=0))[0] == B.PIC_OK
    assert status("pic_tree_mask", None, None, 0, 5, None, 1, None, None)[0] == B.PIC_OK
    assert status("pic_tree_mask", None, None, 3, 0, None, 1, None, None)[0] == B.PIC_OK
    assert status("pic_kv_keep", cfg, None, None, 0, None, None, 0, 0, None, 0, None, None)[0] == B.PIC_OK
    hb = batch([(5, 0), (1, 0)])   # no request drafts anything
    dev = B.pic_batch_dev(OK, 4, OK)
    rc, _ = status("pic_attn_tree", cfg, hb.c, dev, B._rope(None), None, 0, None, None, OK, OK, 4, None, 0, None)
    assert rc == B.PIC_OK
    assert B.pic_tree_workspace_size(cfg, hb) == 0


@pytest.mark.parametrize("args,what", [
    ((OK, OK, -1, 5, OK, 1, None, None), "n_trees"), ((OK, OK, 1, -5, OK, 1, None, None), "n_trees"),
    ((OK, OK, 1, 5, OK, 0, None, None), "mask_words"), ((OK, OK, 1, 5, OK, 65, None, None), "mask_words"),
    ((OK, OK, 65536, 5, OK, 1, None, None), "2^16"), ((None, OK, 1, 5, OK, 1, None, None), "NULL"),
    ((OK, None, 1, 5, OK, 1, None, None), "NULL"), ((OK, OK, 1, 5, None, 1, None, None), "NULL"),
    ((OK, OK, 1, 5, OK + 4, 1, None, None), "aligned"), ((OK + 2, OK, 1, 5, OK, 1, None, None), "aligned"),
    ((OK, OK, 1, 5, OK, 1, OK + 2, None), "aligned"),
])
def test_tree_mask_refuses(args, what):
    rc, msg = status("pic_tree_mask", *args)
    assert rc == B.PIC_EINVAL and what in msg, (rc, msg)


@pytest.mark.parametrize("at,value,what", [
    (0, None, "NULL"), (1, OK + 8, "aligned"), (2, 0, "empty pool"), (2, -1, ">= 0"), (3, None, "NULL"), (4, OK + 1, "aligned"),
    (5, -1, ">= 0"), (5, 1 << 23, "2^23"), (6, -1, ">= 0"), (7, OK + 2, "aligned"), (8, -2, ">= 0"), (9, None, "NULL"),
])
def test_kv_keep_refuses(at, value, what):
    args = [OK, OK, 4, OK, OK, 2, 20, OK, 3, OK]
    args[at] = value
    rc, msg = status("pic_kv_keep", B.make_config(4, 1, 64), *args, None)
    assert rc == B.PIC_EINVAL and what in msg, (rc, msg)


def tree_call(cfg, hb, max_blocks=64, mask=OK, words=1, q=OK, o=OK, ws=OK, ws_bytes=1 << 30, k=OK):
    return status("pic_attn_tree", cfg, hb.c, B.pic_batch_dev(OK, max_blocks, OK), B._rope(None), mask, words, q, o, k, OK, 64, ws,
                  ws_bytes, None)


def test_attn_tree_refuses():
    cfg, hb = B.make_config(4, 1, 64), batch([(900, 70)])
    assert tree_call(cfg, hb, words=1) == (B.PIC_EINVAL, "mask_words too small for a span of 70 drafted tokens")
    for kw, what in ((dict(mask=None, words=2), "tree_mask"), (dict(words=-1), "mask_words"), (dict(mask=OK + 4, words=2), "aligned"),
                     (dict(q=None, words=2), "q and o"), (dict(max_blocks=60, words=2), "max_blocks"),
                     (dict(o=OK + 8, words=2), "aligned"), (dict(k=None, words=2), "pools"), (dict(ws=OK + 8, words=2), "aligned")):
        rc, msg = tree_call(cfg, hb, **kw)
        assert rc == B.PIC_EINVAL and what in msg, (kw, rc, msg)
    need = B.pic_tree_workspace_size(cfg, hb)
    assert need > 0
    rc, msg = tree_call(cfg, hb, words=2, ws_bytes=need - 1)
    assert rc == B.PIC_EWORKSPACE, msg
    rc, msg = tree_call(cfg, hb, words=2, ws=None, ws_bytes=0)
    assert rc == B.PIC_EWORKSPACE, msg
    with pytest.raises(P.PicError):
        B.pic_tree_workspace_size(B.make_config(4, 1, 96), hb)


def test_binding_refuses_rows_that_are_not_dense():
    torch = pytest.importorskip("torch")
    cfg = B.make_config(4, 1, 64, k_prerotated=1)
    k = torch.zeros(3, 1, 128)[:, :, ::2]
    pool, ids = torch.zeros(1, 1, 16, 64), torch.zeros(3, dtype=torch.int32)
    good = torch.zeros(3, 1, 64)
    with pytest.raises(ValueError):
        B.pic_kv_append(cfg, pool, pool, k, good, ids, ids, stream=0)
    with pytest.raises(ValueError):
        B.pic_kv_append(cfg, pool, pool, good, good, ids, ids, q=torch.zeros(3, 4, 64), q_out=torch.zeros(3, 8, 64)[:, ::2], stream=0)


@pytest.mark.parametrize("dtype", [B.PIC_BF16, B.PIC_F32])
@pytest.mark.parametrize("hq,hkv,d,lens,window", [
    (32, 8, 128, [(1537, 8)], None), (32, 8, 128, [(0, 1)], None), (8, 2, 64, [(700, 13), (0, 3), (15, 1), (4, 0), (1, 40)], None),
    (64, 8, 128, [(131072, 26)], None), (12, 12, 64, [(100 + 7 * i, 1 + i % 5) for i in range(90)], None),
    (28, 4, 128, [(333, 19), (5000, 64)], 300), (16, 1, 128, [(64, 17)], 64), (4, 4, 64, [(2000, 700)], None),
])
def test_plan_covers_every_pair_once(dtype, hq, hkv, d, lens, window):
    cfg, hb = B.make_config(hq, hkv, d, dtype=dtype), batch(lens, window)
    items = B.pic_tree_plan_debug(cfg, hb)
    g = hq // hkv
    seen, slots = {}, set()
    for r, h, lo, hi, kl, kh, tok0, slot in items.tolist():
        assert 0 <= lo < hi and kl < kh
        seen.setdefault((r, h), []).append((lo, hi, kl, kh, tok0))
        if slot >= 0:
            assert slot not in slots
            slots.add(slot)
    for r, (ctx, n) in enumerate(lens):
        w = 0 if window is None else min(window, ctx)
        for h in range(hkv):
            if n == 0:
                assert (r, h) not in seen
                continue
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
                assert k == ctx + n   # every row tile runs to the span's end
            assert at == n * g


def test_workspace_holds_few_partials():
    # a batch whose items fill the chip is not split
    cfg = B.make_config(32, 8, 128)
    assert B.pic_tree_workspace_size(cfg, batch([(4096, 16)] * 64)) < 64 << 20
    assert B.pic_tree_workspace_size(cfg, batch([(131072, 16)])) <= 256 * 256 * (128 + 2) * 4
