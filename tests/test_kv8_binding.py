"""The binding of the cache held in 8 bits refuses tensors of other types, which the library would read as the types that
it was told: an int64 slot mapping as pairs of int32, integer codes as e4m3.  (No GPU: nothing is launched.)"""
import pytest

torch = pytest.importorskip("torch")
B = pytest.importorskip("paper_2606_13126_amd._binding")

E4M3, INT8 = B.PIC_KV8_E4M3, B.PIC_KV8_INT8


def pool(kind=torch.uint8, code=INT8, scale=torch.float32, v=None):
    k = torch.zeros(3, 1, 16, 64, dtype=torch.uint8)
    as_ = lambda t: k.view(t) if t.itemsize == 1 else k.to(t)   # noqa: E731
    return B.Kv8Pool(as_(kind), as_(v or kind), torch.zeros(3, 1, 2, dtype=scale), code)


def test_pools():
    for kind, code in ((torch.uint8, E4M3), (torch.uint8, INT8), (torch.int8, INT8), (torch.float8_e4m3fn, E4M3)):
        pool(kind, code)
    for kind, code in ((torch.int8, E4M3), (torch.float8_e4m3fn, INT8), (torch.float8_e5m2, E4M3), (torch.float8_e4m3fnuz, E4M3),
                       (torch.bool, INT8), (torch.int16, INT8), (torch.uint8, 2), (torch.uint8, -1)):
        with pytest.raises(ValueError):
            pool(kind, code)
    with pytest.raises(ValueError):
        pool(torch.int8, INT8, v=torch.float8_e4m3fn)
    for scale in (torch.int32, torch.uint32, torch.bfloat16, torch.float64):
        with pytest.raises(ValueError):
            pool(scale=scale)


@pytest.mark.parametrize("dtype,cfg_dtype", [(torch.bfloat16, B.PIC_BF16), (torch.float32, B.PIC_F32)])
def test_rows_slots_and_positions(dtype, cfg_dtype):
    cfg, other = B.make_config(2, 1, 64, dtype=cfg_dtype), torch.float32 if dtype == torch.bfloat16 else torch.bfloat16
    half = torch.float16
    p = pool()
    q, k, w = torch.zeros(3, 2, 64, dtype=dtype), torch.zeros(3, 1, 64, dtype=dtype), torch.ones(64, dtype=dtype)
    ids = torch.zeros(3, dtype=torch.int32)
    gaps = torch.zeros(6, dtype=torch.int32)[::2]

    def refused(f, *a, **kw):
        with pytest.raises(ValueError):
            f(*a, **kw, stream=0)
    for bad in (ids.long(), ids.short(), gaps, ids.float()):
        refused(B.pic_kv8_write, cfg, p, k, k, bad)
        refused(B.pic_kv8_read, cfg, p, bad, k, k)
        refused(B.pic_qk_norm, cfg, q, k, w, w, 1e-6, bad)
    refused(B.pic_qk_norm, cfg, q, k, w, w, 1e-6, ids[:2])
    for t in (other, half):
        refused(B.pic_kv8_write, cfg, p, k.to(t), k, ids)
        refused(B.pic_kv8_write, cfg, p, k, k.to(t), ids)
        refused(B.pic_kv8_read, cfg, p, ids, k.to(t), k)
        refused(B.pic_kv8_read, cfg, p, ids, k, k.to(t))
        refused(B.pic_qk_norm, cfg, q.to(t), k, w, w, 1e-6, ids)
        refused(B.pic_qk_norm, cfg, q, k.to(t), w, w, 1e-6, ids)
        refused(B.pic_qk_norm, cfg, q, k, w.to(t), w, 1e-6, ids)
        refused(B.pic_qk_norm, cfg, q, k, w, w.to(t), 1e-6, ids)
        refused(B.pic_qk_norm, cfg, q, k, w, w, 1e-6, ids, q_out=torch.zeros(3, 2, 64, dtype=t))
    refused(B.pic_qk_norm, cfg, q, k, w[:32], w, 1e-6, ids)
    refused(B.pic_qk_norm, cfg, q, k, w, torch.ones(128, dtype=dtype)[::2], 1e-6, ids)


@pytest.mark.parametrize("call", [B.pic_attn8_prefill, B.pic_attn8_decode])
def test_attention(call):
    cfg = B.make_config(2, 1, 64)
    host = B.HostBatch([20], [0, 2], [0, 19], [B.PIC_PDEP, B.PIC_PDEP | B.PIC_QUERY])
    good = dict(block_tables=torch.zeros(1, 2, dtype=torch.int32), positions=torch.arange(20, dtype=torch.int32),
                q=torch.zeros(1, 2, 64, dtype=torch.bfloat16), o=torch.zeros(1, 2, 64, dtype=torch.bfloat16), pool=pool())
    for kw in (dict(block_tables=good["block_tables"].long()), dict(positions=good["positions"].long()), dict(positions=torch.arange(40, dtype=torch.int32)[::2]),
               dict(block_tables=torch.zeros(2, 1, dtype=torch.int32).t().expand(2, 2)), dict(q=good["q"].float()), dict(o=good["o"].half()),
               dict(q=torch.zeros(1, 2, 128, dtype=torch.bfloat16)[:, :, ::2])):
        with pytest.raises(ValueError):
            call(cfg, host, **{**good, **kw}, stream=0)
