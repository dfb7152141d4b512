"""Speculative decoding over the paged cache: what its operators are timed on.

A step drafts a tree of tokens for every request, stores the drafted keys and values in
the paged cache, attends from every drafted token to the request's context and to the
token's own ancestors, and keeps the rows of the branch that the model accepts.

Operators
  kv_append   q, k and v rows of a (fused) projection: q and k rotated at the rows'
              positions, q packed, k and v stored in the pool's slots (-1: a padding row).
  tree_mask   the ancestor bits and depths of drafted trees from their parent indices.
  attn_tree   attention of the drafted tokens: a token sees the context's keys inside its
              window and the drafted tokens whose bits its mask row has.
  kv_keep     the accepted rows of every tree move to the front of the tree's slots.
"""
import math
import random

import numpy as np
import torch

own = False

BLOCK = 16
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def attn_tree(reqs=1, nodes=8, ctx=1024, ragged=False, shared=False, window=False, hq=32, hkv=8, d=128, dtype="bf16",
              style="neox", table=True, rotary=0, prerotated=False, theta=5e5, layout=1):
    return dict(op="attn_tree", reqs=reqs, nodes=nodes, ctx=ctx, ragged=ragged, shared=shared, window=window, hq=hq, hkv=hkv,
                d=d, dtype=dtype, style=style, table=table, rotary=rotary, prerotated=prerotated, theta=theta, layout=layout)


def kv_append(rows=64, hq=32, hkv=8, d=128, dtype="bf16", style="neox", rotary=0, fused=True, padded=False, rotate=True,
              theta=5e5, layout=1):
    return dict(op="kv_append", rows=rows, hq=hq, hkv=hkv, d=d, dtype=dtype, style=style, rotary=rotary, fused=fused,
                padded=padded, rotate=rotate, theta=theta, layout=layout)


def tree_mask(trees=64, nodes=64, ragged=False, layout=1):
    return dict(op="tree_mask", trees=trees, nodes=nodes, ragged=ragged, layout=layout)


def kv_keep(trees=64, nodes=64, path=8, hkv=8, d=128, dtype="bf16", layout=1):
    return dict(op="kv_keep", trees=trees, nodes=nodes, path=path, hkv=hkv, d=d, dtype=dtype, layout=layout)


def listed():
    cases = {
        # one user of an 8B-shaped model, a small tree: the latency of one call
        "tree_single": attn_tree(nodes=8, ctx=1537),
        # sixteen users over a common set of documents, contexts and trees of odd sizes
        "tree_batch": attn_tree(reqs=16, nodes=33, ctx=4000, ragged=True, shared=True),
        # sixteen users of a 70B-shaped model, wide trees: the most arithmetic
        "tree_wide": attn_tree(reqs=16, nodes=96, ctx=8192, hq=64),
        # one user with a very long context
        "tree_long": attn_tree(nodes=26, ctx=131072, hq=64),
        # full precision and a small model, as drafting is validated with: interleaved
        # pairs, half of each head rotated, cos/sin not tabulated
        "tree_f32": attn_tree(reqs=3, nodes=13, ctx=700, ragged=True, hq=8, hkv=2, d=64, dtype="f32", style="gptj",
                              table=False, rotary=32, theta=1e4),
        # the drafted rows of sixteen users
        "append_step": kv_append(rows=528, padded=True),
        # a prompt's rows of a 70B-shaped model
        "append_prompt": kv_append(rows=16384, hq=64),
        # full precision, q, k and v in tensors of their own
        "append_f32": kv_append(rows=573, hq=8, hkv=2, d=64, dtype="f32", style="gptj", rotary=32, fused=False, padded=True,
                                theta=1e4),
        # the trees of sixty-four users
        "mask_batch": tree_mask(trees=64, nodes=61, ragged=True),
        # very large trees of few users
        "mask_large": tree_mask(trees=3, nodes=1000),
        # sixty-four users accept a few tokens each
        "keep_batch": kv_keep(trees=64, nodes=64, path=8),
        # many users and long accepted branches, full precision
        "keep_f32": kv_keep(trees=256, nodes=129, path=41, hkv=2, d=64, dtype="f32"),
    }
    return [dict(c, name=n) for n, c in cases.items()]


def _logint(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["attn_tree"] * 5 + ["kv_append"] * 2 + ["tree_mask", "kv_keep"])
    layout = rng.randrange(1, 1 << 20)
    hq, hkv, d = rng.choice([(32, 8, 128), (64, 8, 128), (32, 8, 64), (28, 4, 128), (8, 2, 64), (12, 12, 64), (16, 1, 128)])
    style = rng.choice(["neox", "neox", "gptj"])
    theta = rng.choice([1e4, 5e5])
    rotary = d // 2 if rng.random() < 0.15 else 0
    f32 = rng.random() < 0.2
    if op == "attn_tree":
        reqs = _logint(rng, 1, 64)
        nodes = _logint(rng, 1, 512 // max(1, reqs // 8))
        # at most the arithmetic and the keys of the largest listed case (float32: far below it)
        most = min(131072 // reqs, int((1e10 if f32 else 4e11) / (4.0 * d * hq * reqs * nodes)))
        ctx = _logint(rng, 1, max(2, most)) - 1
        return attn_tree(reqs=reqs, nodes=nodes, ctx=ctx, ragged=rng.random() < 0.6, shared=rng.random() < 0.3,
                         window=rng.random() < 0.15, hq=hq, hkv=hkv, d=d, dtype="f32" if f32 else "bf16", style=style,
                         table=rng.random() < 0.7, rotary=rotary, prerotated=rng.random() < 0.2, theta=theta, layout=layout)
    if op == "kv_append":
        return kv_append(rows=_logint(rng, 1, 8192 if f32 else 16384), hq=hq, hkv=hkv, d=d, dtype="f32" if f32 else "bf16",
                         style=style, rotary=rotary, fused=rng.random() < 0.7, padded=rng.random() < 0.5,
                         rotate=rng.random() < 0.8, theta=theta, layout=layout)
    if op == "tree_mask":
        trees = _logint(rng, 1, 256)
        return tree_mask(trees=trees, nodes=_logint(rng, 1, min(1024, 16384 // trees)), ragged=rng.random() < 0.5, layout=layout)
    nodes = _logint(rng, 2, 256)
    return kv_keep(trees=_logint(rng, 1, 256), nodes=nodes, path=_logint(rng, 1, max(1, nodes // 2)), hkv=hkv, d=d,
                   dtype="f32" if f32 else "bf16", layout=layout)


# ------------------------------------------------------------------------------------
# layout: lengths (from the case alone)
# ------------------------------------------------------------------------------------

def _tree_lengths(c):
    """Per request: context tokens, drafted tokens, window start."""
    rng = random.Random(c["layout"])
    out = []
    for _ in range(c["reqs"]):
        ctx = rng.randint(c["ctx"] // 4, c["ctx"]) if c["ragged"] else c["ctx"]
        n = rng.randint(max(1, c["nodes"] // 4), c["nodes"]) if c["ragged"] else c["nodes"]
        out.append((ctx, n, rng.randint(0, ctx) if c["window"] else 0))
    return out


def _context_blocks(c):
    """Per request the number of each of its full context blocks (shared: drawn from common
    documents of 32 blocks), and how many different ones there are."""
    rng = random.Random(c["layout"] + 1)
    lens = _tree_lengths(c)
    doc = 32
    docs = max(1, max(ctx // BLOCK for ctx, _, _ in lens) // doc + 1)
    out, used = [], 0
    if c["shared"]:
        used = docs * doc
    for ctx, _, _ in lens:
        full = ctx // BLOCK
        if c["shared"]:
            order = rng.sample(range(docs), docs)
            out.append([dd * doc + i for dd in order for i in range(doc)][:full])
        else:
            out.append(list(range(used, used + full)))
            used += full
    return out, used


def _counts(c, n, most):
    rng = random.Random(c["layout"])
    return [rng.randint(max(1, most // 4), most) if c.get("ragged") else most for _ in range(n)]


def _parents(rng, n):
    """A drafted tree: node 0 is the last accepted token, any earlier node may have children."""
    p = np.full(n, -1, np.int32)
    for i in range(1, n):
        p[i] = rng.integers(0, i)
    return p


def _ancestors(p, words):
    """Bits (uint64 words) of every node's ancestors and itself, and its depth."""
    bits = np.zeros((len(p), words), np.uint64)
    depth = np.zeros(len(p), np.int32)
    for i, q in enumerate(p):
        if q >= 0:
            bits[i] = bits[q]
            depth[i] = depth[q] + 1
        bits[i, i // 64] |= np.uint64(1) << np.uint64(i % 64)
    return bits, depth


# ------------------------------------------------------------------------------------
# state
# ------------------------------------------------------------------------------------

def _randn(gen, shape, dtype):
    t = torch.empty(shape, dtype=dtype, device="cuda")
    flat = t.view(-1)
    step = 1 << 26
    for i in range(0, flat.numel(), step):
        n = min(step, flat.numel() - i)
        flat[i:i + n] = torch.randn(n, generator=gen, device="cuda", dtype=torch.float32)
    return t


def _cfg(c):
    from paper_2606_13126_amd import _binding as B
    return B.make_config(c["hq"], c["hkv"], c["d"], dtype=B.PIC_F32 if c["dtype"] == "f32" else B.PIC_BF16,
                         rope_theta=c["theta"], rope_style=B.PIC_ROPE_GPTJ if c["style"] == "gptj" else B.PIC_ROPE_NEOX,
                         rotary_dim=c["rotary"], k_prerotated=int(c.get("prerotated", c.get("rotate", False))))


def _prepare_tree(c, seed):
    rng = np.random.default_rng([seed, 1])
    gen = torch.Generator(device="cuda").manual_seed(seed)
    lens = _tree_lengths(c)
    blocks, used = _context_blocks(c)
    seq = np.array([ctx + n for ctx, n, _ in lens], np.int32)
    table = np.zeros((len(lens), max(-(-int(s) // BLOCK) for s in seq)), np.int32)
    words = max(-(-n // 64) for _, n, _ in lens)
    pos, mask = [], []
    for r, (ctx, n, _) in enumerate(lens):
        full, total = ctx // BLOCK, -(-(ctx + n) // BLOCK)
        table[r, :full] = blocks[r]
        table[r, full:total] = np.arange(used, used + total - full)   # blocks with drafted tokens are the request's own
        used += total - full
        bits, depth = _ancestors(_parents(rng, n), words)
        mask.append(bits)
        pos.append(np.concatenate([np.arange(ctx), ctx + depth]).astype(np.int32))
    table = rng.permutation(used).astype(np.int32)[table]
    dt = DTYPES[c["dtype"]]
    rows = sum(n for _, n, _ in lens)
    s = dict(case=c, lens=lens, seq=seq, mask=torch.from_numpy(np.concatenate(mask).view(np.int64)).cuda(),
             positions=torch.from_numpy(np.concatenate(pos)).cuda(), block_tables=torch.from_numpy(table).cuda(),
             q=_randn(gen, (rows, c["hq"], c["d"]), dt), k_pool=_randn(gen, (used, c["hkv"], BLOCK, c["d"]), dt),
             v_pool=_randn(gen, (used, c["hkv"], BLOCK, c["d"]), dt))
    if own:
        from paper_2606_13126_amd import _binding as B
        cu, start, flags, win = [0], [], [], []
        for ctx, n, w in lens:
            if ctx > 0:
                start.append(0)
                flags.append(B.PIC_PDEP)
                win.append(-1)
            start.append(ctx)
            flags.append(B.PIC_PDEP | B.PIC_QUERY)
            win.append(w)
            cu.append(len(start))
        s["cfg"] = _cfg(c)
        s["host"] = B.HostBatch(seq, cu, start, flags, win)
        s["o"] = torch.empty_like(s["q"])
        s["ws"] = torch.empty(max(1, B.pic_tree_workspace_size(s["cfg"], s["host"])), dtype=torch.uint8, device="cuda")
        s["table"] = None
        if c["table"] and not c["prerotated"]:
            n_pos = int(seq.max())
            s["table"] = torch.empty((n_pos, c["d"] // 2) + ((2,) if c["dtype"] == "f32" else ()), dtype=torch.float32,
                                     device="cuda")
            B.pic_rope_table_build(s["cfg"], s["table"])
    return s


def _prepare_append(c, seed):
    rng = np.random.default_rng([seed, 2])
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n, hq, hkv, d, dt = c["rows"], c["hq"], c["hkv"], c["d"], DTYPES[c["dtype"]]
    nb = -(-n * 5 // 4 // BLOCK) + 1
    slots = rng.permutation(nb)[np.arange(n) // BLOCK] * BLOCK + np.arange(n) % BLOCK   # whole blocks in any order
    if c["padded"]:
        slots[rng.random(n) < 0.1] = -1
    if c["fused"]:
        qkv = _randn(gen, (n, hq + 2 * hkv, d), dt)
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    else:
        q, k, v = (_randn(gen, (n, h, d), dt) for h in (hq, hkv, hkv))
    s = dict(case=c, q=q, k=k, v=v, q_out=torch.empty((n, hq, d), dtype=dt, device="cuda"),
             slots=torch.from_numpy(slots.astype(np.int32)).cuda(),
             positions=torch.from_numpy(rng.integers(0, 131072, n).astype(np.int32)).cuda(),
             k_pool=_randn(gen, (nb, hkv, BLOCK, d), dt), v_pool=_randn(gen, (nb, hkv, BLOCK, d), dt))
    if own:
        s["cfg"] = _cfg(c)
    return s


def _prepare_mask(c, seed):
    rng = np.random.default_rng([seed, 3])
    ns = _counts(c, c["trees"], c["nodes"])
    parents = np.concatenate([_parents(rng, n) for n in ns])
    words = -(-max(ns) // 64)
    return dict(case=c, most=max(ns), words=words, parents=torch.from_numpy(parents).cuda(),
                cu_rows=torch.from_numpy(np.concatenate([[0], np.cumsum(ns)]).astype(np.int32)).cuda(),
                mask=torch.empty((len(parents), words), dtype=torch.int64, device="cuda"),
                depth=torch.empty(len(parents), dtype=torch.int32, device="cuda"))


def _prepare_keep(c, seed):
    rng = np.random.default_rng([seed, 4])
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t, n, m, dt = c["trees"], c["nodes"], c["path"], DTYPES[c["dtype"]]
    per = -(-(n + BLOCK) // BLOCK)
    blocks = rng.permutation(t * per).reshape(t, per)
    at = rng.integers(0, BLOCK, (t, 1)) + np.arange(n)          # a tree starts anywhere in its first block
    slots = blocks[np.arange(t)[:, None], at // BLOCK] * BLOCK + at % BLOCK
    path = np.zeros((t, m), np.int32)
    length = np.zeros(t, np.int32)
    for r in range(t):
        # an accepted node is in its place already or comes from behind the accepted length,
        # so that a second pass over the same state moves the same rows
        k = int(rng.integers(1, m + 1))
        k = min(k, n)
        first = int(rng.integers(1, k + 1))
        tail = np.sort(rng.choice(np.arange(k, n), size=min(k - first, n - k), replace=False))
        length[r] = first + len(tail)
        tail = tail[tail >= length[r]] if len(tail) else tail
        path[r, :first] = np.arange(first)
        length[r] = first + len(tail)
        path[r, first:length[r]] = tail
    nb = t * per
    s = dict(case=c, slots=torch.from_numpy(slots.reshape(-1).astype(np.int32)).cuda(),
             cu_rows=torch.arange(0, t * n + 1, n, dtype=torch.int32, device="cuda"), path=torch.from_numpy(path).cuda(),
             length=torch.from_numpy(length).cuda(), k_pool=_randn(gen, (nb, c["hkv"], BLOCK, c["d"]), dt),
             v_pool=_randn(gen, (nb, c["hkv"], BLOCK, c["d"]), dt))
    if own:
        from paper_2606_13126_amd import _binding as B
        s["cfg"] = B.make_config(c["hkv"], c["hkv"], c["d"], dtype=B.PIC_F32 if c["dtype"] == "f32" else B.PIC_BF16)
    return s


def prepare(case, seed):
    return {"attn_tree": _prepare_tree, "kv_append": _prepare_append, "tree_mask": _prepare_mask,
            "kv_keep": _prepare_keep}[case["op"]](case, seed)


# ------------------------------------------------------------------------------------
# one pass: the framework's calls, or the plain form
# ------------------------------------------------------------------------------------

def _rotate(x, pos, c):
    """x [n][heads][d] float32 turned at positions pos [n]; the angles in 64 bits."""
    rot = c["rotary"] or c["d"]
    half = rot // 2
    freq = c["theta"] ** (-2.0 * torch.arange(half, dtype=torch.float64, device=x.device) / rot)
    ang = pos.double()[:, None] * freq
    cos, sin = torch.cos(ang).float()[:, None, :], torch.sin(ang).float()[:, None, :]
    y = x.clone()
    if c["style"] == "neox":
        a, b = x[..., :half], x[..., half:rot]
        y[..., :half] = a * cos - b * sin
        y[..., half:rot] = b * cos + a * sin
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2] = a * cos - b * sin
        y[..., 1:rot:2] = b * cos + a * sin
    return y


def _plain_tree(s):
    c = s["case"]
    g = c["hq"] // c["hkv"]
    out = torch.empty_like(s["q"])
    row, off = 0, 0
    for r, (ctx, n, w) in enumerate(s["lens"]):
        L = ctx + n
        ids = s["block_tables"][r, :-(-L // BLOCK)].long()
        k, v = (p[ids].transpose(1, 2).reshape(-1, c["hkv"], c["d"])[w:L].float() for p in (s["k_pool"], s["v_pool"]))
        q = s["q"][row:row + n].float()
        pos = s["positions"][off:off + L]
        if not c["prerotated"]:
            k = _rotate(k, pos[w:], c)
            q = _rotate(q, pos[ctx:], c)
        # [hkv][n * g][keys]
        q = q.view(n, c["hkv"], g, c["d"]).permute(1, 0, 2, 3).reshape(c["hkv"], n * g, c["d"]).contiguous()
        score = torch.matmul(q, k.permute(1, 2, 0).contiguous()) / math.sqrt(c["d"])
        j = torch.arange(n, device=q.device)
        seen = ((s["mask"][row:row + n][:, j // 64] >> (j % 64)) & 1).bool()
        score = score.view(c["hkv"], n, g, L - w)
        score[..., ctx - w:].masked_fill_(~seen[None, :, None, :], -math.inf)
        score = score.view(c["hkv"], n * g, L - w)
        p = torch.exp(score - score.amax(-1, keepdim=True))
        o = torch.matmul(p, v.permute(1, 0, 2).contiguous()) / p.sum(-1, keepdim=True)
        out[row:row + n] = o.view(c["hkv"], n, g, c["d"]).permute(1, 0, 2, 3).reshape(n, c["hq"], c["d"]).to(out.dtype)
        row, off = row + n, off + L
    return out


def _plain_append(s):
    c = s["case"]
    q, k = s["q"], s["k"]
    if c["rotate"]:
        q = _rotate(q.float(), s["positions"], c).to(q.dtype)
        k = _rotate(k.float(), s["positions"], c).to(k.dtype)
    s["q_out"].copy_(q)
    rows = (s["slots"] >= 0).nonzero()[:, 0]
    slot = s["slots"][rows].long()
    s["k_pool"][slot // BLOCK, :, slot % BLOCK] = k[rows]
    s["v_pool"][slot // BLOCK, :, slot % BLOCK] = s["v"][rows]
    return s["q_out"], s["k_pool"], s["v_pool"]


def _plain_mask(s):
    n, words = s["most"], s["words"]
    cu = s["cu_rows"].long()
    idx = torch.arange(n, device=cu.device)
    valid = idx < (cu[1:] - cu[:-1])[:, None]                                  # [trees][n]
    at = (cu[:-1, None] + idx).clamp(max=len(s["parents"]) - 1)
    parent = s["parents"][at].long()
    reach = (parent[:, :, None] == idx).float() + torch.eye(n, device=cu.device)   # node to itself and its parent
    reach *= valid[:, :, None]
    for _ in range(max(1, (n - 1).bit_length())):
        reach = (torch.matmul(reach, reach) > 0).float()
    depth = reach.sum(-1).int() - 1
    bits = torch.zeros(reach.shape[0], n, words * 64, dtype=torch.int64, device=cu.device)
    bits[:, :, :n] = reach.long()
    mask = (bits.view(-1, n, words, 64) << torch.arange(64, device=cu.device)).sum(-1)
    s["mask"][at[valid]] = mask[valid]
    s["depth"][at[valid]] = depth[valid]
    return s["mask"], s["depth"]


def _plain_keep(s):
    i = torch.arange(s["path"].shape[1], device=s["path"].device)
    take = i < s["length"][:, None]
    first = s["cu_rows"][:-1, None]
    src = s["slots"][(first + s["path"])[take]].long()
    dst = s["slots"][(first + i)[take]].long()
    for pool in (s["k_pool"], s["v_pool"]):
        pool[dst // BLOCK, :, dst % BLOCK] = pool[src // BLOCK, :, src % BLOCK]
    return s["k_pool"], s["v_pool"]


def run(state):
    s, op = state, state["case"]["op"]
    if not own:
        return {"attn_tree": _plain_tree, "kv_append": _plain_append, "tree_mask": _plain_mask, "kv_keep": _plain_keep}[op](s)
    from paper_2606_13126_amd import _binding as B
    if op == "attn_tree":
        B.pic_attn_tree(s["cfg"], s["host"], s["block_tables"], s["positions"], s["mask"], s["q"], s["o"], s["k_pool"],
                        s["v_pool"], workspace=s["ws"], table=s["table"])
        return s["o"]
    if op == "kv_append":
        B.pic_kv_append(s["cfg"], s["k_pool"], s["v_pool"], s["k"], s["v"], s["positions"], s["slots"], q=s["q"],
                        q_out=s["q_out"])
        return s["q_out"], s["k_pool"], s["v_pool"]
    if op == "tree_mask":
        B.pic_tree_mask(s["parents"], s["cu_rows"], s["mask"], depth=s["depth"])
        return s["mask"], s["depth"]
    B.pic_kv_keep(s["cfg"], s["k_pool"], s["v_pool"], s["slots"], s["cu_rows"], s["path"], s["length"])
    return s["k_pool"], s["v_pool"]


def work(case):
    c = case
    es = 4 if c.get("dtype") == "f32" else 2
    if c["op"] == "attn_tree":
        lens = _tree_lengths(c)
        rows = sum(n for _, n, _ in lens)
        blocks, _ = _context_blocks(c)
        seen = set()
        keys = 0
        for (ctx, n, w), b in zip(lens, blocks):
            seen.update(b[w // BLOCK:])
            keys += ctx + n - max(w, ctx // BLOCK * BLOCK)   # the request's own blocks
        keys += len(seen) * BLOCK
        pairs = sum(n * (ctx - w + 1) for ctx, n, w in lens)
        return {"bytes": 2 * rows * c["hq"] * c["d"] * es + 2 * keys * c["hkv"] * c["d"] * es, "flops": 4 * c["d"] * c["hq"] * pairs}
    if c["op"] == "kv_append":
        each = (c["hq"] + 2 * c["hkv"]) * c["d"]
        return {"bytes": c["rows"] * (2 * each * es + 8), "flops": 3 * c["rows"] * (c["hq"] + c["hkv"]) * c["d"] if c["rotate"] else 0}
    if c["op"] == "tree_mask":
        ns = _counts(c, c["trees"], c["nodes"])
        return {"bytes": sum(ns) * (8 + 8 * -(-max(ns) // 64)), "flops": 0}
    rows = c["trees"] * max(1, c["path"] // 4)   # about what the accepted branches move
    return {"bytes": 4 * rows * c["hkv"] * c["d"] * es, "flops": 0}


# ------------------------------------------------------------------------------------
# the definitions in 64 bits
# ------------------------------------------------------------------------------------

def _turned(x, pos, c):
    """x [n][heads][d] float64, each pair as a complex number times e^(i pos omega)."""
    rot = c["rotary"] or c["d"]
    om = torch.tensor([c["theta"] ** (-2.0 * i / rot) for i in range(rot // 2)], dtype=torch.float64, device=x.device)
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=x.device), pos.double()[:, None, None] * om)
    if c["style"] == "neox":
        z = torch.complex(x[..., :rot // 2], x[..., rot // 2:rot]) * turn
        return torch.cat([z.real, z.imag, x[..., rot:]], -1)
    z = torch.complex(x[..., 0:rot:2].contiguous(), x[..., 1:rot:2].contiguous()) * turn
    return torch.cat([torch.stack([z.real, z.imag], -1).flatten(-2), x[..., rot:]], -1)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "tree_mask":
        cu, parents = s["cu_rows"].tolist(), s["parents"].cpu().numpy()
        got = [_ancestors(parents[a:b], s["words"]) for a, b in zip(cu, cu[1:])]
        return (torch.from_numpy(np.concatenate([m for m, _ in got]).view(np.int64)),
                torch.from_numpy(np.concatenate([d for _, d in got])))
    if c["op"] == "kv_keep":
        pools = [s["k_pool"].double(), s["v_pool"].double()]
        slots = s["slots"].tolist()
        for r, (path, m) in enumerate(zip(s["path"].tolist(), s["length"].tolist())):
            for i in range(m):   # ascending: no row is overwritten before it has moved
                a, b = slots[r * c["nodes"] + path[i]], slots[r * c["nodes"] + i]
                if a != b:
                    for p in pools:
                        p[b // BLOCK, :, b % BLOCK] = p[a // BLOCK, :, a % BLOCK]
        return tuple(pools)
    if c["op"] == "kv_append":
        q, k, v = s["q"].double(), s["k"].double(), s["v"].double()
        if c["rotate"]:
            q, k = _turned(q, s["positions"], c), _turned(k, s["positions"], c)
        out = []
        at = [(i, t) for i, t in enumerate(s["slots"].tolist()) if t >= 0]
        rows, slot = (torch.tensor([x[e] for x in at], dtype=torch.long, device="cuda") for e in (0, 1))
        for pool, new in ((s["k_pool"], k), (s["v_pool"], v)):
            flat = pool.double().transpose(1, 2).reshape(-1, c["hkv"], c["d"])
            flat[slot] = new[rows]
            out.append(flat.view(-1, BLOCK, c["hkv"], c["d"]).transpose(1, 2).contiguous())
        return q, out[0], out[1]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    row, off, g = 0, 0, c["hq"] // c["hkv"]
    for r, (ctx, n, w) in enumerate(s["lens"]):
        L = ctx + n
        j = torch.arange(w, L, device="cuda")
        blk = s["block_tables"][r].long()[j // BLOCK]
        bit = torch.arange(n, device="cuda")
        see = ((s["mask"][row:row + n][:, bit // 64] >> (bit % 64)) & 1).bool()
        see = torch.cat([torch.ones(n, ctx - w, dtype=torch.bool, device="cuda"), see], 1)
        pos = s["positions"][off:off + L]
        for h in range(c["hkv"]):
            k = s["k_pool"][blk, h, j % BLOCK].double()
            v = s["v_pool"][blk, h, j % BLOCK].double()
            q = s["q"][row:row + n, h * g:(h + 1) * g].double()
            if not c["prerotated"]:
                k = _turned(k[:, None], pos[w:], c)[:, 0]
                q = _turned(q, pos[ctx:], c)
            for a in range(g):
                x = torch.matmul(q[:, a], k.T.contiguous()) * c["d"] ** -0.5
                x = torch.where(see, x, -math.inf)
                out[row:row + n, h * g + a] = torch.matmul(torch.softmax(x, -1), v)
        row, off = row + n, off + L
    return out
