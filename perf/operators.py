"""What the operators of tree drafting and of policy log-probabilities are timed on.

Five kinds of pass, named by a case's "op":
  append         keys and values of new positions rotated and written into the paged cache, the
                 queries rotated beside them (a prompt's rows, or the nodes of a draft tree)
  attention      the attention of a draft tree's nodes over the cache and their own ancestors
  commit         the walk of a draft tree along the target's tokens, and the commit of the path in
                 every layer of the cache
  logprobs       log-probabilities of given tokens, entropies and top alternatives of logits rows
  logprobs_grad  the gradient of log-probabilities and entropies in the logits

Inputs are made on the GPU from the seed alone.  With `own` false a pass runs in elementary torch
operations in float32 (float64 for rotary angles and for sums over the vocabulary); with `own` true
it makes the calls of paper_2609_16648_amd.gm.  `exact` computes the same outputs in float64.
"""
from __future__ import annotations

import math
from types import SimpleNamespace

import numpy as np
import torch

own = False

_DEV = "cuda"
ROPE_BASE, EPS = 10000.0, 1e-6


# ------------------------------------------------------------------------------------- cases
def listed():
    qwen = dict(heads=32, kv_heads=8, dim=128, dtype="bf16")     # the attention of the Qwen3-4B and MiMo-7B shapes
    return [
        # one interactive sequence drafting a small tree: the smallest call, all latency
        dict(name="append_tree_b1", op="append", **qwen, page=16, batch=1, nodes=8, rows_lo=0, rows_hi=0, ctx_lo=4001,
             ctx_hi=4001, norm=True, q=True),
        # a rollout batch's prompts entering the cache: 32 prompts of up to 2000 tokens, none aligned to a page
        dict(name="append_prompts_b32", op="append", **qwen, page=16, batch=32, nodes=0, rows_lo=37, rows_hi=2001,
             ctx_lo=0, ctx_hi=0, norm=True, q=True),
        # the small float32 decoder: a full tree of 64 nodes
        dict(name="attention_f32_n64", op="attention", heads=8, kv_heads=2, dim=64, dtype="f32", page=16, batch=4,
             nodes=64, ctx_lo=100, ctx_hi=1000, ragged=True),
        # one interactive sequence
        dict(name="attention_b1_n8", op="attention", **qwen, page=16, batch=1, nodes=8, ctx_lo=4001, ctx_hi=4001,
             ragged=False),
        # the default rollout batch with trees of 16 nodes
        dict(name="attention_b64_n16", op="attention", **qwen, page=16, batch=64, nodes=16, ctx_lo=1024, ctx_hi=4096,
             ragged=False),
        # the largest trees over long contexts: up to 256 query rows per KV head
        dict(name="attention_b32_n64", op="attention", **qwen, page=32, batch=32, nodes=64, ctx_lo=512, ctx_hi=8704,
             ragged=True),
        # one interactive sequence: all launches and latency
        dict(name="commit_b1_l36", op="commit", **qwen, page=16, batch=1, nodes=8, ctx_lo=50, ctx_hi=50, layers=36),
        # a rollout batch in the whole cache of the 36-layer Qwen3-4B configuration
        dict(name="commit_b64_l36", op="commit", **qwen, page=16, batch=64, nodes=16, ctx_lo=16, ctx_hi=128, layers=36),
        # a decode step's rows with the alternatives that a draft tree is grown from
        dict(name="logprobs_b64_top8", op="logprobs", dtype="f32", rows=64, vocab=151936, temperature=1.0, topk=8,
             masked=False),
        # a policy update's rows
        dict(name="logprobs_m4096", op="logprobs", dtype="f32", rows=4096, vocab=151936, temperature=1.0, topk=0,
             masked=False),
        # a short response of a model with an odd vocabulary
        dict(name="grad_m257_odd", op="logprobs_grad", dtype="f32", rows=257, vocab=50257, temperature=0.7,
             entropy=True),
        # a policy update's rows as bf16 logits, with an entropy bonus
        dict(name="grad_m4096_bf16", op="logprobs_grad", dtype="bf16", rows=4096, vocab=151936, temperature=1.0,
             entropy=True),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


_HEADS = [(32, 8), (32, 8), (32, 8), (16, 8), (28, 4), (8, 8), (64, 8)]
_VOCABS = [151936, 151680, 128256, 50257, 32001, 5003]


def draw(rng):
    op = rng.choice(["append", "append", "attention", "attention", "attention", "commit", "logprobs", "logprobs",
                     "logprobs_grad", "logprobs_grad"])
    if op in ("logprobs", "logprobs_grad"):
        V = rng.choice(_VOCABS)
        c = dict(op=op, dtype=rng.choice(["f32", "f32", "bf16"]), rows=_log_int(rng, 1, 4096), vocab=V,
                 temperature=rng.choice([1.0, 1.0, 0.7, 1.3]))
        if op == "logprobs":
            c.update(topk=rng.choice([0, 0, 1, 4, 8, 20, 64]), masked=rng.choice([False, False, True]))
            if c["topk"]:
                c.update(rows=min(c["rows"], 1024))
        else:
            c.update(entropy=rng.choice([True, True, False]))
        return c
    if rng.random() < 0.15:
        heads, kv = rng.choice([(4, 4), (8, 2)])
        c = dict(op=op, heads=heads, kv_heads=kv, dim=rng.choice([64, 64, 128]), dtype="f32")
    else:
        heads, kv = rng.choice(_HEADS)
        c = dict(op=op, heads=heads, kv_heads=kv, dim=128, dtype="bf16")
    c.update(page=rng.choice([16, 16, 32, 64]))
    small = c["dtype"] == "f32"
    if op == "append":
        B = _log_int(rng, 1, 256)
        c.update(batch=B, norm=rng.choice([True, False]), q=rng.choice([True, True, False]))
        if rng.random() < 0.5:
            c.update(nodes=_log_int(rng, 1, 64), rows_lo=0, rows_hi=0)
        else:
            hi = _log_int(rng, 1, min(16384, 32768 // B))
            c.update(nodes=0, rows_lo=rng.choice([0, hi // 4, hi]), rows_hi=hi)
        hi = _log_int(rng, 1, max(2, min(16384, 131072 // B)))
        c.update(ctx_lo=rng.choice([0, hi // 8, hi]), ctx_hi=hi)
        return c
    if op == "commit":
        B = _log_int(rng, 1, 64)
        c.update(batch=B, nodes=_log_int(rng, 2, 64), ctx_lo=0, ctx_hi=_log_int(rng, 1, 128),
                 layers=rng.choice([1, 2, 8, 36]))
        return c
    B = _log_int(rng, 1, 32 if small else 128)
    N = _log_int(rng, 1, 64)
    tokens = 8192 if small else min(800_000, 150_000 * 256 // (N * max(heads // kv, 1)))
    hi = _log_int(rng, 16, max(17, min(32768, tokens // B)))
    c.update(batch=B, nodes=N, ctx_lo=max(0, hi // rng.choice([1, 2, 8, 64]) - rng.choice([0, 1])), ctx_hi=hi,
             ragged=rng.choice([False, True]))
    return c


# ------------------------------------------------------------------------------------- inputs
_TAGS = {t: i for i, t in enumerate(["kv", "rows", "lens", "pages", "tree", "logits", "misc"])}


def _gen(seed, tag):
    g = torch.Generator(device=_DEV)
    g.manual_seed(seed * 1013 + _TAGS[tag])
    return g


def _rng(seed, tag):
    return np.random.default_rng([int(seed), _TAGS[tag]])


def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _normal(g, *shape, dtype=torch.float32):
    return torch.empty(shape, dtype=dtype, device=_DEV).normal_(generator=g)


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(_DEV)


def _spread(n, lo, hi, seed, tag):
    """n whole numbers spread evenly over lo..hi, in a shuffled order: the same total for every seed."""
    v = lo + ((hi - lo + 1) * (2 * np.arange(n) + 1)) // (2 * n)
    return _rng(seed, tag).permutation(v)


def _trees(B, N, seed):
    """Draft trees as a head grows them: node 0 is the pending token, later nodes extend the newest
    node or any earlier one.  Returns parents, depths [B][N] and ancestor masks (bit j: node j, the
    node itself included)."""
    r = _rng(seed, "tree")
    parents = np.full((B, N), -1, np.int32)
    depths = np.zeros((B, N), np.int32)
    masks = np.ones((B, N), np.uint64)
    rows = np.arange(B)
    for i in range(1, N):
        p = np.where(r.random(B) < 0.3, i - 1, (i * r.random(B) ** 2).astype(np.int64))
        parents[:, i] = p
        depths[:, i] = depths[rows, p] + 1
        masks[:, i] = masks[rows, p] | np.uint64(1 << i)
    return parents, depths, masks


def _walks(parents, vocab, seed):
    """Tokens of the nodes, and the target's token after each node: at three of four nodes with
    children one of theirs."""
    B, N = parents.shape
    r = _rng(seed, "misc")
    tokens = r.integers(0, vocab, (B, N)).astype(np.int32)
    nxt = r.integers(0, vocab, (B, N)).astype(np.int32)
    for i in range(1, N):
        take = r.random(B) < 0.75
        p = parents[:, i]
        nxt[np.arange(B)[take], p[take]] = tokens[take, i]
    return tokens, nxt


def _cache(c, seed, layers, lens, extra):
    """A paged cache of N(0, 1) entries: pools [layers][pages][kv_heads * page * dim], a block table
    dealt from a shuffled pool, committed lengths."""
    need = (lens + extra + c["page"] - 1) // c["page"]
    need = np.maximum(need, 1)
    perm = _rng(seed, "pages").permutation(int(need.sum()))
    width = -(-(int(lens.max()) + int(np.max(extra))) // c["page"])       # room for the longest and the most rows
    table = np.full((len(lens), max(1, width)), -1, np.int32)
    ends = np.cumsum(need)
    for b, n in enumerate(need):
        table[b, :n] = perm[ends[b] - n:ends[b]]
    g = _gen(seed, "kv")
    shape = (layers, int(need.sum()), c["kv_heads"] * c["page"] * c["dim"])
    s = SimpleNamespace(k=_normal(g, *shape, dtype=_dtype(c)), v=_normal(g, *shape, dtype=_dtype(c)),
                        table=_i32(table), lens=_i32(lens), max_ctx=int(lens.max()))
    if own:
        from paper_2609_16648_amd import gm

        s.cfg = gm.model_config(_shape(c, layers))
        s.handle = gm.PagedCache(_shape(c, layers), layers, lens, lens + extra, page_size=c["page"], table=table,
                                 pools=(s.k, s.v))
        s.lens = s.handle.seq_lens
    return s


def _shape(c, layers):
    return SimpleNamespace(n_layers=layers, hidden=2560, n_heads=c["heads"], n_kv_heads=c["kv_heads"],
                           head_dim=c["dim"], ffn=9728, vocab=151936, rope_base=ROPE_BASE, rms_eps=EPS,
                           dtype=c["dtype"], qk_norm=bool(c.get("norm")), tie_embed=False)


def _spiky(g, rows, V):
    """Logits as a language model's at T = 1: a broad floor and sixteen likely ids falling off by
    about 1.2 each (the first holds about half of the mass).  Returns (logits, likely ids)."""
    z = _normal(g, rows, V).mul_(1.5)
    ids = torch.randint(0, V, (rows, 16), generator=g, device=_DEV)
    z.scatter_(1, ids, 16.0 - 1.2 * torch.arange(16, device=_DEV) + _normal(g, rows, 16).mul_(0.5))
    return z, ids


def prepare(case, seed):
    c = dict(case)
    op = c["op"]
    s = SimpleNamespace(c=c)
    if op == "append":
        B = c["batch"]
        lens = _spread(B, c["ctx_lo"], c["ctx_hi"], seed, "lens")
        n = np.full(B, c["nodes"]) if c["nodes"] else _spread(B, c["rows_lo"], c["rows_hi"], seed, "rows")
        T = int(n.sum())
        s.__dict__.update(_cache(c, seed, 1, lens, n).__dict__)
        g = _gen(seed, "rows")
        width = (c["heads"] + 2 * c["kv_heads"]) * c["dim"]
        qkv = _normal(g, T, width, dtype=_dtype(c))         # the rows of one projection
        a, b = c["heads"] * c["dim"], (c["heads"] + c["kv_heads"]) * c["dim"]
        s.q, s.kn, s.vn = (t.unflatten(1, (-1, c["dim"])) for t in (qkv[:, :a], qkv[:, a:b], qkv[:, b:]))
        s.q = s.q if c["q"] else None
        s.q_out = torch.empty((T, c["heads"], c["dim"]), dtype=_dtype(c), device=_DEV) if c["q"] else None
        s.max_rows = int(n.max())
        s.row_start = _i32(np.concatenate([[0], np.cumsum(n)])) if not c["nodes"] else None
        s.offsets = _i32(_trees(B, c["nodes"], seed)[1].reshape(-1)) if c["nodes"] else None
        s.q_norm, s.k_norm = ((1 + 0.1 * _normal(g, c["dim"])).to(_dtype(c)) if c["norm"] else None for _ in range(2))
    elif op == "attention":
        B, N = c["batch"], c["nodes"]
        lens = _spread(B, c["ctx_lo"], c["ctx_hi"], seed, "lens")
        s.__dict__.update(_cache(c, seed, 1, lens, N).__dict__)
        s.q = _normal(_gen(seed, "rows"), B, N, c["heads"], c["dim"], dtype=_dtype(c))
        s.out = torch.empty_like(s.q)
        s.masks = torch.from_numpy(_trees(B, N, seed)[2].view(np.int64)).to(_DEV)
        s.n_nodes = _i32(_rng(seed, "misc").integers(1, N + 1, B)) if c["ragged"] else None
    elif op == "commit":
        B, N = c["batch"], c["nodes"]
        lens = _spread(B, c["ctx_lo"], c["ctx_hi"], seed, "lens")
        s.__dict__.update(_cache(c, seed, c["layers"], lens, N).__dict__)
        s.lens0 = s.lens.clone()
        parents = _trees(B, N, seed)[0]
        tokens, nxt = _walks(parents, 151936, seed)
        s.parents, s.tokens, s.nxt = _i32(parents), _i32(tokens), _i32(nxt)
        s.path, s.out_tokens = (torch.empty((B, N), dtype=torch.int32, device=_DEV) for _ in range(2))
        s.n_accept = torch.empty(B, dtype=torch.int32, device=_DEV)
    else:
        M, V = c["rows"], c["vocab"]
        g = _gen(seed, "logits")
        z, likely = _spiky(g, M, V)
        if c.get("masked"):       # constrained decoding: two ids of three are not allowed
            at = z.gather(1, likely)
            z.masked_fill_(torch.arange(V, device=_DEV)[None, :] % 3 != torch.arange(M, device=_DEV)[:, None] % 3,
                           -math.inf)
            z.scatter_(1, likely, at)
        s.z = z.to(_dtype(c))
        pick = torch.randint(0, 8, (M, 1), generator=g, device=_DEV)
        s.ids = likely.gather(1, pick)[:, 0].to(torch.int32)
        s.ids[torch.rand(M, generator=g, device=_DEV) < 0.05] = -1     # padding
        f32 = lambda *shape: torch.empty(shape, dtype=torch.float32, device=_DEV)  # noqa: E731
        if op == "logprobs":
            k = c["topk"]
            s.logp, s.ent, s.stats = f32(M), f32(M), f32(M, 2)
            s.top_logp = f32(M, k) if k else None
            s.top_ids = torch.empty((M, k), dtype=torch.int32, device=_DEV) if k else None
        else:
            s.stats, s.ent = _row_stats(s.z, c["temperature"])
            s.g_logp = _normal(g, M).div_(M)
            s.g_ent = _normal(g, M).mul_(0.01 / M) if c["entropy"] else None
            s.grad = torch.empty_like(s.z)
    if own:
        from paper_2609_16648_amd import gm

        s.ws = gm.Workspace()
    return s


def _row_stats(z, T):
    """What the forward pass leaves for the gradient: (row max, sum of exp((z - max) / T)) and the entropy."""
    st = torch.empty((z.shape[0], 2), dtype=torch.float32, device=_DEV)
    ent = torch.empty(z.shape[0], dtype=torch.float32, device=_DEV)
    for r in range(0, z.shape[0], 512):
        x = z[r:r + 512].double()
        m = x.amax(1, keepdim=True)
        d = (x - m) / T
        e = d.exp()
        S = e.sum(1)
        st[r:r + 512, 0], st[r:r + 512, 1] = m[:, 0], S
        ent[r:r + 512] = S.log() - (e * d).sum(1) / S
    return st, ent


# ------------------------------------------------------------------------------------- the passes
def run(s):
    op = s.c["op"]
    return {"append": _append, "attention": _attention, "commit": _commit, "logprobs": _logprobs,
            "logprobs_grad": _logprobs_grad}[op](s)


def _append(s):
    if own:
        from paper_2609_16648_amd import gm

        gm.kv_append(s.cfg, s.handle, 0, s.kn, s.vn, q=s.q, q_out=s.q_out, row_start=s.row_start, offsets=s.offsets,
                     q_norm=s.q_norm, k_norm=s.k_norm, max_rows=s.max_rows)
    else:
        _plain_append(s)
    return {"q": s.q_out, "k": s.k, "v": s.v}


def _attention(s):
    if own:
        from paper_2609_16648_amd import gm

        gm.tree_attention(s.cfg, s.handle, 0, s.q, s.masks, s.out, s.ws, n_nodes=s.n_nodes)
        return s.out
    return _plain_attention(s)


def _commit(s):
    s.lens.copy_(s.lens0)
    if own:
        from paper_2609_16648_amd import gm

        gm.tree_accept(s.parents, s.tokens, s.nxt, s.path, s.n_accept, s.out_tokens)
        gm.tree_commit(s.cfg, s.handle, s.path, s.n_accept)
    else:
        _plain_commit(s)
    return {"path": s.path, "n_accept": s.n_accept, "out_tokens": s.out_tokens, "lens": s.lens, "k": s.k, "v": s.v}


def _logprobs(s):
    if own:
        from paper_2609_16648_amd import gm

        gm.token_logprobs(s.z, s.ids, s.ws, logp=s.logp, entropy=s.ent, top_logp=s.top_logp, top_ids=s.top_ids,
                          stats=s.stats, temperature=s.c["temperature"])
        return {"logp": s.logp, "entropy": s.ent, "stats": s.stats, "top_logp": s.top_logp, "top_ids": s.top_ids}
    return _plain_logprobs(s)


def _logprobs_grad(s):
    if own:
        from paper_2609_16648_amd import gm

        gm.token_logprobs_grad(s.z, s.ids, s.stats, s.g_logp, s.grad, entropy=s.ent, g_entropy=s.g_ent,
                               temperature=s.c["temperature"])
        return s.grad
    return _plain_logprobs_grad(s)


# ---- plain forms
def _tile_index(D, which):
    """Element of token t and channel c in a tile of 16 tokens, [16][D]."""
    t = torch.arange(16, device=_DEV)[:, None]
    ch = torch.arange(D, device=_DEV)[None, :]
    if which == "k":
        return ch // 32 * 512 + ch % 32 // 8 * 128 + t * 8 + ch % 8
    return ch // 32 * 512 + t // 4 * 128 + ch % 16 * 8 + ch // 16 % 2 * 4 + t % 4


def _slot_index(s, seq, slot, which):
    """Element index into one layer's pool of (sequence, slot) for every KV head and channel: [..., kv_heads, dim]."""
    c = s.c
    page = s.table[seq, slot // c["page"]].long()
    off = slot % c["page"]
    head = torch.arange(c["kv_heads"], device=_DEV)
    base = (page[..., None] * c["kv_heads"] + head) * (c["page"] * c["dim"]) + (off // 16 * 16 * c["dim"])[..., None]
    return base[..., None] + _tile_index(c["dim"], which)[off % 16][..., None, :]


def _plain_rotate(x, pos, norm):
    x = x.float()
    D = x.shape[-1]
    if norm is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * norm.float()
    freq = ROPE_BASE ** (-2.0 * torch.arange(D // 2, device=_DEV, dtype=torch.float64) / D)
    ang = pos.double()[:, None] * freq
    cs, sn = ang.cos().float()[:, None, :], ang.sin().float()[:, None, :]
    a, b = x[..., :D // 2], x[..., D // 2:]
    return torch.cat([a * cs - b * sn, b * cs + a * sn], -1)


def _plain_append(s):
    T = s.kn.shape[0]
    r = torch.arange(T, device=_DEV)
    if s.row_start is None:
        n = T // s.lens.shape[0]
        seq, i = r // n, r % n
    else:
        seq = torch.searchsorted(s.row_start[1:].long(), r, right=True)
        i = r - s.row_start[seq]
    slot = s.lens[seq] + i
    pos = s.lens[seq] + (s.offsets if s.offsets is not None else i)
    if s.q is not None:
        s.q_out.copy_(_plain_rotate(s.q, pos, s.q_norm))
    s.k.view(-1)[_slot_index(s, seq, slot.long(), "k")] = _plain_rotate(s.kn, pos, s.k_norm).to(s.k.dtype)
    s.v.view(-1)[_slot_index(s, seq, slot.long(), "v")] = s.vn


def _plain_attention(s):
    c = s.c
    B, N, D, kv = c["batch"], c["nodes"], c["dim"], c["kv_heads"]
    G, P = c["heads"] // kv, s.table.shape[1]
    pages = s.table.clamp(min=0).long()
    k = s.k[0][pages].view(B, P, kv, c["page"] // 16, D // 32, 4, 16, 8).permute(0, 2, 1, 3, 6, 4, 5, 7)
    v = s.v[0][pages].view(B, P, kv, c["page"] // 16, D // 32, 4, 16, 2, 4).permute(0, 2, 1, 3, 5, 8, 4, 7, 6)
    k, v = (t.reshape(B, kv, P * c["page"], D).float() for t in (k, v))
    q = s.q.float().view(B, N, kv, G, D).permute(0, 2, 3, 1, 4).reshape(B, kv, G * N, D)
    x = torch.matmul(q, k.transpose(-1, -2)) * (1.0 / math.sqrt(D))
    n = s.n_nodes[:, None, None] if s.n_nodes is not None else N
    t = torch.arange(P * c["page"], device=_DEV)[None, None, :] - s.lens[:, None, None]
    vis = (t < 0) | ((s.masks[:, :, None] >> t.clamp(0, 63)) & 1).bool() & (t >= 0) & (t < N) & (t < n)
    vis = vis & (torch.arange(N, device=_DEV)[None, :, None] < n)
    x = x.view(B, kv, G, N, -1).masked_fill_(~vis[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    p = x.sub_(m.masked_fill(m == -math.inf, 0)).exp_()
    den = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, kv, G * N, -1), v).view(B, kv, G, N, D) / den.masked_fill(den == 0, 1)
    return o.permute(0, 3, 1, 2, 4).reshape(B, N, c["heads"], D).to(s.q.dtype)


def _plain_commit(s):
    B, N = s.parents.shape
    node = torch.arange(N, device=_DEV)
    par = s.parents.long()
    up = (par[:, :, None] == node).double() + torch.eye(N, dtype=torch.float64, device=_DEV)
    anc = torch.linalg.matrix_power(up, N) > 0                    # [b][i][j]: j is i or above it
    match = s.tokens == torch.gather(s.nxt, 1, par.clamp(min=0))
    twin = (par[:, :, None] == par[:, None, :]) & (s.tokens[:, :, None] == s.tokens[:, None, :])
    match &= ~(twin & (node[None, :] < node[:, None])).any(-1) & (par >= 0)
    match[:, 0] = True
    acc = (match[:, None, :] | ~anc).all(-1) & anc[:, :, 0]
    n = acc.sum(-1)
    order = torch.where(acc, node, N).sort(-1).values
    live = node < n[:, None]
    s.path.copy_(torch.where(live, order, -1))
    s.n_accept.copy_(n - 1)
    last = torch.gather(order, 1, n[:, None] - 1)
    nxt = torch.cat([order[:, 1:], order[:, :1]], 1).clamp(max=N - 1)
    out = torch.where(node < n[:, None] - 1, torch.gather(s.tokens, 1, nxt), torch.gather(s.nxt, 1, last))
    s.out_tokens.copy_(torch.where(live, out, -1))
    seq = torch.arange(B, device=_DEV)[:, None].expand(B, N)
    src = s.lens.long()[:, None] + torch.where(live, order, node)
    dst = s.lens.long()[:, None] + node
    layers = s.k.shape[0]
    for pool, which in ((s.k.view(layers, -1), "k"), (s.v.view(layers, -1), "v")):
        i, j = (_slot_index(s, seq, x, which).view(-1) for x in (src, dst))
        pool[:, j] = pool[:, i]
    s.lens.add_(n.to(torch.int32))


def _plain_logprobs(s):
    T, k = s.c["temperature"], s.c["topk"]
    z = s.z.float()
    m = z.amax(1, keepdim=True)
    d = (z - m) / T
    e = d.exp()
    S = e.sum(1, dtype=torch.float64)
    W = torch.where(e > 0, e * d, 0.0).sum(1, dtype=torch.float64)
    at = torch.gather(d, 1, s.ids.long().clamp(min=0)[:, None])[:, 0]
    log_s = S.log()
    out = {"logp": torch.where(s.ids < 0, 0.0, at - log_s).float(), "entropy": (log_s - W / S).float(),
           "stats": torch.stack([m[:, 0], S.float()], 1), "top_logp": None, "top_ids": None}
    if k:
        order = d.sort(dim=1, descending=True, stable=True)
        out["top_logp"] = (order.values[:, :k] - log_s[:, None]).float()
        out["top_ids"] = order.indices[:, :k].to(torch.int32)
    return out


def _plain_logprobs_grad(s):
    T = s.c["temperature"]
    d = (s.z.float() - s.stats[:, :1]) / T
    S = s.stats[:, 1:]
    p = d.exp() / S
    g = torch.where(s.ids < 0, 0.0, s.g_logp)[:, None]
    if s.g_ent is not None:
        w = p * (g + s.g_ent[:, None] * (torch.where(p > 0, d, 0.0) - S.log() + s.ent[:, None]))
    else:
        w = p * g
    return w.neg_().scatter_add_(1, s.ids.long().clamp(min=0)[:, None], g).div_(T).to(s.z.dtype)


# ------------------------------------------------------------------------------------- work
def work(case):
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    if c["op"] in ("logprobs", "logprobs_grad"):
        n = c["rows"] * c["vocab"]
        if c["op"] == "logprobs":
            return dict(bytes=n * e + c["rows"] * (24 + 8 * c["topk"]), flops=5 * n)
        return dict(bytes=2 * n * e + c["rows"] * 24, flops=6 * n)
    B, D, kv = c["batch"], c["dim"], c["kv_heads"]
    if c["op"] == "append":
        T = B * c["nodes"] if c["nodes"] else int(_spread(B, c["rows_lo"], c["rows_hi"], 0, "rows").sum())
        q = c["heads"] if c["q"] else 0
        return dict(bytes=max(1, T) * (q + 2 * kv) * D * e * 2 + B * 8, flops=T * (q + kv) * D * 8)
    if c["op"] == "commit":
        _, moved = _moves(c)
        return dict(bytes=c["layers"] * moved * 2 * kv * D * e * 2 + B * c["nodes"] * 20, flops=B * c["nodes"])
    lens = _spread(B, c["ctx_lo"], c["ctx_hi"], 0, "lens")
    N = c["nodes"] / 2 if c["ragged"] else c["nodes"]      # (a ragged batch's trees hold half of the nodes)
    return dict(bytes=int((lens + N).sum()) * 2 * kv * D * e + 2 * B * N * c["heads"] * D * e,
                flops=4 * c["heads"] * D * N * int((lens + N / 4).sum()))


def _moves(c):
    """Accepted nodes of a batch and the entries among them that change place, for one seed's trees."""
    parents = _trees(c["batch"], c["nodes"], 0)[0]
    tokens, nxt = _walks(parents, 151936, 0)
    accepted = moved = 0
    for b in range(c["batch"]):
        cur, at = 0, 0
        for i in range(1, c["nodes"]):
            if parents[b, i] == cur and tokens[b, i] == nxt[b, cur]:
                cur, at = i, at + 1
                moved += i != at
        accepted += at
    return accepted, max(1, moved)


# ------------------------------------------------------------------------------------- float64
def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "append":
        return _exact_append(s)
    if op == "attention":
        return _exact_attention(s)
    if op == "commit":
        return None               # whole numbers and moved values
    return _exact_logits(s)


def _exact_entries(c, table, lens_b, which, n):
    """Flat pool indices [n][kv_heads][dim] of the first n slots of one sequence (numpy)."""
    t = np.arange(n)
    ch = np.arange(c["dim"])
    page = np.asarray(table)[t // c["page"]].astype(np.int64)
    tok = t % 16
    if which == "k":
        el = (ch >> 5) * 512 + ((ch >> 3) & 3) * 128 + tok[:, None] * 8 + (ch & 7)
    else:
        el = (ch >> 5) * 512 + (tok[:, None] >> 2) * 128 + (ch & 15) * 8 + ((ch >> 4) & 1) * 4 + (tok[:, None] & 3)
    block = page[:, None] * c["kv_heads"] + np.arange(c["kv_heads"])
    start = block * (c["page"] * c["dim"]) + (t % c["page"] - tok)[:, None] * c["dim"]
    return torch.from_numpy(start[:, :, None] + el[:, None, :]).to(_DEV)


def _exact_append(s):
    c = s.c
    lens, table = s.lens.cpu().numpy(), s.table.cpu().numpy()
    D, T = c["dim"], s.kn.shape[0]
    starts = s.row_start.cpu().numpy() if s.row_start is not None else np.arange(c["batch"] + 1) * c["nodes"]
    k, v = s.k.double().view(-1), s.v.double().view(-1)
    q = torch.zeros((T, c["heads"], D), dtype=torch.float64, device=_DEV) if s.q is not None else None

    def turn(x, pos, w):
        x = x.double()
        if w is not None:
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w.double()
        half = torch.arange(D // 2, device=_DEV, dtype=torch.float64)
        rot = torch.polar(torch.ones((), dtype=torch.float64, device=_DEV),
                          pos.double()[:, None] * torch.exp(half * (-2.0 / D * math.log(ROPE_BASE))))
        y = torch.complex(x[..., :D // 2].contiguous(), x[..., D // 2:].contiguous()) * rot[:, None, :]
        return torch.cat([y.real, y.imag], -1)

    for b in range(c["batch"]):
        lo, hi = int(starts[b]), int(starts[b + 1])
        if lo == hi:
            continue
        m, n = int(lens[b]), hi - lo
        off = s.offsets[lo:hi].double() if s.offsets is not None else torch.arange(n, device=_DEV)
        if q is not None:
            q[lo:hi] = turn(s.q[lo:hi], m + off, s.q_norm)
        k[_exact_entries(c, table[b], m, "k", m + n)[m:]] = turn(s.kn[lo:hi], m + off, s.k_norm)
        v[_exact_entries(c, table[b], m, "v", m + n)[m:]] = s.vn[lo:hi].double()
    return {"q": q, "k": k.view(s.k.shape), "v": v.view(s.v.shape)}


def _exact_attention(s):
    c = s.c
    lens, table = s.lens.cpu().numpy(), s.table.cpu().numpy()
    masks = s.masks.cpu().numpy().view(np.uint64)
    N, G = c["nodes"], c["heads"] // c["kv_heads"]
    out = torch.zeros(s.q.shape, dtype=torch.float64, device=_DEV)
    for b in range(c["batch"]):
        m = int(lens[b])
        n = int(s.n_nodes[b]) if s.n_nodes is not None else N
        L = m + n
        k = s.k.view(-1)[_exact_entries(c, table[b], m, "k", L)].double()
        v = s.v.view(-1)[_exact_entries(c, table[b], m, "v", L)].double()
        see = np.ones((n, L), bool)
        see[:, m:] = (masks[b, :n, None] >> np.arange(n, dtype=np.uint64)) & np.uint64(1)
        see = torch.from_numpy(see).to(_DEV)
        for h in range(c["kv_heads"]):
            q = s.q[b, :n, h * G:(h + 1) * G].double().transpose(0, 1)                 # [G][n][D]
            x = q.reshape(G * n, -1).mm(k[:, h].t().contiguous()).view(G, n, L) / math.sqrt(c["dim"])
            w = torch.softmax(x.masked_fill(~see, -math.inf), -1)
            out[b, :n, h * G:(h + 1) * G] = w.view(G * n, L).mm(v[:, h].contiguous()).view(G, n, -1).transpose(0, 1)
    return out


def _exact_logits(s):
    c = s.c
    M, T = c["rows"], c["temperature"]
    grads, parts = [], {n: [] for n in ("logp", "entropy", "stats", "top_logp", "top_ids")}
    for r in range(0, M, 256):
        z = s.z[r:r + 256].double()
        ids = s.ids[r:r + 256].long()
        lp = torch.log_softmax(z / T, 1)
        p = lp.exp()
        H = -torch.where(p > 0, p * lp, 0.0).sum(1)
        if c["op"] == "logprobs":
            at = lp.gather(1, ids.clamp(min=0)[:, None])[:, 0]
            m = z.amax(1)
            parts["logp"].append(torch.where(ids < 0, 0.0, at))
            parts["entropy"].append(H)
            parts["stats"].append(torch.stack([m, (torch.logsumexp(z / T, 1) - m / T).exp()], 1))
            if c["topk"]:
                parts["top_logp"].append(lp.topk(c["topk"], 1).values)
        else:
            g = torch.where(ids < 0, 0.0, s.g_logp[r:r + 256].double())[:, None]
            y = -p * g
            y[torch.arange(len(ids), device=_DEV), ids.clamp(min=0)] += g[:, 0]
            if s.g_ent is not None:
                y -= s.g_ent[r:r + 256].double()[:, None] * p * (torch.where(p > 0, lp, 0.0) + H[:, None])
            grads.append(y / T)
    if c["op"] == "logprobs_grad":
        return torch.cat(grads)
    return {n: torch.cat(v) if v else None for n, v in parts.items()}
