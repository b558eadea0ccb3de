"""Draft trees on the GPU against float64: the append, the masks, the nodes' attention, the walk, the
commit, and a whole step of them.

Tolerances (u = 2^-24, half a float32 step; bf16 outputs round once by at most 2^-8 of the value):
* append: the sum of squares of D channels is a chain of at most D / 4 + 2 additions (its error halves in the
  root), the angle is off by 2^-25 turns (2 pi / 2 u), sine and cosine by 2 u, products, quotient and sums
  by 6 u: at most (D / 8 + 13) u of |y_c| + |y_{c + D/2}|; 64 u is taken.
* attention: a score is a sum of D products, off by at most D u sum |q_c k_c| / sqrt(D) =: D u s_abs; weights
  are off by twice that and by 2^-16 where they are carried as two bf16 parts; the sums over L tokens in
  float32 add at most (L / 16 + 64) u: times sum p |v| =: mag.
"""
import dataclasses

import numpy as np
import pytest
import torch

import synth
from helpers import need_gpu, t32, i32
from oracle import tree as otree
from paper_2609_16648_amd import gm, layout

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF16 = synth.QWEN3_4B_LAYER
F32 = synth.ModelShape(1, 256, 4, 4, 64, 1024, 1024, dtype="f32")
SHAPES = {
    "qwen": BF16,
    "mqa16": dataclasses.replace(BF16, n_heads=16, n_kv_heads=1),
    "g7": dataclasses.replace(BF16, n_heads=28, n_kv_heads=4),
    "mha": dataclasses.replace(BF16, n_heads=6, n_kv_heads=6),
    "g64": dataclasses.replace(BF16, n_heads=64, n_kv_heads=1),
    "f32": F32,
    "f32_g4_d128": synth.ModelShape(1, 512, 8, 2, 128, 1024, 1024, dtype="f32"),
}


def _half(shape):
    return 2.0 ** -8 if shape.dtype == "bf16" else U


def _rand(shape, *size, seed=0, scale=1.0):
    r = np.random.default_rng([seed, len(size)])
    return synth.quantise((r.standard_normal(size) * scale).astype(np.float32), shape.dtype)


def _trees(B, N, seed, forest=False):
    r = np.random.default_rng(seed)
    p = np.full((B, N), -1, np.int32)
    for i in range(1, N):
        p[:, i] = np.where(r.random(B) < 0.3, i - 1, r.integers(-1 if forest else 0, i, B))
    return p


def _masks(parents, n_nodes=None):
    B, N = parents.shape
    n = [None] * B if n_nodes is None else n_nodes
    both = [otree.tree_masks(parents[b], n[b]) for b in range(B)]
    return np.stack([m for m, _ in both]), np.stack([d for _, d in both]).astype(np.int32)


def _bits(masks):
    """bool [B, N, N] -> int64 [B, N] on the device."""
    w = (masks.astype(np.uint64) << np.arange(masks.shape[-1], dtype=np.uint64)).sum(-1, dtype=np.uint64)
    return torch.from_numpy(w.view(np.int64)).cuda()


def _err():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


def _entries(cache, shape, lens, n, seed):
    """Fills the first lens + n positions of every sequence; returns [K], [V] per sequence (float32)."""
    ks, vs = [], []
    for b, m in enumerate(lens):
        k, v = (_rand(shape, m + n, shape.n_kv_heads, shape.head_dim, seed=seed + 2 * b + i) for i in range(2))
        if m + n:
            cache.write(0, b, np.arange(m + n), k, v)
        ks.append(k)
        vs.append(v)
    return ks, vs


# ------------------------------------------------------------------------------------- append
APPEND = [
    # shape, committed lengths, rows per sequence (None: equal), page, norm, packed rows, offsets
    ("qwen", [0, 5, 16, 31], [1, 16, 3, 40], 16, True, True, False),
    ("qwen", [4001], [8], 16, True, True, True),
    ("qwen", [7, 0, 100, 63, 64, 65], [0, 0, 17, 33, 0, 1], 32, False, False, True),
    ("qwen", [10, 20, 30], None, 16, True, False, False),
    ("g7", [0], [700], 64, True, True, False),
    ("mha", [3, 9], [15, 21], 16, False, True, True),
    ("f32", [0, 13, 130], [5, 64, 2], 16, True, True, False),
    ("f32_g4_d128", [33, 1], [31, 18], 32, True, False, True),
    ("f32", [2, 2], None, 16, False, True, True),
    ("mha", [7 * i % 50 for i in range(600)], [5 * i % 4 for i in range(600)], 16, False, True, True),
]


@pytest.mark.parametrize("name,lens,rows,page,norm,packed,with_off", APPEND)
def test_append(name, lens, rows, page, norm, packed, with_off):
    need_gpu()
    shape = dataclasses.replace(SHAPES[name], qk_norm=norm)
    B, D, kv, H = len(lens), shape.head_dim, shape.n_kv_heads, shape.n_heads
    even = rows is None
    n = np.full(B, 9) if even else np.array(rows)
    pad = 0 if even else 3                                  # rows behind the last sequence
    T = int(n.sum()) + pad
    starts = np.concatenate([[0], np.cumsum(n)])
    seed = int(n.sum()) + page
    r = np.random.default_rng(seed)
    W = (H + 2 * kv) * D
    x = _rand(shape, T, W, seed=seed, scale=2.0)
    dt = gm.torch_dtype(shape)
    if packed:       # column blocks of one projection, one element off 16-byte alignment
        buf = torch.empty(T * (W + 3) + 1, dtype=dt, device="cuda")
        full = buf[1:].view(T, W + 3)[:, :W]
        full.copy_(t32(x))
        q, k, v = (full[:, a:b].unflatten(1, (-1, D)) for a, b in
                   ((0, H * D), (H * D, (H + kv) * D), ((H + kv) * D, W)))
    else:
        q, k, v = (t32(x[:, a:b].reshape(T, -1, D), dt) for a, b in
                   ((0, H * D), (H * D, (H + kv) * D), ((H + kv) * D, W)))
    qn, kn = (_rand(shape, D, seed=seed + i) for i in (5, 6))
    off = r.integers(0, 30000, T).astype(np.int32) if with_off else None
    cap = np.full(B, max(lens) + n.max())
    cache = gm.PagedCache(shape, 1, lens, cap, page_size=page, seed=seed)
    for p in cache.k + cache.v:
        p.copy_(torch.randn(p.shape, device="cuda"))
    old_k, old_v = cache.k[0].clone(), cache.v[0].clone()
    q_out = torch.full((T, H, D), 7.0, dtype=dt, device="cuda")
    err = _err()
    gm.kv_append(gm.model_config(shape), cache, 0, k, v, q=q, q_out=q_out, row_start=None if even else i32(starts),
                 offsets=i32(off) if with_off else None, q_norm=t32(qn, dt) if norm else None,
                 k_norm=t32(kn, dt) if norm else None, max_rows=None if even else int(n.max()), dev_err=err)
    torch.cuda.synchronize()
    assert int(err.item()) == 0
    got_q = q_out.float().cpu().numpy()
    assert (got_q[starts[-1]:] == 7.0).all()
    xs = x.reshape(T, -1, D)
    for b in range(B):
        at = np.arange(starts[b], starts[b + 1])
        if not len(at):
            continue
        i = np.arange(len(at))
        pos = lens[b] + (off[at] if with_off else i)
        got_k, got_v = cache.read(0, b, lens[b] + i)
        for what, got, src, w in (("q", got_q[at], xs[at, :H], qn), ("k", got_k, xs[at, H:H + kv], kn)):
            want = otree.append_rows(src, pos, shape.rope_base, shape.rms_eps, w if norm else None)
            pair = np.abs(want) + np.abs(np.roll(want, D // 2, -1))
            bad = np.abs(got - want) > _half(shape) * np.abs(want) + 64 * U * pair
            assert not bad.any(), (what, b, np.abs(got - want).max())
        assert np.array_equal(got_v, xs[at, H + kv:])
        # nothing else moved: with the old entries put back, the pools are the old ones
    keep = gm.PagedCache(shape, 1, lens, cap, page_size=page, seed=seed)
    keep.k[0].copy_(old_k)
    keep.v[0].copy_(old_v)
    for b in range(B):
        if n[b]:
            i = lens[b] + np.arange(n[b])
            cache.write(0, b, i, *keep.read(0, b, i))
    assert torch.equal(cache.k[0], old_k) and torch.equal(cache.v[0], old_v)


def test_append_in_place_and_keys_alone():
    need_gpu()
    T, B = 24, 3
    cfg, dt = gm.model_config(BF16), torch.bfloat16
    mk = lambda h, s: t32(_rand(BF16, T, h, 128, seed=s), dt)  # noqa: E731
    k, v, q = mk(8, 1), mk(8, 2), mk(32, 3)
    a, b = (gm.PagedCache(BF16, 1, [3, 50, 7], [30, 60, 30], seed=4) for _ in range(2))
    out = torch.empty_like(q)
    gm.kv_append(cfg, a, 0, k, v, q=q, q_out=out)
    gm.kv_append(cfg, b, 0, k, v, q=q, q_out=q)
    assert torch.equal(q, out) and torch.equal(a.k[0], b.k[0])
    c = gm.PagedCache(BF16, 1, [3, 50, 7], [30, 60, 30], seed=4)
    gm.kv_append(cfg, c, 0, k, v)
    assert torch.equal(a.k[0], c.k[0]) and torch.equal(a.v[0], c.v[0]) and B * 8 == T


def test_append_far_positions_and_bad_pages():
    """Offsets of two million positions; a page outside the pool is reported and only its rows are left out."""
    need_gpu()
    shape = F32
    cache = gm.PagedCache(shape, 1, [10, 10], [60, 60], seed=3)
    cache.block_table[0, 1] = cache.num_pages          # slots 16..31 of sequence 0
    cache.block_table[1, 2] = -7                        # slots 32..47 of sequence 1
    T = 60
    k, v = (_rand(shape, T, 4, 64, seed=s) for s in (1, 2))
    off = (2_000_000 + np.arange(T)).astype(np.int32)
    err = _err()
    gm.kv_append(gm.model_config(shape), cache, 0, t32(k), t32(v), offsets=i32(off), dev_err=err)
    assert int(err.item()) == gm.GM_DEVERR_PAGE
    for b, lost in ((0, range(16, 32)), (1, range(32, 40))):
        live = [s for s in range(10, 40) if s not in lost]
        got_k, got_v = cache.read(0, b, live)
        at = 30 * b + np.array(live) - 10
        want = otree.append_rows(k[at], 10 + off[at], shape.rope_base, shape.rms_eps)
        pair = np.abs(want) + np.abs(np.roll(want, 32, -1))
        assert (np.abs(got_k - want) <= U * np.abs(want) + 64 * U * pair).all() and np.array_equal(got_v, v[at])
    written = sum((cache.k[0] != 0).any(-1).sum().item() for _ in range(1))
    assert written <= 2 * 4                            # pages of the slots 10..39 but the two lost ones


# ------------------------------------------------------------------------------------- masks
@pytest.mark.parametrize("B,N,ragged", [(1, 1, False), (5, 64, False), (9, 33, True), (300, 7, True)])
def test_masks(B, N, ragged):
    need_gpu()
    parents = _trees(B, N, B + N, forest=True)
    n = np.random.default_rng(N).integers(-2, N + 3, B).astype(np.int32) if ragged else None
    masks, depths, err = torch.zeros((B, N), dtype=torch.int64, device="cuda"), i32(np.full((B, N), 9)), _err()
    gm.tree_masks(i32(parents), masks, depths, i32(n) if ragged else None, err)
    want_m, want_d = _masks(parents, n)
    assert int(err.item()) == 0
    assert torch.equal(masks, _bits(want_m)) and np.array_equal(depths.cpu().numpy(), want_d)


def test_masks_report_bad_parents():
    need_gpu()
    parents = np.array([[-1, 0, 2, 2, 1]], np.int32)     # node 2 is its own parent
    masks, depths, err = torch.zeros((1, 5), dtype=torch.int64, device="cuda"), i32(np.zeros((1, 5))), _err()
    gm.tree_masks(i32(parents), masks, depths, None, err)
    assert int(err.item()) == gm.GM_DEVERR_TREE
    assert masks.cpu().tolist() == [[1, 3, 4, 12, 19]] and depths.cpu().tolist() == [[0, 1, 0, 1, 2]]
    err.zero_()
    parents[0, 2], parents[0, 3] = 0, 99                 # behind the last node nothing is looked at
    gm.tree_masks(i32(parents), masks, depths, i32([3]), err)
    assert int(err.item()) == 0 and masks.cpu().tolist() == [[1, 3, 5, 0, 0]]


# ------------------------------------------------------------------------------------- attention
def _check_attention(shape, lens, N, page, seed, n_nodes=None, masks=None, parts=2.0 ** -16):
    B, H, D = len(lens), shape.n_heads, shape.head_dim
    cache = gm.PagedCache(shape, 1, lens, np.array(lens) + N, page_size=page, seed=seed, fill="empty")
    for p in cache.k + cache.v:
        p.fill_(float("nan"))                            # slots behind the last node hold anything
    ks, vs = _entries(cache, shape, lens, N, seed)
    q = _rand(shape, B, N, H, D, seed=seed + 1)
    if masks is None:
        masks = _masks(_trees(B, N, seed))[0]
    dt = gm.torch_dtype(shape)
    out, err, ws = torch.full((B, N, H, D), 3.0, dtype=dt, device="cuda"), _err(), gm.Workspace()
    args = (gm.model_config(shape), cache, 0, t32(q, dt), _bits(masks), out, ws)
    gm.tree_attention(*args, n_nodes=i32(n_nodes) if n_nodes is not None else None, dev_err=err)
    torch.cuda.synchronize()
    assert int(err.item()) == 0
    got = out.float().cpu().numpy()
    for b in range(B):
        want, mag = otree.tree_attention(q[b], ks[b], vs[b], lens[b], masks[b],
                                         None if n_nodes is None else n_nodes[b])
        s_abs = np.abs(q[b]).max(0).sum(-1).max() * np.abs(ks[b]).max() / np.sqrt(D)
        tol = (2 * D * U * s_abs + parts + ((lens[b] + N) / 16 + 64) * U) * mag + _half(shape) * np.abs(want)
        over = np.abs(got[b] - want) - tol
        assert over.max() <= 0, (b, np.abs(got[b] - want).max(), over.max())
    gm.tree_attention(*args, n_nodes=i32(n_nodes) if n_nodes is not None else None, dev_err=err)
    assert np.array_equal(out.float().cpu().numpy(), got)        # the same call twice gives the same bits


ATTENTION = [
    ("qwen", [0, 1, 15, 16, 17, 40], 8, 16, None),
    ("qwen", [300, 7, 1000, 63], 16, 32, [16, 1, 0, 9]),
    ("qwen", [100, 5], 64, 16, [64, 37]),
    ("qwen", [33], 1, 16, None),
    ("qwen", [2049, 0], 33, 64, None),
    ("g7", [50, 129, 0], 9, 16, [3, 9, 9]),
    ("g7", [20], 64, 16, None),
    ("mha", [90, 31], 3, 16, None),
    ("mha", [14, 500], 64, 16, [64, 50]),
    ("mqa16", [77, 3], 5, 16, None),
    ("mqa16", [77, 3], 21, 16, [21, 20]),
    ("g64", [19], 7, 16, None),
    ("f32", [0, 5, 130], 7, 16, [7, 3, 0]),
    ("f32", [200], 64, 16, None),
    ("f32_g4_d128", [66, 0], 20, 32, [20, 19]),
]


@pytest.mark.parametrize("name,lens,N,page,n_nodes", ATTENTION)
def test_attention(name, lens, N, page, n_nodes):
    need_gpu()
    _check_attention(SHAPES[name], lens, N, page, len(lens) + N, n_nodes,
                     parts=0.0 if SHAPES[name].dtype == "f32" else 2.0 ** -16)


@pytest.mark.parametrize("name,N,B", [("mqa16", 9, 1100), ("mqa16", 5, 700), ("qwen", 9, 300), ("qwen", 2, 300)])
def test_attention_many_sequences(name, N, B):
    """More sequences than a workgroup has threads, one and two KV heads per workgroup, four, and small trees."""
    need_gpu()
    lens = np.random.default_rng(B).integers(0, 40, B).tolist()
    lens[255:258] = [17, 0, 16]
    _check_attention(SHAPES[name], lens, N, 16, B, parts=2.0 ** -16)


@pytest.mark.parametrize("heads,kv,N,lens,page", [
    (72, 24, 64, [9000, 8007, 100, 17900, 0, 9000, 42011], 64),      # 192 rows: one KV head per workgroup
    (72, 24, 33, [39000, 8007, 100, 77900, 52000], 16),              # 99 rows: two
    (42, 42, 40, [39000, 8007, 100, 50001], 16),                     # 40 rows: four
    (42, 42, 8, [9000, 8007, 100, 50001], 32),                       # a small tree
])
def test_attention_long_ranges(heads, kv, N, lens, page):
    """Ranges of many tiles per workgroup, over several of its windows; a few heads are compared."""
    need_gpu()
    shape = dataclasses.replace(BF16, n_heads=heads, n_kv_heads=kv)
    B, D, G, total = len(lens), 128, heads // kv, [m + N for m in lens]
    cache = gm.PagedCache(shape, 1, lens, total, page_size=page, seed=N, fill="empty")
    g = torch.Generator(device="cuda").manual_seed(N)
    for p in cache.k + cache.v:
        p.copy_(torch.randn(p.shape, generator=g, device="cuda", dtype=torch.bfloat16))
    q = _rand(shape, B, N, heads, D, seed=N + 1)
    masks = _masks(_trees(B, N, N))[0]
    out = torch.full((B, N, heads, D), 3.0, dtype=torch.bfloat16, device="cuda")
    gm.tree_attention(gm.model_config(shape), cache, 0, t32(q, torch.bfloat16), _bits(masks), out, gm.Workspace())
    for b in range(B):
        for h in (0, kv - 1):
            kvs = []
            for which in ("k", "v"):
                page_ids, elem = layout.element_index(np.arange(total[b]), cache.block_table_host[b], page, D, which)
                pool = cache._pool(0, which)[:, h]
                kvs.append(pool[torch.from_numpy(page_ids).cuda()[:, None], torch.from_numpy(elem).cuda()]
                           .float().cpu().numpy()[:, None])
            rows = slice(h * G, (h + 1) * G)
            k, v = (x[:, 0].astype(np.float64) for x in kvs)
            sc = np.einsum("ihd,td->iht", q[b][:, rows].astype(np.float64), k, optimize=True) / np.sqrt(D)
            sc[:, :, lens[b]:] = np.where(masks[b][:, None], sc[:, :, lens[b]:], -np.inf)
            p = np.exp(sc - sc.max(-1, keepdims=True))
            p /= p.sum(-1, keepdims=True)
            want, mag = p @ v, p @ np.abs(v)
            s_abs = np.abs(q[b][:, rows]).max((0, 1)).sum() * np.abs(kvs[0]).max() / np.sqrt(D)
            tol = (2 * D * U * s_abs + 2.0 ** -16 + (total[b] / 16 + 64) * U) * mag + 2.0 ** -8 * np.abs(want)
            over = np.abs(out[b][:, rows].float().cpu().numpy() - want) - tol
            assert over.max() <= 0, (b, h, over.max())


@pytest.mark.parametrize("name,N", [("qwen", 8), ("qwen", 40), ("f32", 6)])
def test_attention_any_mask(name, N):
    """Masks that are no tree's: rows that see nothing of the block, later nodes, everything."""
    need_gpu()
    B = 4
    masks = np.random.default_rng(N).random((B, N, N)) < 0.4
    masks[0, 0] = masks[1] = False                       # with no committed token the row is empty
    masks[2] = True
    _check_attention(SHAPES[name], [0, 0, 20, 100], N, 16, N, masks=masks,
                     parts=0.0 if name == "f32" else 2.0 ** -16)


@pytest.mark.parametrize("name,N", [("qwen", 8), ("qwen", 40), ("mha", 12), ("f32", 9)])
def test_attention_unseen_entries_do_not_reach_a_row(name, N):
    """A node's K or V of inf or NaN reaches its descendants and nobody else."""
    need_gpu()
    shape = SHAPES[name]
    lens, B = [21, 5], 2
    parents = np.stack([np.array([-1, 0] + [1] * (N - 2)), _trees(1, N, 3)[0]]).astype(np.int32)
    masks = _masks(parents)[0]
    q = _rand(shape, B, N, shape.n_heads, shape.head_dim, seed=5)
    dt = gm.torch_dtype(shape)
    outs = []
    for bad in (None, float("inf"), float("nan")):
        cache = gm.PagedCache(shape, 1, lens, np.array(lens) + N, seed=2)
        ks, vs = _entries(cache, shape, lens, N, 11)
        if bad is not None:
            for b in range(B):
                for node, kind in ((3, "v"), (5, "k")):
                    k, v = ks[b][lens[b] + node].copy(), vs[b][lens[b] + node].copy()
                    (v if kind == "v" else k)[..., 1::3] = bad
                    cache.write(0, b, [lens[b] + node], k[None], v[None])
        out = torch.empty((B, N, shape.n_heads, shape.head_dim), dtype=dt, device="cuda")
        gm.tree_attention(gm.model_config(shape), cache, 0, t32(q, dt), _bits(masks), out, gm.Workspace())
        outs.append(out.float().cpu().numpy())
    hit = masks[:, :, 3] | masks[:, :, 5]
    for o in outs[1:]:
        assert np.array_equal(o[~hit], outs[0][~hit])
        assert not np.isfinite(o[hit]).all()
    # the channels of V that hold nothing special are as before for a row that sees node 3 alone
    only = masks[:, :, 3] & ~masks[:, :, 5]
    keep = np.ones(shape.head_dim, bool)
    keep[1::3] = False
    assert only.any() and np.allclose(outs[1][only][..., keep], outs[0][only][..., keep], rtol=2.0 ** -7, atol=1e-6)
    assert not np.isfinite(outs[2][only][..., ~keep]).any()


@pytest.mark.parametrize("name,N", [("qwen", 8), ("qwen", 16), ("qwen", 40), ("g7", 64), ("mha", 12), ("f32", 9)])
@pytest.mark.parametrize("pos", [20, 15, 2])
def test_attention_committed_infinities_reach_every_row(name, N, pos):
    """V of a committed token that is inf in some channels (in the tile of the first nodes, or before it)."""
    need_gpu()
    shape, lens = SHAPES[name], [21]
    q = _rand(shape, 1, N, shape.n_heads, shape.head_dim, seed=5, scale=0.25)
    masks = _masks(_trees(1, N, 3))[0]
    dt = gm.torch_dtype(shape)
    outs = []
    for bad in (False, True):
        cache = gm.PagedCache(shape, 1, lens, [21 + N], seed=2)
        ks, vs = _entries(cache, shape, lens, N, 11)
        if bad:
            v = vs[0][pos].copy()
            v[..., 1::3] = np.inf
            cache.write(0, 0, [pos], ks[0][pos][None], v[None])
        out = torch.empty((1, N, shape.n_heads, shape.head_dim), dtype=dt, device="cuda")
        gm.tree_attention(gm.model_config(shape), cache, 0, t32(q, dt), _bits(masks), out, gm.Workspace())
        outs.append(out.float().cpu().numpy())
    assert not np.isfinite(outs[1][..., 1::3]).any()
    for c in (0, 2):
        assert np.allclose(outs[1][..., c::3], outs[0][..., c::3], rtol=2.0 ** -7, atol=1e-6)


def test_attention_bad_page_ends_its_sequence():
    need_gpu()
    lens, N = [100, 100], 8
    cache = gm.PagedCache(BF16, 1, lens, [108, 108], seed=1)
    ks, vs = _entries(cache, BF16, lens, N, 3)
    good = cache.block_table.clone()
    cache.block_table[0, 2] = cache.num_pages + 5
    q = _rand(BF16, 2, N, 32, 128, seed=9)
    masks = _masks(_trees(2, N, 5))[0]
    out, err = torch.empty((2, N, 32, 128), dtype=torch.bfloat16, device="cuda"), _err()
    call = lambda: gm.tree_attention(gm.model_config(BF16), cache, 0, t32(q, torch.bfloat16), _bits(masks), out,  # noqa: E731
                                     gm.Workspace(), dev_err=err)
    call()
    assert int(err.item()) == gm.GM_DEVERR_PAGE
    bad = out.clone()
    cache.block_table.copy_(good)
    err.zero_()
    call()
    assert int(err.item()) == 0 and torch.equal(out[1], bad[1]) and bool(torch.isfinite(bad).all())


# ------------------------------------------------------------------------------------- accept and commit
@pytest.mark.parametrize("B,N", [(1, 1), (7, 2), (33, 16), (5, 64)])
def test_accept(B, N):
    need_gpu()
    r = np.random.default_rng(B * N)
    parents = _trees(B, N, B, forest=True)
    tokens, nxt = r.integers(0, 3, (B, N)), r.integers(0, 3, (B, N))     # many twins and long walks
    parents[0] = np.arange(N) - 1                                        # a chain, all accepted
    nxt[0, :-1] = tokens[0, 1:]
    n = r.integers(0, N + 1, B)
    n[0] = N
    for counts in (None, n):
        path, out, na = i32(np.full((B, N), 77)), i32(np.full((B, N), 77)), i32(np.full(B, 77))
        gm.tree_accept(i32(parents), i32(tokens), i32(nxt), path, na, out, i32(counts) if counts is not None else None)
        for b in range(B):
            p, o = otree.tree_accept(parents[b], tokens[b], nxt[b], None if counts is None else counts[b])
            assert int(na[b]) == len(p) - 1
            assert path[b].cpu().tolist() == p + [-1] * (N - len(p))
            assert out[b].cpu().tolist() == o + [-1] * (N - len(o))


@pytest.mark.parametrize("name,layers,lens,N,page", [
    ("qwen", 1, [0, 15, 16, 100], 16, 16), ("qwen", 36, [30, 3], 64, 32), ("mha", 2, [9, 63, 64], 9, 64),
    ("f32", 2, [0, 40], 64, 16), ("f32_g4_d128", 3, [17], 12, 16),
    ("mha", 130, [9], 9, 16)])                                     # layers for two launches
def test_commit(name, layers, lens, N, page):
    need_gpu()
    shape = dataclasses.replace(SHAPES[name], n_layers=max(1, layers - 1))     # the cache's layers are its own
    B = len(lens)
    cache = gm.PagedCache(shape, layers, lens, np.array(lens) + N, page_size=page, seed=N)
    for p in cache.k + cache.v:
        p.copy_(torch.randn(p.shape, device="cuda"))
    r = np.random.default_rng(N)
    n = r.integers(-1, N, B)
    n[0] = N // 2
    path = np.full((B, N), -1)
    for b in range(B):
        if n[b] >= 0:
            path[b, :n[b] + 1] = np.concatenate([[0], 1 + np.sort(r.choice(N - 1, n[b], replace=False))])
    old = [[cache.read(l, b, np.arange(lens[b] + N)) for b in range(B)] for l in range(layers)]
    slots, err = i32(np.full((B, N), 5)), _err()
    gm.tree_commit(gm.model_config(shape), cache, i32(path), i32(n), slots, err)
    assert int(err.item()) == 0
    assert cache.seq_lens.cpu().tolist() == [lens[b] + int(n[b]) + 1 for b in range(B)]
    table = cache.block_table_host
    for b in range(B):
        pos = lens[b] + np.arange(N)
        want = np.where(np.arange(N) <= n[b], table[b][pos // page] * page + pos % page, -1)
        assert np.array_equal(slots[b].cpu().numpy(), want)
        for l in range(layers):
            src = np.arange(lens[b] + N)
            src[lens[b]:lens[b] + n[b] + 1] = lens[b] + path[b, :n[b] + 1]
            for got, was in zip(cache.read(l, b, np.arange(lens[b] + N)), old[l][b]):
                assert np.array_equal(got, was[src])


def test_commit_reports_bad_paths_and_pages():
    need_gpu()
    lens, N = [10, 10, 14], 8
    cache = gm.PagedCache(BF16, 1, lens, [32, 32, 32], seed=3)
    for p in cache.k + cache.v:
        p.copy_(torch.randn(p.shape, device="cuda"))
    cache.block_table[2, 1] = -1
    path = np.full((3, N), -1)
    path[0, :3] = [0, 4, 2]                          # not increasing
    path[1, :2] = [0, 9]                             # no node
    path[2, :3] = [0, 1, 3]                          # slot 17 -> 16: the page of slots 16..31 is gone
    old_k, old_v, err = cache.k[0].clone(), cache.v[0].clone(), _err()
    gm.tree_commit(gm.model_config(BF16), cache, i32(path), i32([2, 1, 2]), None, err)
    assert int(err.item()) == gm.GM_DEVERR_TREE | gm.GM_DEVERR_PAGE
    assert torch.equal(cache.k[0], old_k) and torch.equal(cache.v[0], old_v)
    assert cache.seq_lens.cpu().tolist() == [13, 12, 17]


# ------------------------------------------------------------------------------------- together
@pytest.mark.parametrize("name,N", [("qwen", 12), ("g7", 40), ("f32", 12)])
def test_tree_step(name, N):
    """One layer's tree step as a program makes it, twice: masks, append at the nodes' depths, attention of
    the nodes, the target's choice from its logits, walk, commit.  Every node's row is causal attention over
    its own line, and after the commit the cache holds the accepted line as if it had been drafted alone."""
    need_gpu()
    shape = dataclasses.replace(SHAPES[name], qk_norm=True)
    cfg, dt = gm.model_config(shape), gm.torch_dtype(shape)
    H, kv, D, V = shape.n_heads, shape.n_kv_heads, shape.head_dim, 300
    lens, B = np.array([0, 9, 47]), 3
    cache = gm.PagedCache(shape, 1, lens, lens + 4 * N, seed=1)
    ws, err = gm.Workspace(), _err()
    r = np.random.default_rng(N)
    qn, kn = _rand(shape, D, seed=1), _rand(shape, D, seed=2)
    ks, vs = [[] for _ in range(B)], [[] for _ in range(B)]
    prompt = int(lens.sum())
    pk, pv = _rand(shape, prompt, kv, D, seed=3), _rand(shape, prompt, kv, D, seed=4)
    cache.seq_lens.zero_()
    gm.kv_append(cfg, cache, 0, t32(pk, dt), t32(pv, dt), row_start=i32(np.concatenate([[0], np.cumsum(lens)])),
                 max_rows=int(lens.max()), k_norm=t32(kn, dt), dev_err=err)
    cache.seq_lens.copy_(i32(lens))
    s0 = np.concatenate([[0], np.cumsum(lens)])
    for b in range(B):
        rows = slice(s0[b], s0[b + 1])
        ks[b] = list(synth.quantise(otree.append_rows(pk[rows], np.arange(lens[b]), shape.rope_base, shape.rms_eps,
                                                      kn).astype(np.float32), shape.dtype))
        vs[b] = list(pv[rows])
    for step in range(2):
        parents = _trees(B, N, 10 * N + step)
        tokens = r.integers(0, V, (B, N))
        x = _rand(shape, B * N, (H + 2 * kv) * D, seed=20 + step)
        xd = t32(x, dt)
        q, k, v = (xd[:, a:b].unflatten(1, (-1, D)) for a, b in
                   ((0, H * D), (H * D, (H + kv) * D), ((H + kv) * D, (H + 2 * kv) * D)))
        masks, depths = torch.empty((B, N), dtype=torch.int64, device="cuda"), i32(np.zeros((B, N)))
        q_out = torch.empty((B * N, H, D), dtype=dt, device="cuda")
        out = torch.empty((B, N, H, D), dtype=dt, device="cuda")
        gm.tree_masks(i32(parents), masks, depths, dev_err=err)
        gm.kv_append(cfg, cache, 0, k, v, q=q, q_out=q_out, offsets=depths.view(-1), q_norm=t32(qn, dt),
                     k_norm=t32(kn, dt), dev_err=err)
        gm.tree_attention(cfg, cache, 0, q_out.view(B, N, H, D), masks, out, ws, dev_err=err)
        # logits that lead along the tree: each node's likely next token is its last child's, if any
        z = r.standard_normal((B * N, V)).astype(np.float32)
        for b in range(B):
            for i in range(1, N):
                z[b * N + parents[b, i], tokens[b, i]] += 9.0 + 0.01 * i
        top_lp = torch.empty((B * N, 1), dtype=torch.float32, device="cuda")
        top = i32(np.zeros((B * N, 1)))
        gm.token_logprobs(t32(z), None, ws, top_logp=top_lp, top_ids=top)
        path, otok, na = i32(np.zeros((B, N))), i32(np.zeros((B, N))), i32(np.zeros(B))
        gm.tree_accept(i32(parents), i32(tokens), top.view(B, N), path, na, otok)
        gm.tree_commit(cfg, cache, path, na, None, err)
        cache.max_ctx = int(cache.seq_lens.max())
        torch.cuda.synchronize()
        assert int(err.item()) == 0
        assert np.array_equal(top[:, 0].cpu().numpy(), z.argmax(1))
        xs = x.reshape(B, N, -1, D)
        got = out.float().cpu().numpy()
        for b in range(B):
            m = len(ks[b])
            om, od = otree.tree_masks(parents[b])
            quant = lambda a: synth.quantise(a.astype(np.float32), shape.dtype)  # noqa: E731
            rk = quant(otree.append_rows(xs[b, :, H:H + kv], m + od, shape.rope_base, shape.rms_eps, kn))
            rq = quant(otree.append_rows(xs[b, :, :H], m + od, shape.rope_base, shape.rms_eps, qn))
            rv = xs[b, :, H + kv:]
            want, mag = otree.tree_attention(rq, np.stack(ks[b] + list(rk)), np.stack(vs[b] + list(rv)), m, om)
            # a query or key that falls on the other side of a rounding is a step off: scores move by at
            # most 2 * 2 half steps of sum |q k| / sqrt(D), the weights by twice that
            s_abs = np.abs(rq).max(0).sum(-1).max() * max(np.abs(np.stack(ks[b] + list(rk))).max(), 1) / np.sqrt(D)
            tol = (8 * _half(shape) * s_abs + 2.0 ** -8) * mag + _half(shape) * np.abs(want)
            assert (np.abs(got[b] - want) <= tol).all()
            p, o = otree.tree_accept(parents[b], tokens[b], z.reshape(B, N, V)[b].argmax(-1))
            assert path[b].cpu().tolist()[:len(p)] == p and int(na[b]) == len(p) - 1
            assert otok[b].cpu().tolist()[:len(o)] == o
            ks[b] += [rk[i] for i in p]
            vs[b] += [rv[i] for i in p]
            assert int(cache.seq_lens[b]) == len(ks[b])
            gk, gv = cache.read(0, b, np.arange(len(ks[b])))
            assert np.array_equal(gv, np.stack(vs[b]))
            assert (np.abs(gk - np.stack(ks[b])) <= 2 * _half(shape) * np.abs(gk) + 64 * U * 8).all()


def test_chain_as_a_tree_is_the_verify_attention():
    need_gpu()
    lens, k = [5, 300, 1000], 7
    cache = gm.PagedCache(BF16, 1, lens, np.array(lens) + k + 1, seed=2)
    _entries(cache, BF16, lens, k + 1, 7)
    cfg = gm.model_config(BF16)
    q = t32(_rand(BF16, 3, k + 1, 32, 128, seed=1), torch.bfloat16)
    a, b = torch.empty_like(q), torch.empty_like(q)
    gm.verify_attention(cfg, cache, 0, q, a, gm.Workspace())
    masks = torch.empty((3, k + 1), dtype=torch.int64, device="cuda")
    depths = i32(np.zeros((3, k + 1)))
    gm.tree_masks(i32(np.tile(np.arange(k + 1) - 1, (3, 1))), masks, depths)
    gm.tree_attention(cfg, cache, 0, q, masks, b, gm.Workspace())
    # both are within half a step and 2^-15 of the same value
    d = (a.float() - b.float()).abs()
    assert bool((d <= 2.0 ** -7 * a.float().abs() + 1e-3).all())


def test_pools_past_32_bits():
    """Pools of more than 2^32 bytes and 2^31 elements, with the sequence in their last pages."""
    need_gpu()
    lens, N, pages = [40], 8, 140_000
    table = np.full((1, 4), -1, np.int32)
    table[0] = [pages - 1, 3, pages - 2, pages - 3]
    pools = [torch.empty((1, pages, 8 * 16 * 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    cache = gm.PagedCache(BF16, 1, lens, [64], table=table, pools=pools)
    assert cache.k[0].numel() > 2 ** 31
    ks, vs = _entries(cache, BF16, lens, 0, 5)
    cfg, dt, err = gm.model_config(BF16), torch.bfloat16, _err()
    k, v, q = (_rand(BF16, N, h, 128, seed=s) for h, s in ((8, 1), (8, 2), (32, 3)))
    parents = _trees(1, N, 4)
    masks, depths = _masks(parents)
    q_out, out = (torch.empty((N, 32, 128), dtype=dt, device="cuda") for _ in range(2))
    gm.kv_append(cfg, cache, 0, t32(k, dt), t32(v, dt), q=t32(q, dt), q_out=q_out, offsets=i32(depths[0]), dev_err=err)
    gm.tree_attention(cfg, cache, 0, q_out.view(1, N, 32, 128), _bits(masks), out.view(1, N, 32, 128), gm.Workspace(),
                      dev_err=err)
    gk, gv = cache.read(0, 0, np.arange(48))
    assert np.array_equal(gv[40:], v) and np.array_equal(gv[:40], vs[0]) and np.array_equal(gk[:40], ks[0])
    want, mag = otree.tree_attention(q_out.float().cpu().numpy(), gk, gv, 40, masks[0])
    assert (np.abs(out.float().cpu().numpy() - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -8 * mag).all()
    path = np.full((1, N), -1)
    path[0, :3] = [0, 2, 5]
    gm.tree_commit(cfg, cache, i32(path), i32([2]), None, err)
    ck, cv = cache.read(0, 0, np.arange(43))
    assert int(err.item()) == 0
    assert np.array_equal(ck[40:], gk[[40, 42, 45]]) and np.array_equal(cv[40:], gv[[40, 42, 45]])


def test_graph_and_other_stream():
    """The step captured once and replayed, between eager calls on another stream that share nothing with it;
    each replay gives the eager call's bits."""
    need_gpu()
    lens, N, B = [20, 333], 24, 2
    cfg, dt = gm.model_config(BF16), torch.bfloat16
    parents = _trees(B, N, 3)
    tokens = np.random.default_rng(1).integers(0, 4, (B, N))

    def make(seed):
        cache = gm.PagedCache(BF16, 1, lens, np.array(lens) + N, seed=1)
        _entries(cache, BF16, lens, 0, 5)
        t = dict(k=t32(_rand(BF16, B * N, 8, 128, seed=seed), dt), v=t32(_rand(BF16, B * N, 8, 128, seed=seed + 1), dt),
                 q=t32(_rand(BF16, B * N, 32, 128, seed=seed + 2), dt), parents=i32(parents), tokens=i32(tokens),
                 masks=torch.empty((B, N), dtype=torch.int64, device="cuda"), depths=i32(np.zeros((B, N))),
                 q_out=torch.empty((B * N, 32, 128), dtype=dt, device="cuda"),
                 out=torch.empty((B, N, 32, 128), dtype=dt, device="cuda"), path=i32(np.zeros((B, N))),
                 na=i32(np.zeros(B)), otok=i32(np.zeros((B, N))), ws=gm.Workspace(), lens0=i32(lens))
        nxt = i32(np.roll(tokens, -1, 1))

        def step():
            cache.seq_lens.copy_(t["lens0"])
            gm.tree_masks(t["parents"], t["masks"], t["depths"])
            gm.kv_append(cfg, cache, 0, t["k"], t["v"], q=t["q"], q_out=t["q_out"], offsets=t["depths"].view(-1))
            gm.tree_attention(cfg, cache, 0, t["q_out"].view(B, N, 32, 128), t["masks"], t["out"], t["ws"])
            gm.tree_accept(t["parents"], t["tokens"], nxt, t["path"], t["na"], t["otok"])
            gm.tree_commit(cfg, cache, t["path"], t["na"])

        return step, lambda: [t["q_out"].clone(), t["out"].clone(), t["path"].clone(), cache.seq_lens.clone(),
                              cache.k[0].clone(), cache.v[0].clone()]

    step, read = make(1)
    other, read_other = make(50)
    step()
    other()
    torch.cuda.synchronize()
    want, want_other = read(), read_other()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    side = torch.cuda.Stream()
    for _ in range(4):
        with torch.cuda.stream(side):
            other()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(read(), want))
        assert all(torch.equal(a, b) for a, b in zip(read_other(), want_other))
