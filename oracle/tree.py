"""Draft trees: masks, attention of the nodes, the accept walk and the commit of a path.

A tree of N nodes continues the committed tokens: node 0 is the pending token, node i > 0 follows
node parents[i] < i.  The method drafts a chain (Sec. 2.2), which is the tree parents[i] = i - 1.
"""
from __future__ import annotations

import numpy as np


def tree_masks(parents, n_nodes=None):
    """(masks bool [N, N], depths [N]): masks[i, j] iff j is i or one of its ancestors; a parent that is
    no earlier node of the tree ends the line."""
    parents = np.asarray(parents)
    N = len(parents)
    n = N if n_nodes is None else int(np.clip(n_nodes, 0, N))
    masks = np.zeros((N, N), bool)
    for i in range(n):
        j = i
        while True:
            masks[i, j] = True
            up = int(parents[j])
            if not 0 <= up < j:
                break
            j = up
    return masks, np.maximum(masks.sum(1) - 1, 0)


def tree_attention(q, k, v, m, masks, n_nodes=None):
    """q [N, heads, D]; k, v [m + N, kv_heads, D]; masks bool [N, N] over the entries m .. m + N - 1.
    Rows of nodes past n_nodes, and of nodes that see nothing, are 0.  float64; also returns
    sum_t p_t |v_t|, the scale of the rounding errors of the weights."""
    q, k, v = (np.asarray(a, np.float64) for a in (q, k, v))
    N, H, D = q.shape
    G = H // k.shape[1]
    n = N if n_nodes is None else int(np.clip(n_nodes, 0, N))
    out, mag = np.zeros_like(q), np.zeros_like(q)
    for i in range(n):
        see = np.concatenate([np.ones(m, bool), masks[i] & (np.arange(N) < n)])
        if not see.any():
            continue
        for h in range(H):
            kk, vv = k[:m + N][see, h // G], v[:m + N][see, h // G]
            s = kk @ q[i, h] / np.sqrt(D)
            p = np.exp(s - s.max())
            p /= p.sum()
            out[i, h], mag[i, h] = p @ vv, p @ np.abs(vv)
    return out, mag


def tree_accept(parents, tokens, next_ids, n_nodes=None):
    """(path, accepted tokens and the final one) of one tree; empty lists for a tree without nodes."""
    N = len(parents)
    n = N if n_nodes is None else int(np.clip(n_nodes, 0, N))
    if n == 0:
        return [], []
    path, out, cur = [0], [], 0
    while True:
        out.append(int(next_ids[cur]))
        child = [i for i in range(max(cur, 0) + 1, n) if parents[i] == cur and tokens[i] == next_ids[cur]]
        if not child:
            return path, out
        cur = child[0]
        path.append(cur)


def append_rows(x, positions, base, eps, weight=None):
    """RMSNorm over the channels (with a weight) and rotate-half rotation of x [T, heads, D], float64."""
    x = np.asarray(x, np.float64)
    D = x.shape[-1]
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(weight, np.float64)
    ang = np.asarray(positions, np.float64)[:, None] * float(base) ** (-2.0 * np.arange(D // 2) / D)
    cs, sn = np.cos(ang)[:, None], np.sin(ang)[:, None]
    a, b = x[..., :D // 2], x[..., D // 2:]
    return np.concatenate([a * cs - b * sn, b * cs + a * sn], -1)
