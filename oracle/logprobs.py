"""Log-probabilities of given tokens, entropy, alternatives, and their gradient in the logits (float64)."""
from __future__ import annotations

import numpy as np


def token_logprobs(z, ids, temperature=1.0, topk=0):
    """z [M, V]; returns (logp, entropy, top ids, top logp, max, sum exp((z - max) / T)).  A row without a
    logit above -inf: log p -inf, entropy 0, sum 0."""
    z = np.asarray(z, np.float64)
    mx = z.max(1)
    with np.errstate(invalid="ignore", divide="ignore"):
        y = (z - np.where(np.isneginf(mx), 0.0, mx)[:, None]) / temperature
        e = np.exp(y)
        S = e.sum(1)
        lp = y - np.log(S)[:, None]
        lp[S == 0] = -np.inf
        ent = np.where(S > 0, -np.where(e > 0, e * np.where(e > 0, lp, 0.0), 0.0).sum(1) / np.where(S > 0, S, 1), 0.0)
    ids = np.asarray(ids)
    ok = (ids >= 0) & (ids < z.shape[1])
    logp = np.where(ok, lp[np.arange(len(z)), np.where(ok, ids, 0)], 0.0)
    top = np.argsort(-z, axis=1, kind="stable")[:, :topk]      # decreasing, the lower id first among equals
    return logp, ent, top, np.take_along_axis(lp, top, 1), mx, S


def token_logprobs_grad(z, ids, g_logp, g_entropy=None, temperature=1.0):
    z = np.asarray(z, np.float64)
    M, V = z.shape
    _, ent, _, _, mx, S = token_logprobs(z, np.full(M, -1), temperature)
    out = np.zeros((M, V))
    for r in range(M):
        if S[r] == 0:
            continue
        y = (z[r] - mx[r]) / temperature
        p = np.exp(y) / S[r]
        lp = np.where(p > 0, y, 0.0) - np.log(S[r])
        ok = ids is not None and 0 <= ids[r] < V
        g = float(g_logp[r]) if ok else 0.0
        gh = float(g_entropy[r]) if g_entropy is not None else 0.0
        out[r] = -p * (g + gh * (lp + ent[r]))
        if ok:
            out[r, ids[r]] += g
    return out / temperature
