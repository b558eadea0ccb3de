"""Token log-probabilities and their gradient on the GPU against float64.

Tolerances, u = 2^-24 (half a float32 step).  With y = (z - max) / T in units of log 2: a term exp2(y) is off by
(3 |y| ln 2 + 2) u (difference, scale and product each by u; the exponential by 2 u), a lane's float32 sum of at
most 64 terms by 64 u, the sum of a lane's two and of 64 lanes by pairs by 7 u more, float64 beyond: S and log S
by at most (3 E|y| + 73) u with E the mean under p, 78 taken; W / S by (3 E y^2 + 156 E|y| + 3 (E|y|)^2) u.  The quotients and the last rounding add 4 u of the value.
"""
import math

import numpy as np
import pytest
import torch

from helpers import need_gpu, i32
from oracle import logprobs as olp
from paper_2609_16648_amd import gm

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _logits(M, V, dtype, seed, kind="spiky", ld=None):
    """[M, V] with rows ld apart, on the device, and the same values in float64 on the host."""
    r = np.random.default_rng([seed, M, V])
    z = r.standard_normal((M, V)).astype(np.float32) * 1.5
    if kind == "spiky":
        at = r.integers(0, V, (M, 8))
        z[np.arange(M)[:, None], at] = 12 - 1.2 * np.arange(8)
    elif kind == "flat":
        z[:] = 0.75
    elif kind == "ramp":
        z[:] = np.linspace(-8, 8, V)[None, :] * np.where(np.arange(M) % 2, 1, -1)[:, None]
    elif kind == "masked":
        z[:, ::3] = -np.inf
        z[0] = -np.inf
        if M > 1:
            z[1] = -np.inf
            z[1, V // 2] = 3.0                    # one id left
    elif kind == "lowest":
        z[r.random((M, V)) < 0.5] = np.finfo(np.float32).min if dtype == torch.float32 else -3.3895e38
        z[0] = np.finfo(np.float32).min if dtype == torch.float32 else -3.3895e38
    elif kind == "far":
        z = z * 40 + 3000
    buf = torch.full((M, ld or V), 1e30, dtype=dtype, device="cuda")
    t = buf[:, :V]
    t.copy_(torch.from_numpy(z))
    return t, t.double().cpu().numpy()


def _moments(z, T):
    """Per row E|y|, E y^2 (under p, y in units of log 2) and the whole |y|."""
    mx = z.max(1, keepdims=True)
    with np.errstate(invalid="ignore"):
        y = np.where(np.isneginf(mx), 0.0, (z - np.where(np.isneginf(mx), 0, mx)) / T)
        p = np.exp(y)
        p /= p.sum(1, keepdims=True)
        a = np.where(p > 0, np.abs(y) / math.log(2), 0.0)
    return (p * a).sum(1), (p * a * a).sum(1), p, a


def _buffers(M, k=0):
    f = lambda *s: torch.full(s, 99.0, dtype=torch.float32, device="cuda")  # noqa: E731
    return f(M), f(M), f(M, 2), (f(M, k), i32(np.full((M, k), 99))) if k else (None, None)


FORWARD = [
    # M, V, dtype, T, topk, kind, ld
    (1, 1, torch.float32, 1.0, 1, "normal", None),
    (3, 2, torch.bfloat16, 0.7, 2, "normal", 5),
    (5, 7, torch.float32, 1.3, 3, "normal", None),
    (4, 65, torch.float32, 1.0, 64, "spiky", None),
    (2, 513, torch.bfloat16, 1.0, 64, "normal", None),
    (3, 2047, torch.float32, 0.5, 20, "masked", 2050),
    (3, 2049, torch.float32, 1.0, 64, "masked", None),
    (6, 5003, torch.float32, 1.0, 64, "spiky", None),
    (6, 5003, torch.bfloat16, 0.7, 64, "flat", 5007),
    (3, 16384, torch.float32, 1.0, 8, "lowest", None),
    (3, 16385, torch.bfloat16, 0.5, 8, "lowest", 16391),
    (4, 32001, torch.bfloat16, 1.0, 64, "spiky", None),
    (4, 50257, torch.float32, 1.0, 64, "ramp", None),
    (2, 50257, torch.float32, 1.0, 64, "flat", None),
    (300, 50257, torch.float32, 1.0, 4, "spiky", None),
    (9, 151936, torch.float32, 1.0, 8, "spiky", None),
    (5, 151936, torch.bfloat16, 1.0, 64, "masked", None),
    (2, 151936, torch.float32, 1.0, 20, "far", None),
    (1, 524288, torch.float32, 1.0, 64, "normal", None),
    (700, 1000, torch.bfloat16, 1.0, 0, "spiky", None),
]


@pytest.mark.parametrize("M,V,dtype,T,topk,kind,ld", FORWARD)
def test_forward(M, V, dtype, T, topk, kind, ld):
    need_gpu()
    t, z = _logits(M, V, dtype, V + topk, kind, ld)
    r = np.random.default_rng(V)
    ids = r.integers(0, V, M)
    ids[r.random(M) < 0.2] = -1
    ids[0] = V - 1
    logp, ent, stats, (top_lp, top) = _buffers(M, topk)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    gm.token_logprobs(t, i32(ids), gm.Workspace(), logp=logp, entropy=ent, top_logp=top_lp, top_ids=top, stats=stats,
                      temperature=T, dev_err=err)
    assert int(err.item()) == 0
    w_logp, w_ent, w_top, w_lp, mx, S = olp.token_logprobs(z, ids, float(np.float32(T)), topk)
    # a value past float32's range, 2^128 (1 - 2^-25) and beyond, rounds to infinity: the lowest logit at T < 1
    for a in (w_logp, w_lp):
        a[a <= -(2.0 ** 128) * (1 - 2.0 ** -25)] = -np.inf
    e1, e2, _, _ = _moments(z, T)
    ds = (3 * e1 + 78) * U
    got = logp.cpu().numpy()
    live = np.isfinite(w_logp)
    assert np.array_equal(got[~live], w_logp[~live])
    assert (np.abs(got[live] - w_logp[live]) <= (ds + 4 * U * np.abs(w_logp))[live]).all()
    dh = ds + (3 * e2 + 156 * e1 + 3 * e1 * e1) * U + 4 * U * w_ent
    assert (np.abs(ent.cpu().numpy() - w_ent) <= dh).all()
    st = stats.cpu().numpy()
    assert np.array_equal(st[:, 0], mx.astype(np.float32))
    assert (np.abs(st[:, 1] - S) <= (ds + 2 * U) * S).all()
    if topk:
        assert np.array_equal(top.cpu().numpy(), w_top)
        g = top_lp.cpu().numpy()
        ok = np.isfinite(w_lp)
        assert np.array_equal(g[~ok], w_lp[~ok])
        assert (np.abs(g[ok] - w_lp[ok]) <= (ds[:, None] + 4 * U * np.abs(w_lp))[ok]).all()


def test_each_output_alone_and_bad_ids():
    need_gpu()
    M, V = 70, 3001
    t, z = _logits(M, V, torch.float32, 1)
    ids = np.arange(M) * 40
    ids[5], ids[6] = V, 2 ** 31 - 1
    logp, ent, stats, (top_lp, top) = _buffers(M, 6)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = gm.Workspace()
    gm.token_logprobs(t, i32(ids), ws, logp=logp, entropy=ent, top_logp=top_lp, top_ids=top, stats=stats, dev_err=err)
    assert int(err.item()) == gm.GM_DEVERR_TOKEN and logp[5] == 0 and logp[6] == 0
    l2, e2, s2, (tl2, t2) = _buffers(M, 6)
    gm.token_logprobs(t, i32(ids), ws, logp=l2)
    gm.token_logprobs(t, None, ws, entropy=e2)
    gm.token_logprobs(t, None, ws, stats=s2)
    gm.token_logprobs(t, None, ws, top_logp=tl2, top_ids=t2)
    for a, b in ((logp, l2), (ent, e2), (stats, s2), (top_lp, tl2), (top, t2)):
        assert torch.equal(a, b)


def test_rows_with_nan_and_inf():
    need_gpu()
    M, V = 6, 20000
    t, _ = _logits(M, V, torch.float32, 2)
    t[0, 100] = float("nan")
    t[1, V - 1] = float("inf")
    t[2] = float("nan")
    t[3] = float("-inf")
    t[3, 17000] = float("nan")
    logp, ent, stats, (top_lp, top) = _buffers(M, 5)
    gm.token_logprobs(t, i32(np.full(M, 7)), gm.Workspace(), logp=logp, entropy=ent, top_logp=top_lp, top_ids=top,
                      stats=stats)
    assert bool(torch.isnan(logp[:4]).all()) and bool(torch.isnan(ent[:4]).all())
    assert bool(torch.isnan(top_lp[:4]).all()) and bool((top[:4] == -1).all())
    assert bool(torch.isfinite(logp[4:]).all()) and bool((top[4:] >= 0).all())


GRAD = [
    # M, V, dtype, T, entropy, tokens, kind, ld
    (1, 1, torch.float32, 1.0, True, True, "normal", None),
    (3, 7, torch.bfloat16, 0.7, True, True, "normal", 9),
    (5, 1023, torch.float32, 0.7, True, True, "spiky", None),
    (4, 4097, torch.float32, 1.3, True, False, "masked", 4100),
    (4, 16385, torch.bfloat16, 1.0, True, True, "masked", None),
    (3, 50257, torch.float32, 0.5, True, True, "lowest", None),
    (33, 50257, torch.bfloat16, 1.0, False, True, "spiky", 50260),
    (6, 151936, torch.float32, 1.0, True, True, "spiky", None),
    (6, 151936, torch.bfloat16, 1.0, True, True, "spiky", None),
]


@pytest.mark.parametrize("M,V,dtype,T,entropy,tokens,kind,ld", GRAD)
def test_gradient(M, V, dtype, T, entropy, tokens, kind, ld):
    """Against the formula.  A value is e (a + b y) with e as above, a and b off by (S, quotients, entropy)
    at most (3 E|y| + 90 + dH) u of their terms; then the gradient's own type."""
    need_gpu()
    t, z = _logits(M, V, dtype, V + 1, kind, ld)
    r = np.random.default_rng(V + 1)
    ids = r.integers(0, V, M)
    ids[r.random(M) < 0.2] = -1
    g, gh = (r.standard_normal(M).astype(np.float32) for _ in range(2))
    logp, ent, stats, _ = _buffers(M)
    ws = gm.Workspace()
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    gm.token_logprobs(t, i32(ids), ws, logp=logp, entropy=ent, stats=stats, temperature=T)
    buf = torch.full((M, (ld or V) + 2), 5.0, dtype=dtype, device="cuda")
    grad = buf[:, :V]
    args = dict(entropy=ent if entropy else None, g_entropy=dev(gh) if entropy else None, temperature=T)
    gm.token_logprobs_grad(t, i32(ids) if tokens else None, stats, dev(g) if tokens else None, grad, **args)
    assert bool((buf[:, V:] == 5.0).all())                      # nothing behind a row
    want = olp.token_logprobs_grad(z, ids if tokens else None, g, gh if entropy else None, float(np.float32(T)))
    e1, e2, p, a = _moments(z, T)
    w_ent = olp.token_logprobs(z, np.full(M, -1), T)[1]
    S = np.exp(z - z.max(1, keepdims=True)).sum(1) if kind != "masked" else np.full(M, float(V))
    gg = np.abs(g) * (ids >= 0) * tokens
    hh = np.abs(gh) * entropy
    terms = gg[:, None] + hh[:, None] * (a + w_ent[:, None] + np.log(np.maximum(S, 1))[:, None])
    c = 3 * a + (3 * e1 + 90)[:, None] + (3 * e2 + 156 * e1 + 3 * e1 * e1)[:, None]
    half = 2.0 ** -8 if dtype == torch.bfloat16 else U
    step = half * np.abs(want) + (U * c * p * terms + 4 * U * gg[:, None] * (np.arange(V) == ids[:, None])) / T
    tiny = 2.0 ** -133 if dtype == torch.bfloat16 else 2.0 ** -125      # below the smallest normal values
    got = grad.double().cpu().numpy()
    bad = np.abs(got - want) > (1 + half) * step + tiny
    assert not bad.any(), (np.abs(got - want)[bad][:4], step[bad][:4], np.argwhere(bad)[:4])
    # in place
    gm.token_logprobs_grad(t, i32(ids) if tokens else None, stats, dev(g) if tokens else None, t, **args)
    assert torch.equal(t, grad)


def test_gradient_against_differences():
    """The gradient predicts how the library's own outputs move: a central difference of h = 2^-5 in one direction
    (float32 outputs, so coarse: truncation h^2 / 6 times a third derivative of at most 8, and rounding of the
    summed outputs 2^-17 / h)."""
    need_gpu()
    M, V, h = 4, 300, 2.0 ** -5
    t, _ = _logits(M, V, torch.float32, 9, "normal")
    ids = i32(np.array([1, 299, 7, -1]))
    logp, ent, stats, _ = _buffers(M)
    ws, one = gm.Workspace(), torch.ones(M, device="cuda")
    d = torch.randn(M, V, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    d /= d.norm(dim=1, keepdim=True)

    def f(z):
        gm.token_logprobs(z, ids, ws, logp=logp, entropy=ent, stats=stats)
        return logp.double() + ent.double()

    f(t)
    grad = torch.empty_like(t)
    gm.token_logprobs_grad(t, ids, stats, one, grad, entropy=ent, g_entropy=one)
    slope = (grad.double() * d.double()).sum(1)
    up, dn = f(t + h * d), f(t - h * d)
    assert bool(((up - dn) / (2 * h) - slope).abs().max() < 8 * h * h / 6 + 2.0 ** -17 / h)


def test_rows_past_32_bits():
    """More than 2^31 logits in one call, rows further apart than they are long: the last rows are right."""
    need_gpu()
    M, V, ld = 16400, 131100, 131104
    buf = torch.zeros((M, ld), dtype=torch.bfloat16, device="cuda")
    t = buf[:, :V]
    assert M * ld > 2 ** 31
    z, h = _logits(3, V, torch.bfloat16, 3)
    t[-3:] = z
    logp, ent, stats, (top_lp, top) = _buffers(M, 4)
    ids = np.full(M, 5)
    gm.token_logprobs(t, i32(ids), gm.Workspace(), logp=logp, entropy=ent, top_logp=top_lp, top_ids=top, stats=stats)
    w = olp.token_logprobs(h, ids[:3], 1.0, 4)
    assert np.allclose(logp[-3:].cpu().numpy(), w[0], rtol=1e-5) and np.array_equal(top[-3:].cpu().numpy(), w[2])
    assert np.allclose(ent[:5].cpu().numpy(), math.log(V), rtol=1e-6) and top[0].cpu().tolist() == [0, 1, 2, 3]
    g = torch.ones(M, device="cuda")
    gm.token_logprobs_grad(t, i32(ids), stats, g, t)
    want = olp.token_logprobs_grad(h, ids[:3], np.ones(3))
    assert np.abs(t[-3:].double().cpu().numpy() - want).max() <= 2.0 ** -8
    assert abs(float(t[0, 5]) - (1 - 1 / V)) <= 2.0 ** -8 and bool((buf[:, V:] == 0).all())


def test_graph_replays_and_streams():
    """Forward and gradient captured once and replayed, with eager calls of their own workspace in between."""
    need_gpu()
    M, V = 40, 50257
    t, _ = _logits(M, V, torch.float32, 4)
    y, _ = _logits(M, V, torch.float32, 5)
    ids, g = i32(np.arange(M)), torch.ones(M, device="cuda")

    def make(z):
        out = _buffers(M, 8)
        logp, ent, stats, (top_lp, top) = out
        grad, ws = torch.empty_like(z), gm.Workspace()

        def step():
            gm.token_logprobs(z, ids, ws, logp=logp, entropy=ent, top_logp=top_lp, top_ids=top, stats=stats)
            gm.token_logprobs_grad(z, ids, stats, g, grad, entropy=ent, g_entropy=g)

        return step, lambda: [a.clone() for a in (logp, ent, stats, top_lp, top, grad)]

    step, read = make(t)
    other, read_other = make(y)
    step()
    other()
    torch.cuda.synchronize()
    want, want_other = read(), read_other()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    side = torch.cuda.Stream()
    for _ in range(4):
        with torch.cuda.stream(side):
            other()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(read(), want))
        assert all(torch.equal(a, b) for a, b in zip(read_other(), want_other))
