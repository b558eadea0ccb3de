"""Refusals of the draft-tree and log-probability entry points, on the host, before anything is launched."""
import ctypes

import pytest
import torch

import synth
from paper_2609_16648_amd import gm

FAKE = ctypes.c_void_p(1 << 20)          # never dereferenced: every call below fails validation first
BF16 = gm.model_config(synth.QWEN3_4B_LAYER)
F32 = gm.model_config(synth.ModelShape(2, 256, 4, 4, 64, 1024, 1024, dtype="f32"))


def _cache(n_layers=1, max_ctx=100, page_size=16, max_pages=10, table=FAKE):
    kp = (ctypes.c_void_p * n_layers)(*([1 << 20] * n_layers))
    d = gm.KVCacheDesc(kp, kp, n_layers, page_size, 100, max_pages, table, FAKE, max_ctx)
    d.keep = kp
    return d


def _cfg(**kw):
    c = gm.ModelConfig.from_buffer_copy(BF16)
    for n, v in kw.items():
        setattr(c, n, v)
    return c


def _append(cfg=BF16, cache=None, layer=0, B=4, T=32, max_rows=8, row_start=None, offsets=None, q=FAKE, sq=4096,
            k=FAKE, sk=1024, v=FAKE, sv=1024, qn=None, kn=None, qo=FAKE):
    return gm.lib().gm_kv_append(ctypes.byref(cfg), ctypes.byref(cache or _cache()), layer, B, T, max_rows, row_start,
                                 offsets, q, sq, k, sk, v, sv, qn, kn, qo, None, None)


def test_kv_append_rejects():
    A, U, C = gm.GM_ERR_INVALID_ARG, gm.GM_ERR_UNSUPPORTED, gm.GM_ERR_CAPACITY
    assert _append(cfg=_cfg(head_dim=64)) == U
    assert _append(layer=1) == A and _append(layer=-1) == A
    assert _append(cache=_cache(max_ctx=153)) == C and "exceed" in gm.last_error()    # 153 + 8 > 160
    assert _append(cache=_cache(page_size=24)) == U
    assert _append(cache=_cache(table=None)) == A
    assert _append(T=30) == A and _append(max_rows=7) == A                # not B equal shares; shares of 8
    assert _append(max_rows=-1) == A and _append(T=-1) == A and _append(B=-1) == A
    # a bound above the rows that there are counts as those (129 + 31 fit in 160, 130 + 31 do not)
    assert _append(row_start=FAKE, T=31, max_rows=200, cache=_cache(max_ctx=130)) == C
    assert _append(row_start=FAKE, T=31, max_rows=200, cache=_cache(max_ctx=129), k=None) == A
    assert _append(T=(1 << 27) + 4, max_rows=8, row_start=FAKE) == U
    assert _append(k=None) == A and _append(v=None) == A
    assert _append(q=None) == A and _append(qo=None) == A and "together" in gm.last_error()
    assert _append(sq=4095) == A and _append(sk=1023) == A and _append(sv=0) == A
    assert _append(cfg=_cfg(qk_norm=1), kn=FAKE) == A and _append(cfg=_cfg(qk_norm=1), qn=FAKE) == A
    assert _append(B=0) == gm.GM_OK and _append(T=0, max_rows=0) == gm.GM_OK


def _attn(cfg=BF16, cache=None, layer=0, B=4, N=16, q=FAKE, masks=FAKE, out=FAKE, ws=FAKE, nbytes=1 << 40):
    return gm.lib().gm_tree_attention(ctypes.byref(cfg), ctypes.byref(cache or _cache()), layer, B, N, q, masks, None,
                                      out, ws, nbytes, None, None)


def test_tree_attention_rejects():
    A, U = gm.GM_ERR_INVALID_ARG, gm.GM_ERR_UNSUPPORTED
    assert _attn(N=0) == U and _attn(N=65) == U and _attn(B=-1) == A
    assert _attn(cache=_cache(max_ctx=145)) == gm.GM_ERR_CAPACITY                      # 145 + 16 > 160
    assert _attn(layer=3) == A and _attn(q=None) == A and _attn(masks=None) == A and _attn(out=None) == A
    need = gm.workspace_size(gm.GM_OP_TREE_ATTENTION, BF16, 4, 16, 100)
    assert need > 0 and _attn(nbytes=need - 1) == gm.GM_ERR_WORKSPACE
    assert _attn(ws=ctypes.c_void_p((1 << 20) + 64)) == gm.GM_ERR_WORKSPACE
    assert _attn(B=0) == gm.GM_OK
    assert gm.workspace_size(gm.GM_OP_TREE_ATTENTION, BF16, 4, 65, 100) == 0
    assert gm.workspace_size(gm.GM_OP_TREE_ATTENTION, BF16, 4, 0, 100) == 0
    assert gm.workspace_size(gm.GM_OP_TREE_ATTENTION, F32, 4, 64, 100) == 0            # needs no scratch
    wide = _cfg(n_heads=65, n_kv_heads=1)
    assert gm.workspace_size(gm.GM_OP_TREE_ATTENTION, wide, 4, 1, 100) == 0            # more than 64 heads per KV head


def test_tree_index_calls_reject():
    L, A, U = gm.lib(), gm.GM_ERR_INVALID_ARG, gm.GM_ERR_UNSUPPORTED
    assert L.gm_tree_masks(4, 65, FAKE, None, FAKE, FAKE, None, None) == U
    assert L.gm_tree_masks(4, 8, None, None, FAKE, FAKE, None, None) == A
    assert L.gm_tree_masks(4, 8, FAKE, None, None, FAKE, None, None) == A
    assert L.gm_tree_masks(0, 8, None, None, None, None, None, None) == gm.GM_OK
    acc = [FAKE, FAKE, FAKE, None, FAKE, FAKE, FAKE]
    assert L.gm_tree_accept(4, 0, *acc, None) == U and L.gm_tree_accept(-1, 8, *acc, None) == A
    for i in (0, 1, 2, 4, 5, 6):
        assert L.gm_tree_accept(4, 8, *(acc[:i] + [None] + acc[i + 1:]), None) == A
    com = lambda cfg=BF16, c=None, B=4, N=16, path=FAKE, n=FAKE: L.gm_tree_commit(  # noqa: E731
        ctypes.byref(cfg), ctypes.byref(c or _cache()), B, N, path, n, None, None, None)
    assert com(c=_cache(max_ctx=145)) == gm.GM_ERR_CAPACITY
    assert com(path=None) == A and com(n=None) == A and com(N=65) == U and com(B=(1 << 22) + 1) == U
    assert com(cfg=_cfg(head_dim=96)) == U and com(B=0) == gm.GM_OK


def _lp(M=8, V=1000, dtype=gm.GM_F32, z=FAKE, ld=1000, T=1.0, ids=FAKE, logp=FAKE, ent=FAKE, topk=0, tl=None, ti=None,
        st=None, ws=FAKE, nbytes=1 << 40):
    return gm.lib().gm_token_logprobs(M, V, dtype, z, ld, T, ids, logp, ent, topk, tl, ti, st, ws, nbytes, None, None)


def test_token_logprobs_rejects():
    A, U = gm.GM_ERR_INVALID_ARG, gm.GM_ERR_UNSUPPORTED
    assert _lp(V=0) == A and _lp(M=-1) == A and _lp(dtype=2) == A and _lp(ld=999) == A
    assert _lp(V=524289, ld=524289) == U and _lp(M=(1 << 23) + 1) == U
    for T in (0.0, -1.0, float("nan"), float("inf")):
        assert _lp(T=T) == A and "temperature" in gm.last_error()
    assert _lp(T=9e-38) == U and _lp(T=1e-45) == U
    assert _lp(z=None) == A and _lp(ids=None) == A
    assert _lp(topk=4, tl=FAKE) == A and _lp(topk=4, ti=FAKE) == A
    assert _lp(topk=0, tl=FAKE, ti=FAKE) == A and _lp(topk=65, tl=FAKE, ti=FAKE) == A
    assert _lp(V=3, ld=3, topk=4, tl=FAKE, ti=FAKE) == A                               # more than there are
    assert _lp(logp=None, ent=None) == A                                               # nothing asked for
    cfg = gm.ModelConfig()
    cfg.vocab = 1000
    need = gm.workspace_size(gm.GM_OP_TOKEN_LOGPROBS, cfg, 8, 4, 0)
    assert need > gm.workspace_size(gm.GM_OP_TOKEN_LOGPROBS, cfg, 8, 0, 0) > 0
    assert _lp(topk=4, tl=FAKE, ti=FAKE, nbytes=need - 1) == gm.GM_ERR_WORKSPACE
    assert gm.workspace_size(gm.GM_OP_TOKEN_LOGPROBS, cfg, 8, 65, 0) == 0
    assert _lp(M=0) == gm.GM_OK


def test_token_logprobs_grad_rejects():
    A, F = gm.GM_ERR_INVALID_ARG, FAKE
    other = ctypes.c_void_p(1 << 21)

    def call(V=1000, dtype=gm.GM_F32, z=F, ld=1000, T=1.0, ids=F, st=F, ent=F, g=F, gh=F, out=other, ldg=1000):
        return gm.lib().gm_token_logprobs_grad(8, V, dtype, z, ld, T, ids, st, ent, g, gh, out, ldg, None)

    assert call(ldg=999) == A and call(ld=999) == A and call(T=0.0) == A and call(dtype=7) == A
    assert call(ids=None) == A and call(g=None) == A and call(ent=None) == A
    assert call(z=None) == A and call(st=None) == A and call(out=None) == A
    assert call(out=F, ldg=1008) == A and "in place" in gm.last_error()
    assert call(V=600000, ld=600000, ldg=600000) == gm.GM_ERR_UNSUPPORTED


def test_binding_rejects_host_tensors_and_shapes():
    cfg = BF16
    cache = type("C", (), dict(B=2, dtype=torch.bfloat16, max_ctx=10))()
    t = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype)  # noqa: E731
    with pytest.raises(ValueError, match="device tensor"):
        gm.kv_append(cfg, cache, 0, t(4, 8, 128), t(4, 8, 128))
    with pytest.raises(ValueError, match="expected"):
        gm.kv_append(cfg, cache, 0, t(4, 8, 64), t(4, 8, 128))
    with pytest.raises(ValueError, match="expected"):
        gm.tree_attention(cfg, cache, 0, t(3, 4, 32, 128), t(3, 4, dtype=torch.int64), t(3, 4, 32, 128), None)
    with pytest.raises(ValueError, match="expected"):
        gm.tree_masks(t(2, 4, dtype=torch.int64), None, None)
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        gm.token_logprobs(t(2, 4, dtype=torch.float16), None, None)
    with pytest.raises(ValueError, match="device tensor"):
        gm.token_logprobs(t(2, 4), None, None)


def test_binding_takes_the_current_device_only(monkeypatch):
    on = lambda d: type("T", (), dict(get_device=lambda self: d, device="cuda:%d" % d))()  # noqa: E731
    stream = lambda d: type("S", (), dict(device_index=d, cuda_stream=77))()  # noqa: E731
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    assert gm._here(stream(1), on(1), None, on(1)) == 77
    with pytest.raises(ValueError, match="the current device is 1"):
        gm._here(stream(1), on(1), on(0))
    with pytest.raises(ValueError, match="a stream of device 0"):
        gm._here(stream(0), on(1))
