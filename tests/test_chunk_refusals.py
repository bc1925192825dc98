"""The chunk entry points refuse what they cannot do before anything is launched
(host only: every call here fails its checks)."""
import ctypes as C
import os

import pytest
import torch

from chunk_cases import config
from paper_2609_13141_amd import sas

P = 0x1000
BAD, UNSUP, WS = sas.SAS_ERR_INVALID_ARGUMENT, sas.SAS_ERR_UNSUPPORTED, sas.SAS_ERR_WORKSPACE


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(sas.LIB_PATH):
        pytest.skip("libsas.so not built")
    return sas.lib()


def kv(**kw):
    f = dict(k_pages=P, v_pages=P, block_table=P, k_summary=P, num_pages=8, page_size=16, max_pages_per_seq=8,
             max_blocks=2)
    f.update(kw)
    return sas.PagedKV(*[f[n] for n, _ in sas.PagedKV._fields_])


def plan(L, b=2, rows=8, cache=None, capacity=4, ins=None, outs=None):
    i = dict(ctx_len=P, new_len=P, pages_held=P, free_pages=P, free_count=P)
    i.update(ins or {})
    o = {f: 0x2000 + 16 * n for n, (f, _) in enumerate(sas.PlanOut._fields_)}
    o.update(outs or {})
    pi = sas.PlanIn(*[i[f] for f, _ in sas.PlanIn._fields_[:5]], capacity)
    po = sas.PlanOut(*[o[f] for f, _ in sas.PlanOut._fields_])
    return L.sas_plan_chunk(b, rows, C.byref(pi), C.byref(cache or kv()), C.byref(po), None)


@pytest.mark.parametrize("kw,status,word", [
    (dict(b=0), BAD, b"batch"), (dict(rows=0), BAD, b"rows"), (dict(b=4097), UNSUP, b"4096"),
    (dict(capacity=-1), BAD, b"capacity"), (dict(ins=dict(ctx_len=None)), BAD, b"ctx_len"),
    (dict(ins=dict(free_pages=None)), BAD, b"free_pages"), (dict(ins=dict(new_len=0x1002)), BAD, b"aligned"),
    (dict(outs=dict(slot=None)), BAD, b"out.slot"), (dict(outs=dict(pages_held=P)), BAD, b"out.pages_held is"),
    (dict(cache=kv(page_size=24)), UNSUP, b"page_size"), (dict(cache=kv(page_size=256)), UNSUP, b"page_size"),
    (dict(cache=kv(num_pages=0)), BAD, b"geometry"), (dict(cache=kv(block_table=None)), BAD, b"block_table"),
])
def test_plan(L, kw, status, word):
    assert plan(L, **kw) == status
    assert word in L.sas_last_error()


def rotary(axes=1, section=(64, 0, 0), pos=P, gain_q=P, gain_k=P):
    return sas.Rotary(gain_q, gain_k, pos, axes, (C.c_int32 * 3)(*section))


def qkv(q=P, k=P, v=P, qs=0, ks=0, vs=0):
    return sas.Qkv(q, k, v, qs, ks, vs)


QK = [
    (dict(rows=0), BAD, b"rows"), (dict(rot=rotary(axes=0)), BAD, b"axes"), (dict(rot=rotary(axes=4)), BAD, b"axes"),
    (dict(rot=rotary(section=(63, 0, 0))), BAD, b"pairs"), (dict(rot=rotary(3, (65, -1, 0))), BAD, b"section"),
    (dict(rot=rotary(pos=None)), BAD, b"rot.pos"), (dict(rot=rotary(gain_k=0x1004)), BAD, b"aligned"),
    (dict(x=qkv(q=None)), BAD, b"in.q"), (dict(x=qkv(qs=8)), BAD, b"q_stride"), (dict(x=qkv(ks=261)), BAD, b"k_stride"),
    (dict(x=qkv(qs=-512)), BAD, b"q_stride"), (dict(rows=2 ** 30), UNSUP, b"2^30"),
    (dict(rows=2 ** 27, cfg=dict(n_heads=2)), UNSUP, b"2^25 rows"), (dict(x=qkv(qs=2 ** 61)), BAD, b"q_stride"),
    (dict(cfg=dict(rope_base=0.0)), BAD, b"rope_base"), (dict(cfg=dict(rms_eps=-1.0)), BAD, b"rms_eps"),
    (dict(cfg=dict(head_dim=96)), UNSUP, b"head_dim"), (dict(rot=None), BAD, b"NULL"),
]


def qk_cfg(kw):
    cfg = config(4, 2, 128)
    for k, v in kw.get("cfg", {}).items():
        setattr(cfg, k, v)
    return cfg


@pytest.mark.parametrize("kw,status,word", QK)
def test_norm_and_rotation(L, kw, status, word):
    cfg = qk_cfg(kw)
    rot, x, rows = kw.get("rot", rotary()), kw.get("x", qkv()), kw.get("rows", 4)
    ref = C.byref(rot) if rot is not None else None
    assert L.sas_qk_norm_rope(C.byref(cfg), rows, ref, C.byref(x), 0x2000, 0x3000, None) == status
    assert word in L.sas_last_error()
    assert L.sas_qk_norm_rope_backward(C.byref(cfg), rows, ref, C.byref(x), P, P, 0x2000, 0x3000, P, P, P, 1 << 30,
                                       None) == status
    assert L.sas_cache_append(C.byref(cfg), 2, rows, ref, C.byref(x), P, P, P, None, C.byref(kv()), 0x2000,
                              None) == status


def test_norm_and_rotation_outputs(L):
    cfg, rot = config(4, 2, 128), rotary()
    fwd = lambda x, q, k: L.sas_qk_norm_rope(C.byref(cfg), 4, C.byref(rot), C.byref(x), q, k, None)  # noqa: E731
    assert fwd(qkv(), None, P) == BAD and fwd(qkv(), P, None) == BAD
    assert fwd(qkv(qs=1024), P, 0x3000) == BAD and b"q_out is its input" in L.sas_last_error()
    bwd = lambda r, *a: L.sas_qk_norm_rope_backward(C.byref(cfg), 4, C.byref(r), C.byref(qkv()), P, P, *a, None)  # noqa: E731
    assert bwd(rot, 0x2000, 0x3000, None, P, P, 1 << 30) == BAD and b"dgain_q" in L.sas_last_error()
    assert bwd(rotary(gain_q=None), 0x2000, 0x3000, P, P, P, 1 << 30) == BAD
    assert bwd(rot, P, 0x3000, P, P, P, 1 << 30) == BAD and b"input" in L.sas_last_error()
    assert bwd(rot, 0x2000, 0x3000, P, P, None, 0) == WS
    assert bwd(rot, 0x2000, 0x3000, P, P, P, 16) == WS


def test_append(L):
    cfg, rot, x = config(4, 2, 128), rotary(), qkv()
    call = lambda b=2, rows=4, x=x, slot=P, cl=P, kl=P, cache=kv(), q=0x2000: L.sas_cache_append(  # noqa: E731
        C.byref(cfg), b, rows, C.byref(rot), C.byref(x), slot, cl, kl, None, C.byref(cache) if cache else None, q, None)
    assert call(b=0) == BAD and call(b=4097) == UNSUP
    assert call(slot=None) == BAD and call(cl=None) == BAD and call(kl=None) == BAD and call(q=None) == BAD
    assert call(x=qkv(v=None)) == BAD and call(x=qkv(vs=4)) == BAD and call(cache=None) == BAD
    assert call(cache=kv(page_size=48)) == BAD and call(cache=kv(k_pages=None)) == BAD
    assert call(cache=kv(max_blocks=8193)) == UNSUP


def test_attention(L):
    cfg = config(4, 2, 128)
    call = lambda cfg=cfg, b=2, rows=4, q=P, rs=P, kl=P, cache=kv(), o=P, ws=P, n=1 << 30: L.sas_attention_chunk(  # noqa: E731
        C.byref(cfg), b, rows, q, rs, kl, C.byref(cache) if cache else None, o, None, ws, n, None)
    assert call(b=0) == BAD and call(rows=0) == BAD and call(b=4097) == UNSUP
    for k in ("q", "rs", "kl", "cache", "o"):
        assert call(**{k: None}) == BAD
    assert call(q=0x1008) == BAD and b"aligned" in L.sas_last_error()
    assert call(cfg=config(129, 1, 64)) == UNSUP and b"per KV head" in L.sas_last_error()
    assert call(cache=kv(max_pages_per_seq=2 ** 26 + 1)) == UNSUP and b"positions" in L.sas_last_error()
    assert call(cache=kv(page_size=12)) == BAD
    assert call(rows=2 ** 29) == UNSUP
    assert call(ws=None) == WS and call(n=64) == WS
    assert call() == BAD and b"o is q" in L.sas_last_error()   # (q and o are both P)
    assert sas.workspace_size(cfg, sas.OP_ATTENTION_CHUNK, 4097, 1) == 0
    assert 0 < sas.workspace_size(cfg, sas.OP_ATTENTION_CHUNK, 4096, 1) < 70 << 20


def test_verify(L):
    vi = dict(target=P, draft=P, tokens=P, draft_start=P, u_accept=P, u_sample=P)
    def call(b=2, rows=4, V=10, D=3, out=P, acc=P, ws=P, n=1 << 20, **kw):
        v = sas.VerifyIn(*[{**vi, **kw}[f] for f, _ in sas.VerifyIn._fields_])
        return L.sas_verify_drafts(b, rows, V, D, C.byref(v), out, acc, ws, n, None)
    assert call(b=0) == BAD and call(rows=-1) == BAD and call(V=0) == BAD and call(D=-1) == BAD
    assert call(b=4097) == UNSUP and call(V=2 ** 30 + 1) == UNSUP
    for k in ("target", "tokens", "draft_start", "u_accept", "u_sample", "out", "acc"):
        assert call(**{k: None}) == BAD
    assert call(draft=0x1001) == BAD
    assert call(V=65537, ws=None) == WS and call(V=65537, n=4095) == WS
    assert L.sas_workspace_size(None, sas.OP_VERIFY_DRAFTS, 2, 65537) == 4096
    assert L.sas_workspace_size(None, sas.OP_VERIFY_DRAFTS, 2, 65536) == 0
    assert L.sas_workspace_size(None, sas.OP_VERIFY_DRAFTS, 128, 65537) == 0
    assert L.sas_workspace_size(None, sas.OP_ATTENTION_CHUNK, 3, 4) == 0


def test_layer(L):
    cfg = config(4, 2, 128)
    W = sas.LayerWeights(*([P] * 9 + [None, None, None]))
    ch = dict(row_start=P, ctx_len=P, kv_len=P, slot=P)

    def call(cfg=cfg, b=2, rows=4, x=P, W=W, rot=rotary(), cache=kv(), y=0x2000, ws=P, n=1 << 30, **kw):
        c = sas.Chunk(*[{**ch, **kw}[f] for f, _ in sas.Chunk._fields_])
        return L.sas_layer_chunk(C.byref(cfg), b, rows, x, C.byref(W), C.byref(rot) if rot else None, C.byref(c),
                                 C.byref(cache) if cache else None, y, ws, n, None)
    assert call(b=0) == BAD and call(rows=0) == BAD and call(b=5000) == UNSUP
    for k in ("x", "y", "cache", "row_start", "ctx_len", "kv_len", "slot", "rot"):
        assert call(**{k: None}) == BAD, k
    assert call(W=sas.LayerWeights()) == BAD and b"w.rms1" in L.sas_last_error()
    assert call(rot=rotary(section=(3, 0, 0))) == BAD and call(cache=kv(page_size=48)) == BAD
    assert call(ws=None) == WS and call(n=4096) == WS
    assert sas.workspace_size(cfg, sas.OP_LAYER_CHUNK, 2, 0) == 0


def test_the_binding_refuses_host_tensors():
    t = torch.zeros(4, 4, 128, dtype=torch.bfloat16)
    i = torch.zeros(4, dtype=torch.int32)
    cfg = config(4, 2, 128)
    with pytest.raises(sas.SasError, match="not a tensor on the GPU"):
        sas.qk_norm_rope(cfg, t, t[:, :2], i)
    with pytest.raises(sas.SasError, match="not a tensor on the GPU"):
        sas.plan_chunk(None, i, i, i, i, i[:1], 4)
    with pytest.raises(sas.SasError, match="not a tensor on the GPU"):
        sas.verify_drafts(t[0].float(), None, i, i, i, i, 4)


def test_the_binding_refuses_rows_that_overlap():
    cfg, cpu = config(4, 2, 128), torch.device("cpu")
    t = torch.zeros(1, 4, 128, dtype=torch.bfloat16)
    for x in (t.expand(5, 4, 128), torch.zeros(2048, dtype=torch.bfloat16).as_strided((5, 4, 128), (256, 128, 1))):
        with pytest.raises(sas.SasError, match="do not overlap"):
            sas._heads_arg(cfg, "q", x, 4, 5, cpu)
    assert sas._heads_arg(cfg, "q", t, 4, 1, cpu)[1] == 512


@pytest.mark.parametrize("n,least", [(-1, 0), (0, 1), (2 ** 31, 0), (2 ** 32 + 5, 1)])
def test_counts_fit_the_arguments(n, least):
    with pytest.raises(sas.SasError, match="from"):
        sas._count("rows", n, least)
