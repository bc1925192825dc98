"""The chunk operators together, as a server uses them: pages handed out, a layer
over ragged chunks into the paged cache (sas_layer_chunk), sparse decoding behind
it, a stack's logits and the verification of drafted tokens.  Prompts taken in
pieces have to give what they give taken whole.

A layer over pieces rounds Q and K once more than sas_layer_forward (before the
rotation) and sums in other orders; both are held to the activation tolerance of the
oracle tests, so that two of them differ by at most twice that."""
import numpy as np
import pytest
import torch

import oracle
from chunk_cases import f64
from helpers import TOL, assert_close
from paper_2609_13141_amd import configs, inputs, model, sas

pytestmark = pytest.mark.gpu


def workload(**kw):
    base = dict(name="chunk", dtype="bf16", batch=3, seq_len=200, d_model=256, n_heads=4, n_kv_heads=2, head_dim=64,
                d_ff=512, block_size=16, top_k=32, mode="sparse", segments=(), index=95, vocab=500)
    base.update(kw)
    n = base["seq_len"]
    base["segments"] = (("img", n // 2), ("txt", n - n // 2))
    return configs.Workload(**base)


CASES = {
    "mha-dh64": workload(),
    "gqa7-dh128": workload(n_heads=7, n_kv_heads=1, head_dim=128, d_model=896, d_ff=640, block_size=64, index=96),
    "f32": workload(dtype="f32", index=97),
}


class Server:
    """Requests' lengths and pages on the device, as a serving loop keeps them."""

    def __init__(self, w, cfg, max_len, ps=16, seed=0):
        self.w, self.cfg = w, cfg
        self.cache = sas.alloc_cache(cfg, w.batch, max_len, page_size=ps, seed=seed)
        self.cache.block_table.fill_(-1)
        num = self.cache.k_pages.shape[0]
        self.free = torch.randperm(num, generator=torch.Generator().manual_seed(seed)).to(torch.int32).cuda()
        self.count = torch.tensor([num], dtype=torch.int32, device="cuda")
        self.held = torch.zeros(w.batch, dtype=torch.int32, device="cuda")
        self.ctx = torch.zeros(w.batch, dtype=torch.int32, device="cuda")

    def plan(self, new, rows=None):
        p = sas.plan_chunk(self.cache, self.ctx, torch.tensor(new, dtype=torch.int32, device="cuda"), self.held,
                           self.free, self.count, rows or sum(new))
        self.held, self.count = p["pages_held"], p["free_count"]
        return p

    def layer(self, x, W, new, **kw):
        p = self.plan(new, x.shape[0])
        y = sas.layer_chunk(self.cfg, x, W, self.cache, self.ctx, p, **kw)
        self.ctx = p["kv_len"]
        return y


def pieces(w, ends):
    """Row counts of every sequence in each round until all reach `ends`."""
    rng = np.random.default_rng(w.index)
    at = [0] * w.batch
    while at != ends:
        new = [int(min(e - a, rng.choice([0, 1, 5, 17, 64, 90]))) for a, e in zip(at, ends)]
        if sum(new):
            yield at, new
            at = [a + m for a, m in zip(at, new)]


def keys_of(cache, i, n):
    ps = cache.page_size
    p = torch.arange(n, device="cuda")
    pg = cache.block_table[i, p // ps].long()
    return cache.k_pages[pg, :, p % ps], cache.v_pages[pg, :, p % ps]


@pytest.mark.parametrize("name", list(CASES))
def test_prompts_in_pieces_equal_whole_prompts(name):
    w = CASES[name]
    print(f"\n[case] layer over pieces {name}", flush=True)
    x = sas.to_device(inputs.embeddings(w), w.dtype)
    W = sas.weights_to_device(inputs.layer_weights(w), w.dtype)
    cfg = sas.make_config(w, "dense")
    ends = [w.seq_len, 131, 77]
    whole = sas.alloc_cache(cfg, w.batch, w.seq_len)
    ref = sas.layer_forward(cfg, x, W, stats=False, cache=whole)["y"]
    srv = Server(w, cfg, w.seq_len + 20)
    got = torch.zeros_like(ref)
    for at, new in pieces(w, ends):
        pad = 3
        xs = torch.cat([x[i, a:a + m] for i, (a, m) in enumerate(zip(at, new))] + [x[0, :pad]])
        y = srv.layer(xs.contiguous(), W, new)
        r = 0
        for i, (a, m) in enumerate(zip(at, new)):
            got[i, a:a + m] = y[r:r + m]
            r += m
    torch.cuda.synchronize()
    assert srv.ctx.tolist() == ends
    B = w.block_size
    for i, n in enumerate(ends):
        assert_close(f64(got[i, :n]), f64(ref[i, :n]), w.dtype, f"y of sequence {i}", tol=2 * TOL[w.dtype])
        k, v = keys_of(srv.cache, i, n)
        k0, v0 = keys_of(whole, i, n)
        assert_close(f64(k), f64(k0), w.dtype, "keys", tol=TOL[w.dtype])
        assert_close(f64(v), f64(v0), w.dtype, "values", tol=TOL[w.dtype])
        want = oracle.block_summaries(f64(k), B, w.dtype)
        np.testing.assert_array_equal(f64(srv.cache.k_summary[i, :, :n // B]), want)
    # the next token by the sparse decode step (all blocks kept), behind pieces and behind whole prompts
    n = 77
    pos = torch.full((1,), n, dtype=torch.int32, device="cuda")
    dec = sas.make_config(w, "sparse")
    out = []
    for cache, i in ((srv.cache, 2), (whole, 2)):
        one = sas.PagedCache(cache.k_pages, cache.v_pages, cache.block_table[i:i + 1].clone(),
                             cache.k_summary[i:i + 1].clone(), cache.page_size)
        if cache is srv.cache:
            srv.plan([0, 0, 1])     # a page for the new token
            one.block_table = srv.cache.block_table[i:i + 1].clone()
        out.append(sas.decode_step(dec, x[2, n:n + 1].clone(), pos, W, one)[0])
    assert_close(f64(out[0]), f64(out[1]), w.dtype, "decode step", tol=2 * TOL[w.dtype])


def test_norms_and_axes_against_the_oracle():
    w = CASES["gqa7-dh128"]
    H, Hkv, dh, d = w.n_heads, w.n_kv_heads, w.head_dim, w.d_model
    x = sas.to_device(inputs.embeddings(w), "bf16")
    Wn = inputs.layer_weights(w)
    W = sas.weights_to_device(Wn, "bf16")
    g = torch.Generator().manual_seed(0)
    gq, gk = ((1 + 0.2 * torch.randn(dh, generator=g)).bfloat16().cuda() for _ in range(2))
    sec = (16, 24, 24)
    pos = torch.randint(0, 3000, (3, 60), generator=g, dtype=torch.int32).cuda()
    cfg = sas.make_config(w.with_(batch=1), "dense")
    srv = Server(w.with_(batch=1), cfg, 100)
    y = torch.cat([srv.layer(x[0, a:b].contiguous(), W, [b - a], pos=pos[:, a:b].contiguous(), gain_q=gq, gain_k=gk,
                             sections=sec) for a, b in ((0, 41), (41, 42), (42, 60))])
    torch.cuda.synchronize()
    X = f64(x[0, :60])
    W64 = {k: None if v is None else f64(v) for k, v in W.items()}
    rho = oracle.round_bf16
    u = rho(oracle.rmsnorm(X, W64["rms1"], w.rms_eps))
    qkv = [rho(u @ W64[f].T).reshape(60, n, dh) for f, n in (("wq", H), ("wk", Hkv), ("wv", Hkv))]
    q = rho(oracle.chunk.norm_rope(qkv[0], f64(gq), f64(pos), sec, w.rope_base, w.rms_eps))
    k = rho(oracle.chunk.norm_rope(qkv[1], f64(gk), f64(pos), sec, w.rope_base, w.rms_eps))
    o = oracle.sas_attention(q, k, qkv[2], w.block_size, "dense", "bf16")[0]
    h1 = rho(X + o.reshape(60, H * dh) @ W64["wo"].T)
    u2 = rho(oracle.rmsnorm(h1, W64["rms2"], w.rms_eps))
    a = rho(oracle.silu(u2 @ W64["w_gate"].T) * (u2 @ W64["w_up"].T))
    assert_close(f64(y), rho(h1 + a @ W64["w_down"].T), "bf16", "y")


def test_a_captured_server_step_follows_the_lengths():
    w = CASES["mha-dh64"]
    x = sas.to_device(inputs.embeddings(w), "bf16")
    W = sas.weights_to_device(inputs.layer_weights(w), "bf16")
    cfg = sas.make_config(w, "dense")
    rows = 24
    xs, new = x[0, :rows].contiguous(), torch.tensor([5, 0, 9], dtype=torch.int32, device="cuda")
    srv = Server(w, cfg, w.seq_len)

    def step():
        p = sas.plan_chunk(srv.cache, srv.ctx, new, srv.held, srv.free, srv.count, rows)
        return sas.layer_chunk(cfg, xs, W, srv.cache, srv.ctx, p), p
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, p = step()
    state = [torch.empty_like(t) for t in (srv.cache.k_pages, srv.cache.v_pages, srv.cache.k_summary, srv.cache.block_table)]
    live = [srv.cache.k_pages, srv.cache.v_pages, srv.cache.k_summary, srv.cache.block_table]
    for t in live[:3]:
        t.zero_()
    live[3].fill_(-1)
    for m in ([5, 0, 9], [1, 1, 1], [20, 4, 0], [0, 3, 0], [8, 8, 8]):
        new.copy_(torch.tensor(m, dtype=torch.int32))
        xs.copy_(x[m[0] % 3, :rows])
        for a, b in zip(state, live):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        after = [t.clone() for t in live]
        got = y.clone()
        for a, b in zip(state, live):
            b.copy_(a)
        want, q = step()
        torch.cuda.synchronize()
        assert torch.equal(got[:sum(m)], want[:sum(m)])
        for a, b in zip(after, live):
            assert torch.equal(a, b)
        srv.ctx.copy_(q["kv_len"]), srv.held.copy_(q["pages_held"]), srv.count.copy_(q["free_count"])


def stack(w, seed=1):
    g = torch.Generator().manual_seed(seed)
    layers = [sas.weights_to_device(inputs.layer_weights(w, layer=i), w.dtype) for i in range(2)]
    ends = {"embed": torch.randn(w.vocab, w.d_model, generator=g).bfloat16().cuda(),
            "w_lm": (torch.randn(w.vocab, w.d_model, generator=g) * 0.1).bfloat16().cuda(),
            "rms_final": torch.ones(w.d_model, dtype=torch.bfloat16, device="cuda")}
    return model.Stack(w, layers, ends, max_len=w.seq_len)


def test_drafted_tokens_through_a_stack():
    # drafts verified by one chunk get the logits of single steps, and the verification is the oracle's
    w = workload(batch=2, n_heads=4, n_kv_heads=2, head_dim=128, d_model=512, block_size=64, n_layers=2, index=98)
    g = torch.Generator().manual_seed(3)
    prompt = torch.randint(0, w.vocab, (2, 90), generator=g, dtype=torch.int32).cuda()
    one, many = stack(w), stack(w)
    tok = one.prefill(prompt)
    assert torch.equal(tok, many.prefill(prompt))
    drafts = torch.randint(0, w.vocab, (2, 4), generator=g, dtype=torch.int32).cuda()
    counts = [4, 2]
    want, t = [], tok
    for s in range(5):
        pos = torch.full((2,), 90 + s, dtype=torch.int32, device="cuda")
        want.append(one.step(t, pos, logits=True)[1])
        t = drafts[:, min(s, 3)].contiguous()
    ids = torch.cat([torch.cat([tok[i:i + 1], drafts[i, :m]]) for i, m in enumerate(counts)] + [tok[:1]])
    ctx = torch.full((2,), 90, dtype=torch.int32, device="cuda")
    x, plan = many.extend(ids, ctx, torch.tensor([m + 1 for m in counts], dtype=torch.int32, device="cuda"))
    assert plan["kv_len"].tolist() == [95, 93] and plan["pos"].tolist() == [90, 91, 92, 93, 94, 90, 91, 92, -1]
    lg = many.logits(x[:8])
    rows = [(0, s) for s in range(5)] + [(1, s) for s in range(3)]
    ref = torch.stack([want[s][i] for i, s in rows])
    assert_close(f64(lg), f64(ref), "bf16", "logits", tol=2 * TOL["bf16"])
    p = torch.softmax(lg, 1)
    start = torch.tensor([0, 4, 6], dtype=torch.int32, device="cuda")
    flat = torch.cat([drafts[0, :4], drafts[1, :2]])
    q = torch.softmax(torch.randn(6, w.vocab, generator=g), 1).cuda()
    for seed in range(4):
        u = torch.rand(8, generator=torch.Generator().manual_seed(seed)).cuda()
        u[:6] *= 10.0 ** -seed
        out = sas.verify_drafts(p, q, flat, start, u[:6].clone(), u[6:].clone(), 4)
        torch.cuda.synchronize()
        wt, wa = oracle.chunk.verify_drafts(*[t.cpu().numpy() for t in (p, q, flat, start, u[:6], u[6:])], 4)
        np.testing.assert_array_equal(out["tokens"].cpu().numpy(), wt)
        np.testing.assert_array_equal(out["accepted"].cpu().numpy(), wa)


@pytest.mark.parametrize("part", ["none", "some"])
def test_less_scratch(part):
    w = CASES["mha-dh64"].with_(batch=1)
    x = sas.to_device(inputs.embeddings(w), "bf16")[0]
    W = sas.weights_to_device(inputs.layer_weights(w), "bf16")
    cfg = sas.make_config(w, "dense")
    full = sas.workspace_size(cfg, sas.OP_LAYER_CHUNK, 1, 7)
    ys = []
    for less in (0, 1):
        srv = Server(w, cfg, w.seq_len)
        srv.layer(x[:180].contiguous(), W, [180])
        p = srv.plan([7])
        opt = 131072 * 66 * 4   # the part for divided attention, which is the largest at this size
        n = full - less * (opt if part == "none" else opt // 3)
        buf = torch.empty(n, dtype=torch.uint8, device="cuda")
        y = torch.empty(7, w.d_model, dtype=torch.bfloat16, device="cuda")
        rot = sas._rotary(cfg, p["pos"], None, None, None, 7, y.device)
        ch = sas.Chunk(*[sas._ptr(t) for t in (p["row_start"], srv.ctx, p["kv_len"], p["slot"])])
        kv = srv.cache.struct()
        xs = x[180:187].contiguous()
        st = sas.lib().sas_layer_chunk(sas.C.byref(cfg), 1, 7, sas._ptr(xs), sas.C.byref(sas.weights_struct(W)),
                                       sas.C.byref(rot), sas.C.byref(ch), sas.C.byref(kv), sas._ptr(y), sas._ptr(buf), n,
                                       sas._stream())
        assert st == 0, sas.lib().sas_last_error()
        torch.cuda.synchronize()
        ys.append(y)
    assert_close(f64(ys[1]), f64(ys[0]), "bf16", "y", tol=2 * TOL["bf16"])
