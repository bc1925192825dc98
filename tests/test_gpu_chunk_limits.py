"""The chunk operators where their work is divided otherwise (many sequences,
more jobs than the chip holds at once) and where offsets pass 32 bits."""
import numpy as np
import pytest
import torch

import oracle
from chunk_cases import Chunk, check_attention, config, f64
from paper_2609_13141_amd import sas

pytestmark = pytest.mark.gpu


def run(c, cfg, **kw):
    out = sas.attention_chunk(cfg, c.q, c.cache, c.row_start, c.kv_len, **kw)
    torch.cuda.synchronize()
    return out


def ragged(b, ctx_hi, new_lo, new_hi, seed, long=0):
    rng = np.random.default_rng(seed)
    ctx, new = rng.integers(0, ctx_hi + 1, size=b), rng.integers(new_lo, new_hi + 1, size=b)
    new[-1] = new_hi
    if long:
        ctx[b // 3] = long
    return ctx.tolist(), new.tolist()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name,lens,H,Hkv,dh", [
    ("divided by a kernel", ragged(65, 90, 0, 3, 1), 2, 1, 64),
    ("one far longer than the rest", ragged(65, 90, 1, 2, 2, long=5000), 4, 2, 128),
    ("more jobs than workgroups", ragged(70, 200, 1, 1, 3, long=3000), 8, 8, 128),
    ("more jobs than workgroups, long rows", ragged(70, 100, 10, 50, 4), 32, 8, 128),
    ("more jobs than workgroups, long rows of 64", ragged(70, 100, 10, 50, 5), 32, 8, 64),
    ("64 sequences of all the workgroups", ragged(64, 60, 1, 1, 6), 8, 8, 64),
    ("all 4096 sequences", ragged(4096, 40, 0, 1, 7), 2, 1, 64),
    ("one prompt of many tiles", ([0], [1030]), 64, 64, 64),
], ids=lambda x: x.replace(" ", "-") if isinstance(x, str) else "")
def test_attention_of_many_jobs(name, lens, H, Hkv, dh, dtype):
    print(f"\n[case] {name} {dtype}", flush=True)
    c = Chunk(*lens, H, Hkv, dh, 16, 16, dtype, seed=40)
    cfg = config(H, Hkv, dh, 16, dtype)
    out = run(c, cfg)
    check_attention(c, out, dtype)
    again = run(c, cfg)
    assert torch.equal(out["o"], again["o"]) and torch.equal(out["lse"], again["lse"])


def test_captured_replays_of_the_job_queues():
    cfg = config(8, 8, 128, 16, "bf16")
    c = Chunk(*ragged(70, 200, 1, 1, 3, long=3000), 8, 8, 128, 16, 16, "bf16", seed=41)
    want = run(c, cfg)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = sas.attention_chunk(cfg, c.q, c.cache, c.row_start, c.kv_len)
    for _ in range(4):
        out["o"].zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out["o"], want["o"]) and torch.equal(out["lse"], want["lse"])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ps,new", [(16, 3), (16, 90), (8, 40), (4, 3), (4, 90), (2, 3), (2, 90)])
def test_pools_past_4_gib(dtype, ps, new):
    """The same pages at the two ends of a pool larger than 2^32 bytes: the same bits."""
    H, Hkv, dh, B = 16, 16, 128, 64
    cfg = config(H, Hkv, dh, B, dtype)
    c = Chunk([200, 75], [new, 5], H, Hkv, dh, ps, B, dtype, seed=42)
    small = c.cache
    q, k, v = [torch.randn(c.rows, h, dh, device="cuda").to(c.q.dtype) for h in (H, Hkv, Hkv)]
    seq = np.repeat([0, 1], [new, 5])
    pos = np.concatenate([200 + np.arange(new), 75 + np.arange(5)])
    row = torch.tensor(seq, device="cuda"), torch.tensor(pos // ps, device="cuda")
    pos_d, at = torch.tensor(pos, dtype=torch.int32, device="cuda"), torch.tensor(pos % ps, device="cuda")
    n = small.k_pages.shape[0]
    num = (9 << 29) // (Hkv * ps * dh * c.q.element_size()) + n
    big = sas.PagedCache(torch.zeros(num, Hkv, ps, dh, dtype=c.q.dtype, device="cuda"),
                         torch.zeros(num, Hkv, ps, dh, dtype=c.q.dtype, device="cuda"),
                         small.block_table.clone(), small.k_summary.clone(), ps)
    t = big.block_table
    t[t >= 0] = torch.where(t[t >= 0] % 2 == 1, num - n + t[t >= 0], t[t >= 0])
    ids = torch.arange(n, device="cuda")
    ids = torch.where(ids % 2 == 1, num - n + ids, ids)
    big.k_pages[ids], big.v_pages[ids] = small.k_pages, small.v_pages
    assert (num - 1) * Hkv * ps * dh * c.q.element_size() > 2 ** 32
    outs = []
    for cache in (small, big):
        slot = cache.block_table[row].long() * ps + at
        qo = sas.cache_append(cfg, cache, q, k, v, pos_d, slot, c.ctx_len, c.kv_len)
        outs.append((qo, *sas.attention_chunk(cfg, qo, cache, c.row_start, c.kv_len).values(), cache.k_summary))
    torch.cuda.synchronize()
    c.q = outs[0][0]
    check_attention(c, {"o": outs[0][1], "lse": outs[0][2]}, dtype)
    for a, b in zip(*outs):
        assert torch.equal(a, b)
    same = lambda a, b: torch.equal(torch.nan_to_num(a, nan=12345.0), torch.nan_to_num(b, nan=12345.0))  # noqa: E731
    assert same(big.k_pages[ids], small.k_pages) and same(big.v_pages[ids], small.v_pages)


def test_rows_far_apart():
    """Rows of a packed projection 2^21 elements apart: offsets past 2^32 elements."""
    H, Hkv, dh, rows, stride = 2, 1, 64, 2100, 1 << 21
    cfg = config(H, Hkv, dh)
    far = torch.empty(rows, stride, dtype=torch.bfloat16, device="cuda")
    q = far[:, :H * dh].view(rows, H, dh)
    k = far[:, -Hkv * dh:].view(rows, Hkv, dh)
    q.copy_(torch.randn(rows, H, dh, device="cuda")), k.copy_(torch.randn(rows, Hkv, dh, device="cuda"))
    assert (rows - 1) * stride > 2 ** 32
    pos = torch.arange(rows, dtype=torch.int32, device="cuda")
    g = torch.ones(dh, dtype=torch.bfloat16, device="cuda")
    dq, dk = torch.randn(rows, H, dh, device="cuda").bfloat16(), torch.randn(rows, Hkv, dh, device="cuda").bfloat16()
    for a, b in zip(sas.qk_norm_rope(cfg, q, k, pos, g, g),
                    sas.qk_norm_rope(cfg, q.contiguous(), k.contiguous(), pos, g, g)):
        assert torch.equal(a, b)
    far_g = sas.qk_norm_rope_backward(cfg, q, k, pos, dq, dk, g, g)
    near = sas.qk_norm_rope_backward(cfg, q.contiguous(), k.contiguous(), pos, dq, dk, g, g)
    for n in near:
        assert torch.equal(far_g[n], near[n]), n


@pytest.mark.parametrize("V,rows", [(32000, 70000), (100003, 22000)])
def test_probabilities_past_2_31_elements(V, rows):
    # a long draft whose first token is refused, and a short one at the far end
    b, m = 2, 3
    start = torch.tensor([0, rows - m, rows], dtype=torch.int32)
    target = torch.zeros(rows + b, V, device="cuda")
    draft = torch.zeros(rows, V, device="cuda")
    assert draft.numel() > 2 ** 31
    g = torch.Generator().manual_seed(50)
    p = torch.softmax(torch.randn(m + 1, V, generator=g), 1)
    q = torch.softmax(p[:m].log() + 0.1 * torch.randn(m, V, generator=g), 1)
    target[-(m + 1):], draft[-m:], target[0] = p.cuda(), q.cuda(), p[0].cuda()
    tok = torch.multinomial(q, 1, generator=g)[:, 0].int()
    tokens, u_accept = torch.full((rows,), -1, dtype=torch.int32), torch.zeros(rows)
    tokens[-m:], u_accept[-m:] = tok, torch.rand(m, generator=g)
    us = torch.rand(2, generator=g)
    out = sas.verify_drafts(target, draft, tokens.cuda(), start.cuda(), u_accept.cuda(), us.cuda(), rows)
    torch.cuda.synchronize()
    first, _ = oracle.chunk.verify_drafts(p[:1].numpy(), None, [], [0, 0], [], us[:1].numpy(), m)
    last, acc = oracle.chunk.verify_drafts(p.numpy(), q.numpy(), tok.numpy(), [0, m], u_accept[-m:].numpy(), us[1:].numpy(), m)
    got = out["tokens"].cpu().numpy()
    np.testing.assert_array_equal(got[:, :m + 1], np.concatenate([first, last]))
    assert (got[:, m + 1:] == -1).all()
    np.testing.assert_array_equal(out["accepted"].cpu().numpy(), [0, acc[0]])


def test_two_captured_backwards_on_two_streams():
    """Each call has scratch of its own: two captured backward passes replayed at
    once, and an eager one between them, give the bits of eager calls."""
    cfg = config(6, 2, 128)
    sets = []
    for seed, rows in ((60, 900), (61, 333)):
        g = torch.Generator().manual_seed(seed)
        mk = lambda *s: torch.randn(*s, generator=g).bfloat16().cuda()  # noqa: E731
        pos = torch.randint(0, 9000, (rows,), generator=g, dtype=torch.int32).cuda()
        sets.append((mk(rows, 6, 128), mk(rows, 2, 128), pos, mk(rows, 6, 128), mk(rows, 2, 128), mk(128), mk(128)))
    want = [sas.qk_norm_rope_backward(cfg, *s) for s in sets]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for s in sets:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append((sas.qk_norm_rope(cfg, *s[:3], *s[5:]), sas.qk_norm_rope_backward(cfg, *s)))
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(4):
        for (_, o), graph, st in zip(outs, graphs, streams):
            with torch.cuda.stream(st):
                for t in o.values():
                    t.zero_()
                graph.replay()
        eager = sas.qk_norm_rope_backward(cfg, *sets[0])
        torch.cuda.synchronize()
        for n in want[0]:
            assert torch.equal(eager[n], want[0][n]), n
        for (f, o), w, s in zip(outs, want, sets):
            for n in w:
                assert torch.equal(o[n], w[n]), n
            for a, b in zip(f, sas.qk_norm_rope(cfg, *s[:3], *s[5:])):
                assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ramp", ["up", "down", "jump", "late"])
def test_logits_that_grow_with_the_position(dtype, ramp):
    """The running maximum moves on many tiles, on one by more than fp32 exponentials
    reach, or never again."""
    cfg = config(4, 2, 128, 64, dtype)
    c = Chunk([700, 90], [200, 150], 4, 2, 128, 16, 64, dtype, seed=70)
    p = torch.arange(900, device="cuda", dtype=torch.float32)
    w = {"up": p / 60, "down": (900 - p) / 60, "jump": torch.where(p < 333, 0.01, 40.0),
         "late": torch.where(p < 690, 0.0, 60.0)}[ramp].to(c.q.dtype)
    for i, n in ((0, 900), (1, 240)):
        at = torch.arange(n, device="cuda")
        pg = c.cache.block_table[i, at // 16].long()
        c.cache.k_pages[pg, :, at % 16] *= w[at][:, None, None]
    check_attention(c, run(c, cfg), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh,ps", [(128, 16), (64, 16), (128, 32), (64, 64), (128, 128)])
def test_long_chunks_over_pages_that_are_missing(dtype, dh, ps):
    """Holes (entry -1, or no page of the pool) before and inside the chunk, at its
    first and last page, a sequence without any page, and a block table that ends
    before the last tokens' positions."""
    B = max(ps, 64)
    cfg = config(4, 2, dh, B, dtype)
    n = 32 // (ps // 16)
    unmap = [(0, 0), (0, n // 2, 10 ** 6), (0, n), (1, 1, -5), (1, 2)] + [(2, j) for j in range(60)]
    c = Chunk([400, 100, 150, 333], [250, 170, 200, 205], 4, 2, dh, ps, B, dtype, seed=80, unmap=unmap, width=128)
    check_attention(c, run(c, cfg), dtype)
    short = -(-480 // ps)
    c.cache.block_table = c.cache.block_table[:, :short].contiguous()
    check_attention(c, run(c, cfg), dtype)
