"""sas_attention_chunk against the fp64 oracle over paged caches whose unused
places are NaN: lengths from none to long, ragged batches, head groups, page
sizes, unmapped pages, non-finite values behind the causal mask, padding rows,
divided and undivided work, captured replays, other streams."""
import numpy as np
import pytest
import torch

from chunk_cases import Chunk, check_attention, config, f64
from paper_2609_13141_amd import sas

pytestmark = pytest.mark.gpu


def run(c, cfg, **kw):
    out = sas.attention_chunk(cfg, c.q, c.cache, c.row_start, c.kv_len, **kw)
    torch.cuda.synchronize()
    return out


SHAPES = [
    # ctx, new, H, Hkv, dh, page size, block
    ([0], [1], 4, 4, 64, 16, 16),
    ([0], [5], 4, 2, 128, 16, 64),
    ([63], [1], 2, 2, 128, 16, 64),
    ([64], [1], 2, 2, 128, 16, 64),
    ([1, 200, 0, 77], [1, 1, 1, 1], 4, 4, 128, 16, 64),
    ([100, 0, 513], [4, 0, 5], 28, 4, 128, 16, 64),
    ([300, 17], [150, 33], 14, 2, 128, 16, 64),
    ([0, 31], [130, 257], 4, 4, 64, 8, 16),
    ([33], [70], 6, 1, 64, 1, 16),
    ([90, 5], [40, 129], 8, 1, 128, 128, 128),
    ([1500], [1], 32, 32, 128, 16, 64),
    ([2049, 10], [9, 3], 28, 4, 128, 16, 64),
    ([0, 0, 0], [0, 2, 0], 4, 4, 128, 32, 32),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"ctx{'-'.join(map(str, s[0]))}+{'-'.join(map(str, s[1]))}"
                         f"-{s[2]}x{s[3]}x{s[4]}-p{s[5]}")
def test_against_the_oracle(shape, dtype):
    ctx, new, H, Hkv, dh, ps, B = shape
    print(f"\n[case] chunk attention {shape} {dtype}", flush=True)
    cfg = config(H, Hkv, dh, B, dtype)
    c = Chunk(ctx, new, H, Hkv, dh, ps, B, dtype, seed=len(ctx) + sum(new))
    check_attention(c, run(c, cfg), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_divided_and_undivided_work_agree_with_the_oracle(dtype):
    # no room for parts, room for few, room for all
    cfg = config(4, 2, 128, 64, dtype)
    c = Chunk([3000, 700], [2, 40], 4, 2, 128, 16, 64, dtype, seed=3)
    full = sas.workspace_size(cfg, sas.OP_ATTENTION_CHUNK, 2, c.rows)
    part = 128 * (128 + 2) * 4
    for nbytes in (full, full - 1024 * part, full - 1024 * part + 7 * part):
        print(f"\n[case] workspace {nbytes}", flush=True)
        ws = sas.Workspace("cuda")
        ws.get(nbytes)
        out = {"o": torch.empty_like(c.q), "lse": torch.empty(c.rows, 4, dtype=torch.float32, device="cuda")}
        st = sas.lib().sas_attention_chunk(sas.C.byref(cfg), 2, c.rows, sas._ptr(c.q), sas._ptr(c.row_start),
                                           sas._ptr(c.kv_len), sas.C.byref(c.cache.struct()), sas._ptr(out["o"]),
                                           sas._ptr(out["lse"]), sas._ptr(ws.buf), nbytes, sas._stream())
        assert st == 0
        torch.cuda.synchronize()
        check_attention(c, out, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 60])
def test_unmapped_pages_are_left_out(dtype, new):
    cfg = config(4, 2, 64, 16, dtype)
    # a hole at the start, in the middle, at the end; ids out of range; a sequence with no page at all
    unmap = [(0, 0), (0, 5, 10 ** 6), (1, 3, -7), (1, 4)] + [(2, j) for j in range(40)] + [(3, 1)]
    c = Chunk([200, 100, 150, 20], [new] * 4, 4, 2, 64, 8, 16, dtype, seed=5, unmap=unmap, width=40)
    out = run(c, cfg)
    check_attention(c, out, dtype)
    assert (out["o"][2 * new:3 * new] == 0).all() and torch.isneginf(out["lse"][2 * new:3 * new]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_values_behind_the_mask_do_not_leak(dtype, bad):
    cfg = config(4, 2, 128, 64, dtype)
    c = Chunk([100], [90], 4, 2, 128, 16, 64, dtype, seed=6)
    p, g, d = 150, 1, 77    # position 150 = row 50 of the chunk
    clean = run(c, cfg)["o"].clone()
    page = int(c.cache.block_table[0, p // 16])
    c.cache.v_pages[page, g, p % 16, d] = bad
    c.cache.k_pages[int(c.cache.block_table[0, 180 // 16]), 0, 180 % 16] = bad
    o = run(c, cfg)["o"]
    # kv head 0 up to row 79, kv head 1 up to row 49: untouched, bit for bit
    assert torch.equal(o[:80, :2], clean[:80, :2])
    assert torch.equal(o[:50, 2:], clean[:50, 2:])
    # from there on dimension d of kv head 1 is not finite (the value itself for infinities), the others as before
    got = o[50:, 2:, d].float()
    assert torch.isnan(got).all() if bad != bad else (got == bad).all()
    keep = [e for e in range(128) if e != d]
    assert torch.equal(o[50:, 2:][..., keep], clean[50:, 2:][..., keep])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_padding_rows_are_left_as_they_were(dtype):
    cfg = config(4, 4, 64, 16, dtype)
    c = Chunk([30, 7], [3, 20], 4, 4, 64, 8, 16, dtype, seed=7, pad_rows=41)
    mark = torch.full_like(c.q, 7.0)
    out = run(c, cfg, out=mark)
    check_attention(c, out, dtype)
    assert (out["o"][23:] == 7.0).all()


def test_rows_before_the_first_position_attend_nothing():
    cfg = config(4, 4, 64, 16, "bf16")
    c = Chunk([0], [20], 4, 4, 64, 8, 16, "bf16", seed=8)
    c.kv_len[0] = 13      # rows 0..6 stand before position 0
    out = run(c, cfg)
    assert (out["o"][:7] == 0).all() and torch.isneginf(out["lse"][:7]).all()
    check_attention(c, out, "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_and_lopsided_logits(dtype):
    cfg = config(2, 1, 128, 64, dtype, sm_scale=1.7)
    c = Chunk([700], [33], 2, 1, 128, 16, 64, dtype, seed=9)
    check_attention(c, run(c, cfg), dtype, 1.7)


def test_captured_replays_follow_the_lengths():
    cfg = config(14, 2, 128, 64, "bf16")
    cases = [Chunk([400, 30, 0], [5, 5, 5], 14, 2, 128, 16, 64, "bf16", seed=10, width=60),
             Chunk([77, 500, 3], [5, 0, 2], 14, 2, 128, 16, 64, "bf16", seed=11, width=60, pad_rows=8),
             Chunk([0, 0, 900], [1, 9, 5], 14, 2, 128, 16, 64, "bf16", seed=12, width=60)]
    pool = max(c.cache.k_pages.shape[0] for c in cases)
    k = torch.zeros(pool, 2, 16, 128, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    table = torch.full((3, 60), -1, dtype=torch.int32, device="cuda")
    cache = sas.PagedCache(k, v, table, cases[0].cache.k_summary, 16)
    q = torch.zeros(15, 14, 128, dtype=torch.bfloat16, device="cuda")
    row_start, kv_len = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")

    def load(c):
        n = c.cache.k_pages.shape[0]
        k[:n].copy_(c.cache.k_pages), v[:n].copy_(c.cache.v_pages)
        table.copy_(c.cache.block_table), row_start.copy_(c.row_start), kv_len.copy_(c.kv_len)
        q.copy_(c.q)
    load(cases[0])
    sas.attention_chunk(cfg, q, cache, row_start, kv_len)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = sas.attention_chunk(cfg, q, cache, row_start, kv_len)
    for c in cases + cases[::-1]:
        load(c)
        graph.replay()
        torch.cuda.synchronize()
        check_attention(c, out, "bf16")
        eager = run(c, cfg)
        assert torch.equal(eager["o"][:c.live], out["o"][:c.live])


def test_two_streams_at_once():
    cfg = config(4, 4, 128, 64, "bf16")
    cs = [Chunk([2000], [3], 4, 4, 128, 16, 64, "bf16", seed=20 + s) for s in range(2)]
    want = [run(c, cfg)["o"] for c in cs]
    streams = [torch.cuda.Stream() for _ in cs]
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for c, s in zip(cs, streams):
            with torch.cuda.stream(s):
                got.append(sas.attention_chunk(cfg, c.q, c.cache, c.row_start, c.kv_len)["o"])
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_same_bits_every_time():
    cfg = config(28, 4, 128, 64, "bf16")
    c = Chunk([1200, 40], [6, 70], 28, 4, 128, 16, 64, "bf16", seed=30)
    first = run(c, cfg)
    for _ in range(3):
        again = run(c, cfg)
        assert torch.equal(first["o"], again["o"]) and torch.equal(first["lse"], again["lse"])


def test_a_whole_prompt_equals_the_prefill_attention():
    cfg = config(8, 2, 128, 64, "bf16")
    c = Chunk([0], [300], 8, 2, 128, 16, 64, "bf16", seed=31)
    pg = c.cache.block_table[0, torch.arange(300, device="cuda") // 16].long()
    at = torch.arange(300, device="cuda") % 16
    k, v = c.cache.k_pages[pg, :, at][None].contiguous(), c.cache.v_pages[pg, :, at][None].contiguous()
    dense = sas.attention_prefill(cfg, c.q[None], k, v)
    out = run(c, cfg)
    # both round P and o to bf16 and sum in other orders
    scale = np.abs(f64(v)).max()
    assert np.abs(f64(out["o"]) - f64(dense["o"])[0]).max() <= 2.0 ** -7 * scale
    assert np.abs(f64(out["lse"]) - f64(dense["lse"])[0].T).max() <= 1e-4
