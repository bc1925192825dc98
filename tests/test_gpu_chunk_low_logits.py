"""Chunk attention where every logit lies far below zero, so that exponentials of the
logits themselves underflow (fp32: below -87), behind keys without a page: the rows
still attend what is there."""
import pytest
import torch

from chunk_cases import Chunk, check_attention, config
from paper_2609_13141_amd import sas

pytestmark = pytest.mark.gpu


def low(c, cfg, lo, hi, seed):
    """Logits of about lo .. hi (negative), a key's the same for every row."""
    g = torch.Generator().manual_seed(seed)
    H, dh = c.q.shape[1:]
    u = torch.randn(dh, generator=g).sign()
    c.q.copy_(u + 0.05 * torch.randn(c.rows, H, dh, generator=g))
    for i, (ctx, new) in enumerate(zip(c.ctx, c.new)):
        p = torch.arange(ctx + new)
        a = (lo + (hi - lo) * torch.rand(ctx + new, generator=g)) / dh ** 0.5
        at = p.cuda()
        pg = c.cache.block_table[i, at // c.ps].long()
        keep = pg >= 0
        k = a[:, None, None] * u + 0.05 * torch.randn(ctx + new, c.cache.k_pages.shape[1], dh, generator=g)
        c.cache.k_pages[pg[keep], :, at[keep] % c.ps] = k.cuda().to(c.q.dtype)[keep]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("span", [(-100, -100), (-300, -100), (-130, -88), (-20000, -10000)], ids=str)
@pytest.mark.parametrize("dh,ps", [(128, 16), (64, 32), (128, 8)])
@pytest.mark.parametrize("holes", ["the first keys", "the first half of every tile", "whole tiles", "no keys"])
def test_rows_behind_missing_pages(dtype, span, dh, ps, holes):
    # long chunks (the pipelined loop in bf16, pages of 16 or more), drafts, one of a single row
    print(f"\n[case] {dtype} {span} {dh} {ps} {holes}", flush=True)
    B = 64
    cfg = config(4, 2, dh, B, dtype)
    lens = [700, 0, 130, 64], [250, 150, 90, 1]
    width = 1024 // ps
    at = [32 * j for j in range(32)]
    keys = {"the first keys": at[:1] + [64], "the first half of every tile": at[::2], "whole tiles": at[:2] + at[6:9],
            "no keys": []}[holes]
    unmap = [(i, (p + o) // ps) for i in range(4) for p in keys for o in range(0, 32, ps)]
    if holes == "the first keys":     # and sequence 0's long stretch of them
        unmap += [(0, j) for j in range(400 // ps)]
    c = Chunk(*lens, 4, 2, dh, ps, B, dtype, seed=90, unmap=unmap, width=width)
    low(c, cfg, *span, seed=91)
    out = sas.attention_chunk(cfg, c.q, c.cache, c.row_start, c.kv_len)
    torch.cuda.synchronize()
    check_attention(c, out, dtype)
