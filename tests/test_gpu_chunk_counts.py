"""Sizes past 2^31 of a dimension whose count is a 32-bit argument of the library: the
binding refuses them (taken modulo 2^32, 2^32 + 5 tokens would be 5)."""
import pytest
import torch

from chunk_cases import Chunk, config
from paper_2609_13141_amd import sas

pytestmark = pytest.mark.gpu


def test_vocabularies_past_32_bits():
    target = torch.empty(1, 2 ** 32 + 5, device="cuda")
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    start = torch.zeros(2, dtype=torch.int32, device="cuda")
    with pytest.raises(sas.SasError, match="vocab"):
        sas.verify_drafts(target, None, none, start, torch.empty(0, device="cuda"), torch.zeros(1, device="cuda"), 0)


def test_block_tables_past_32_bits():
    cfg = config(4, 2, 64, 16)
    c = Chunk([20], [3], 4, 2, 64, 16, 16)
    wide = torch.empty(1, 2 ** 32 + 8, dtype=torch.int32, device="cuda")
    cache = sas.PagedCache(c.cache.k_pages, c.cache.v_pages, wide, c.cache.k_summary, 16)
    one = torch.ones(1, dtype=torch.int32, device="cuda")
    slot = torch.zeros(3, dtype=torch.int64, device="cuda")
    pos = torch.arange(3, dtype=torch.int32, device="cuda")
    kv = torch.randn(3, 2, 64, device="cuda").bfloat16()
    for call in (lambda: sas.plan_chunk(cache, c.ctx_len, one, one, one, one, 3),
                 lambda: sas.cache_append(cfg, cache, c.q, kv, kv, pos, slot, c.ctx_len, c.kv_len),
                 lambda: sas.attention_chunk(cfg, c.q, cache, c.row_start, c.kv_len)):
        with pytest.raises(sas.SasError, match="pages of a sequence"):
            call()
