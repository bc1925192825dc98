"""Row offsets that break the rules (sequences over the same rows), with more jobs
than 31 bits count: the call ends, in bounds."""
import pytest
import torch

from chunk_cases import Chunk, check_attention, config
from paper_2609_13141_amd import sas

pytestmark = pytest.mark.gpu


def test_more_jobs_than_31_bits():
    # 2048 sequences of all the rows: 2048 * 32 heads * rows / 128 jobs
    H, dh, rows, b = 32, 64, (1 << 22) + 128, 4096
    assert 2048 * H * (rows // 128) > 2 ** 31
    cfg = config(H, H, dh, 16)
    c = Chunk([20, 0], [3, 7], H, H, dh, 16, 16)
    table = torch.zeros(b, 64, dtype=torch.int32, device="cuda")
    s = c.cache.k_summary
    cache = sas.PagedCache(c.cache.k_pages, c.cache.v_pages, table, s.new_zeros(b, H, 64, dh), 16)
    start = torch.tensor([0, rows] * (b // 2) + [0], dtype=torch.int32, device="cuda")
    kv = torch.full((b,), 30, dtype=torch.int32, device="cuda")
    q, out = (torch.empty(rows, H, dh, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    sas.attention_chunk(cfg, q, cache, start, kv, lse=False, out=out)
    torch.cuda.synchronize()
    r = sas.attention_chunk(cfg, c.q, c.cache, c.row_start, c.kv_len)
    torch.cuda.synchronize()
    check_attention(c, r, "bf16")
