"""Scratch that a captured graph writes to stays the graph's when the workspace grows:
replays write to nothing that was allocated since."""
import pytest
import torch

from chunk_cases import Chunk, check_attention, config
from paper_2609_13141_amd import sas
from test_gpu_layer_chunk import stack, workload

pytestmark = pytest.mark.gpu


def strangers(nbytes):
    """Tensors where an allocator would put memory of that size that was given back."""
    return [torch.full((n,), 7, dtype=torch.uint8, device="cuda") for n in (nbytes, nbytes, nbytes // 2, nbytes // 4)]


def test_a_larger_call_after_the_capture():
    cfg = config(4, 2, 128, 64, "bf16")
    c = Chunk([900, 70], [3, 40], 4, 2, 128, 16, 64, "bf16", seed=100)
    ws = sas.Workspace()
    sas.attention_chunk(cfg, c.q, c.cache, c.row_start, c.kv_len, ws=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = sas.attention_chunk(cfg, c.q, c.cache, c.row_start, c.kv_len, ws=ws)
    buf = ws.buf
    at, n = buf.data_ptr(), buf.numel()
    del buf
    ws.get(3 * n)
    others = strangers(n)
    assert ws.buf.data_ptr() != at and all(t.data_ptr() != at for t in others)
    for _ in range(3):
        out["o"].zero_()
        graph.replay()
        torch.cuda.synchronize()
        check_attention(c, out, "bf16")
        assert all((t == 7).all() for t in others)


def test_a_long_prompt_after_a_captured_extension():
    w = workload(batch=2, n_heads=4, n_kv_heads=2, head_dim=128, d_model=512, block_size=64, n_layers=2, index=98)
    g = torch.Generator().manual_seed(5)
    text = torch.randint(0, w.vocab, (2, 200), generator=g, dtype=torch.int32).cuda()
    st = stack(w)
    st.prefill(text[:, :20].contiguous())
    ids = torch.cat([text[0, 20:24], text[1, 20:23], text[0, :1]])
    ctx, new = (torch.tensor(a, dtype=torch.int32, device="cuda") for a in ([20, 20], [4, 3]))
    want = st.extend(ids, ctx, new)[0]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x, _ = st.extend(ids, ctx, new)
    n = st.ws.buf.numel()
    st.ws.get(2 * n + 4096)      # as a longer prompt would
    others = strangers(n)
    st.prefill(text[:, :20].contiguous())
    for _ in range(3):
        x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(x[:7], want[:7])
        assert all((t == 7).all() for t in others)
