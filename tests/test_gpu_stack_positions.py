"""Positions of a stack's decode steps behind chunks of new tokens: the steps go on
where each sequence ends, and no cached key is written over."""
import pytest
import torch

from chunk_cases import f64
from helpers import TOL, assert_close
from test_gpu_layer_chunk import keys_of, stack, workload

pytestmark = pytest.mark.gpu


def test_steps_go_on_behind_a_ragged_extension():
    w = workload(batch=2, n_heads=4, n_kv_heads=2, head_dim=128, d_model=512, block_size=64, n_layers=2, index=98)
    g = torch.Generator().manual_seed(4)
    text = torch.randint(0, w.vocab, (2, 60), generator=g, dtype=torch.int32).cuda()
    st = stack(w)
    st.prefill(text[:, :40].contiguous())
    assert [p.tolist() for p in st.positions(2)] == [[40, 40], [41, 41]]
    new = [7, 3]
    ids = torch.cat([text[i, 40:40 + m] for i, m in enumerate(new)])
    ctx = torch.full((2,), 40, dtype=torch.int32, device="cuda")
    _, plan = st.extend(ids, ctx, torch.tensor(new, dtype=torch.int32, device="cuda"))
    pos = st.positions(2)
    assert [p.tolist() for p in pos] == [[47, 43], [48, 44]] and all(p.dtype is torch.int32 for p in pos)
    plan["kv_len"].add_(100)      # the plan is the caller's
    before = [keys_of(st.caches[0], i, 40 + m)[0].clone() for i, m in enumerate(new)]
    tok = torch.stack([text[0, 47], text[1, 43]])
    logits = [st.step(tok, pos[0], logits=True)[1]]
    assert [p.tolist() for p in st.positions(1)] == [[48, 44]]
    tok = torch.stack([text[0, 48], text[1, 44]])
    logits.append(st.step(tok, pos[1], logits=True)[1])
    for i, k in enumerate(before):
        assert torch.equal(keys_of(st.caches[0], i, k.shape[0])[0], k)
    # each sequence's logits are those of its own text taken whole
    for i, n in enumerate((49, 45)):
        other = stack(w)
        lg = other.prefill(text[[i, i], :n].contiguous(), logits=True)[1]
        assert other.positions(1)[0].tolist() == [n, n]
        assert_close(f64(logits[1][i]), f64(lg[0]), "bf16", "logits", tol=2 * TOL["bf16"])
