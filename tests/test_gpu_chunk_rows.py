"""Chunks of more new tokens than rows: what has no row waits for a later chunk, and
the rows that are there get the attention, keys and summaries of their positions."""
import numpy as np
import pytest
import torch

import oracle
from chunk_cases import f64
from helpers import TOL, assert_close
from paper_2609_13141_amd import inputs, sas
from test_gpu_layer_chunk import CASES, Server, keys_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", list(CASES))
@pytest.mark.parametrize("rows", [1, 37, 64])
def test_prompts_through_chunks_of_fixed_rows(name, rows):
    # a layer over pieces and a whole-prompt layer are each held to TOL against the oracle
    w = CASES[name]
    print(f"\n[case] {rows} rows a chunk, {name}", flush=True)
    x = sas.to_device(inputs.embeddings(w), w.dtype)
    W = sas.weights_to_device(inputs.layer_weights(w), w.dtype)
    cfg = sas.make_config(w, "dense")
    ends = [90, 40, 66] if rows > 1 else [3, 0, 5]
    whole = sas.alloc_cache(cfg, w.batch, w.seq_len)
    ref = sas.layer_forward(cfg, x, W, stats=False, cache=whole)["y"]
    srv = Server(w, cfg, w.seq_len)
    got, at = torch.zeros_like(ref), [0] * w.batch
    while at != ends:
        left = [e - a for a, e in zip(at, ends)]
        given, room = [], rows
        for m in left:
            given.append(min(m, room))
            room -= given[-1]
        xs = torch.cat([x[i, a:a + m] for i, (a, m) in enumerate(zip(at, given))] + [x[0, :room]]).contiguous()
        p = srv.plan(left, rows)
        assert p["kv_len"].tolist() == [a + m for a, m in zip(at, given)]
        y = sas.layer_chunk(cfg, xs, W, srv.cache, srv.ctx, p)
        srv.ctx = p["kv_len"]
        r = 0
        for i, (a, m) in enumerate(zip(at, given)):
            got[i, a:a + m] = y[r:r + m]
            r += m
        at = [a + m for a, m in zip(at, given)]
    torch.cuda.synchronize()
    for i, n in enumerate(ends):
        if n == 0:
            continue
        assert_close(f64(got[i, :n]), f64(ref[i, :n]), w.dtype, f"y of sequence {i}", tol=2 * TOL[w.dtype])
        k, v = keys_of(srv.cache, i, n)
        k0, v0 = keys_of(whole, i, n)
        assert_close(f64(k), f64(k0), w.dtype, "keys", tol=TOL[w.dtype])
        assert_close(f64(v), f64(v0), w.dtype, "values", tol=TOL[w.dtype])
        B = w.block_size
        want = oracle.block_summaries(f64(k), B, w.dtype)
        np.testing.assert_array_equal(f64(srv.cache.k_summary[i, :, :n // B]), want)
