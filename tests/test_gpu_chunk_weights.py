"""Chunk attention of few rows keeps its weights: outputs that cancel to nearly nothing
are as exact as the fp32 sums allow, like those of the decode step.

The weights reach the second product within 2^-16 (a bf16 number and the bf16 rest of
it, half a step of 2^-7 each); logits are off by (dh + 4) 2^-24 sum |q||k| sm, the
exponential by as much again, sums of n weighted values by 2^-24 (n / 8 + 64); then one
rounding of the result, 2^-8 of it."""
import numpy as np
import pytest
import torch

from chunk_cases import Chunk, config, f64
from paper_2609_13141_amd import sas

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("ctx,new,H,Hkv,dh,ps", [
    ([1], [1], 32, 32, 128, 16), ([30, 7, 100, 3], [1, 1, 1, 1], 28, 4, 128, 16), ([60, 20], [5, 3], 14, 2, 128, 16),
    ([40, 90], [4, 1], 8, 8, 64, 16), ([700], [1], 4, 4, 128, 16), ([50], [90], 4, 2, 128, 8)])
def test_single_tokens_and_drafts(ctx, new, H, Hkv, dh, ps):
    print(f"\n[case] {ctx}+{new} {H}x{Hkv}x{dh} pages of {ps}", flush=True)
    cfg = config(H, Hkv, dh, 64, "bf16")
    c = Chunk(ctx, new, H, Hkv, dh, ps, 64, "bf16", seed=110)
    c.q *= 0.25
    got = f64(sas.attention_chunk(cfg, c.q, c.cache, c.row_start, c.kv_len)["o"])
    o, _, A, Z = c.reference()
    n = max(c + m for c, m in zip(ctx, new))
    dz = ((dh + 4) * 2.0 ** -24 * Z)[..., None] + 2.0 ** -21
    w = 2.0 ** -16 + 2.0 * dz + 2.0 ** -24 * (n / 8 + 64)
    bound = A * w + 2.0 ** -8 * np.abs(o) * (1 + w) + 1e-30
    bad = ~(np.abs(got - o) <= bound)
    assert not bad.any(), (int(bad.sum()), bad.size, float((np.abs(got - o) / bound).max()))
