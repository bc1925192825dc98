"""The angles of the rotation are fp64 up to the last rounding: turned unit vectors give
cos and sin themselves, whose error near their zeros is that of the angle.

sin and cos of the fp32 fraction are right within 2 units of 2^-23 relative, the step
from there to the fp64 fraction adds a rounding and, by second order, 2^-48; a fp64
angle of up to 12000 rad is off by a few 2^-53 of it, below 2^-36."""
import numpy as np
import pytest
import torch

from chunk_cases import config, f64
from paper_2609_13141_amd import sas

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dh", [64, 128])
def test_cosines_and_sines(dh):
    rows, half = 12000, dh // 2
    cfg = config(2, 1, dh, 64, "f32")
    q = torch.zeros(rows, 2, dh, device="cuda")
    q[:, 0, :half] = 1.0
    q[:, 1, half:] = 1.0
    pos = torch.arange(rows, dtype=torch.int32, device="cuda")
    got = sas.qk_norm_rope(cfg, q, q[:, :1].contiguous(), pos)
    ang = np.arange(rows)[:, None] * np.power(10000.0, -2.0 * np.arange(half) / dh)
    c, s = np.cos(ang), np.sin(ang)
    want = np.stack([np.concatenate([c, s], 1), np.concatenate([-s, c], 1)], 1)
    back = sas.qk_norm_rope_backward(cfg, q, q[:, :1].contiguous(), pos, q, q[:, :1].contiguous())
    wback = np.stack([np.concatenate([c, -s], 1), np.concatenate([s, c], 1)], 1)
    for g, w in ((got[0], want), (got[1], want[:, :1]), (back["dq"], wback), (back["dk"], wback[:, :1])):
        over = np.abs(f64(g) - w) / (3 * 2.0 ** -23 * np.abs(w) + 2.0 ** -36)
        assert over.max() <= 1.0, float(over.max())
