"""Paged caches and chunks for the tests of the chunk operators.  Every place of
the pool that holds no cached token is NaN, so that a read of one shows."""
import numpy as np
import torch

import oracle
from paper_2609_13141_amd import configs, sas

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}   # relative rounding error of the types


def config(H, Hkv, dh, B=64, dtype="bf16", **kw):
    w = configs.TINY.with_(n_heads=H, n_kv_heads=Hkv, head_dim=dh, block_size=B, dtype=dtype, mode="dense")
    return sas.make_config(w, "dense", **kw)


def f64(t):
    return t.detach().double().cpu().numpy()


class Chunk:
    """Sequences of ctx cached and new tokens; `unmap` lists (sequence, page index)
    entries to set to -1 (or to the given value)."""

    def __init__(self, ctx, new, H, Hkv, dh, ps=16, B=64, dtype="bf16", seed=0, unmap=(), pad_rows=0, spare_pages=2,
                 width=None, device="cuda"):
        g = torch.Generator().manual_seed(seed)
        self.rng = np.random.default_rng(seed + 1)
        self.ctx, self.new, self.ps, self.B = list(ctx), list(new), ps, B
        b = len(ctx)
        kv = [c + m for c, m in zip(ctx, new)]
        per = [-(-n // ps) for n in kv]
        width = max(width or 0, -(-max(max(per) * ps, 1) // B) * (B // ps))
        num = sum(per) + spare_pages
        order = torch.randperm(num, generator=g).to(torch.int32)
        table = torch.full((b, width), -1, dtype=torch.int32)
        k = torch.full((num, Hkv, ps, dh), float("nan"), dtype=DT[dtype])
        v = torch.full_like(k, float("nan"))
        at = 0
        for i in range(b):
            table[i, :per[i]] = order[at:at + per[i]]
            at += per[i]
            p = torch.arange(kv[i])
            pg = table[i, p // ps].long()
            for pool in (k, v):
                pool[pg, :, p % ps] = torch.randn(kv[i], Hkv, dh, generator=g).to(DT[dtype])
        for i, j, *val in unmap:
            table[i, j] = val[0] if val else -1
        self.rows = sum(new) + pad_rows
        start = np.concatenate([[0], np.cumsum(new)])
        self.row_start = torch.tensor(start, dtype=torch.int32, device=device)
        self.kv_len = torch.tensor(kv, dtype=torch.int32, device=device)
        self.ctx_len = torch.tensor(ctx, dtype=torch.int32, device=device)
        self.q = (torch.randn(self.rows, H, dh, generator=g) * 1.5).to(DT[dtype]).to(device)
        self.cache = sas.PagedCache(k.to(device), v.to(device), table.to(device),
                                    torch.zeros(b, Hkv, width * ps // B, dh, dtype=DT[dtype], device=device), ps)
        self.live = sum(new)

    def reference(self, sm_scale=None):
        c = self.cache
        return oracle.chunk.attention_chunk(f64(self.q), f64(c.k_pages), f64(c.v_pages), c.block_table.cpu().numpy(),
                                            self.row_start.cpu().numpy(), self.kv_len.cpu().numpy(), sm_scale)


def check_attention(case, out, dtype, sm_scale=None):
    """o and lse within what the arithmetic allows: logits summed in fp32 over dh
    products (dz <= (dh + 4) 2^-24 sum |q||k| sm), weights rounded to the type for the second
    product, fp32 sums over up to n keys, one rounding of the result."""
    o, lse, A, Z = case.reference(sm_scale)
    live = case.live
    dh = o.shape[-1]
    n = max(int(case.kv_len.max()), 1)
    dz = ((dh + 4) * 2.0 ** -24 * Z[:live])[..., None] + 2.0 ** -21
    u = HALF[dtype]
    # weights' rounding and exponent error, then the fp32 sums of up to n weighted values
    w = (u if dtype == "bf16" else 0.0) + 2.0 * dz + 2.0 ** -24 * (n / 8 + 64)
    bound = A[:live] * w + u * np.abs(o[:live]) * (1 + w) + 1e-30
    got = f64(out["o"])[:live]
    bad = ~(np.abs(got - o[:live]) <= bound)
    assert not bad.any(), ("o", np.argwhere(bad)[:4], got[bad][:4], o[:live][bad][:4], bound[bad][:4])
    if "lse" in out:
        gl = f64(out["lse"])[:live]
        none = np.isneginf(lse[:live])
        assert np.array_equal(np.isneginf(gl), none)
        err = np.abs(gl[~none] - lse[:live][~none])
        lim = (2.0 * dz[..., 0] + 2.0 ** -24 * (n / 8 + 64))[~none] + 2.0 ** -22 * np.abs(lse[:live][~none]) + 2.0 ** -22
        assert (err <= lim).all(), ("lse", (err - lim).max())
