"""sas_qk_norm_rope and its backward against the fp64 oracle, and
sas_cache_append's pages and summaries.

Bounds: one rounding to the type (HALF relative) plus the fp32 arithmetic.  A
normed element n = x r g carries the errors of the sum of squares (half of
(dh / 16 + 6) 2^-24 relative), of sqrt, division and two products: below 2^-21
relative; the rotation adds 2^-24 per operation and the angle's 2^-22 (its
fraction of a turn in fp32, times 2 pi, and sincospi's rounding).  Together
2^-20 of |n_i| + |n_{i + dh/2}|."""
import numpy as np
import pytest
import torch

import oracle
from chunk_cases import DT, HALF, Chunk, config, f64
from paper_2609_13141_amd import sas

pytestmark = pytest.mark.gpu
BASE, EPS = 10000.0, 1e-6


def pairs(x):
    """|x_i| + |x_{i + dh/2}| at both places."""
    a = np.abs(x)
    h = a.shape[-1] // 2
    s = a[..., :h] + a[..., h:]
    return np.concatenate([s, s], axis=-1)


def close(got, want, lim, what):
    bad = ~(np.abs(f64(got) - want) <= lim)
    assert not bad.any(), (what, np.argwhere(bad)[:3], f64(got)[bad][:3], want[bad][:3], lim[bad][:3])


def inputs(rows, H, Hkv, dh, dtype, axes, seed, packed):
    g = torch.Generator().manual_seed(seed)
    mk = lambda *s, std=1.0: (torch.randn(*s, generator=g) * std).to(DT[dtype]).cuda()  # noqa: E731
    if packed:
        qkv = mk(rows, (H + 2 * Hkv) * dh, std=1.3)
        q = qkv[:, :H * dh].view(rows, H, dh)
        k = qkv[:, H * dh:(H + Hkv) * dh].view(rows, Hkv, dh)
        v = qkv[:, (H + Hkv) * dh:].view(rows, Hkv, dh)
    else:
        q, k, v = mk(rows, H, dh, std=2.0), mk(rows, Hkv, dh, std=0.5), mk(rows, Hkv, dh)
    sections = {1: None, 2: (dh // 8, dh // 2 - dh // 8), 3: (0, dh // 4, dh // 4)}[axes]
    pos = torch.randint(0, 600000, (axes, rows), generator=g, dtype=torch.int32)
    pos[0, 0] = 0
    pos[-1, -1] = -17
    gq, gk = (1 + mk(dh, std=0.3).float()).to(DT[dtype]), (1 + mk(dh, std=0.3).float()).to(DT[dtype])
    return q, k, v, pos.cuda(), gq, gk, sections


CASES = [(1, 4, 4, 64, 1), (3, 28, 4, 128, 3), (130, 32, 32, 128, 1), (77, 5, 1, 64, 2), (1000, 14, 2, 128, 3),
         (9, 3, 3, 128, 1), (31, 128, 1, 64, 1)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=str)
@pytest.mark.parametrize("normed", ["qk", "q", "none"])
def test_forward(case, dtype, normed):
    rows, H, Hkv, dh, axes = case
    print(f"\n[case] norm+rope {case} {dtype} {normed}", flush=True)
    q, k, _, pos, gq, gk, sec = inputs(rows, H, Hkv, dh, dtype, axes, rows, packed=rows % 2 == 1)
    gq, gk = (gq if "q" in normed else None), (gk if normed == "qk" else None)
    qo, ko = sas.qk_norm_rope(config(H, Hkv, dh, dtype=dtype), q, k, pos, gq, gk, sections=sec)
    torch.cuda.synchronize()
    for x, g, y, what in ((q, gq, qo, "q"), (k, gk, ko, "k")):
        want = oracle.chunk.norm_rope(f64(x), None if g is None else f64(g), pos.cpu().numpy(), sec or (dh // 2,), BASE, EPS)
        close(y, want, HALF[dtype] * np.abs(want) + 2.0 ** -20 * pairs(want) + 1e-37, what)


def test_forward_in_place():
    cfg = config(28, 4, 128)
    q, k, _, pos, gq, gk, sec = inputs(50, 28, 4, 128, "bf16", 3, 5, packed=False)
    want = sas.qk_norm_rope(cfg, q, k, pos, gq, gk, sections=sec)
    rot = sas._rotary(cfg, pos, gq, gk, sec, 50, q.device)
    st = sas.lib().sas_qk_norm_rope(sas.C.byref(cfg), 50, sas.C.byref(rot),
                                    sas.C.byref(sas.Qkv(sas._ptr(q), sas._ptr(k), None, 0, 0, 0)), sas._ptr(q),
                                    sas._ptr(k), sas._stream())
    assert st == 0
    torch.cuda.synchronize()
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])


def test_zero_rows_and_zero_heads_of_zeros():
    cfg = config(4, 2, 64, dtype="f32")
    z = torch.zeros(3, 4, 64, device="cuda")
    pos = torch.arange(3, dtype=torch.int32, device="cuda")
    g = torch.ones(64, device="cuda")
    q, k = sas.qk_norm_rope(cfg, z, z[:, :2].contiguous(), pos, g, g)
    assert (q == 0).all() and (k == 0).all()
    q, k = sas.qk_norm_rope(cfg, z[:0], z[:0, :2].contiguous(), pos[:0], g, g)
    assert q.shape == (0, 4, 64) and k.shape == (0, 2, 64)
    d = sas.qk_norm_rope_backward(cfg, z[:0], z[:0, :2].contiguous(), pos[:0], q, k, g, g)
    assert (d["dgain_q"] == 0).all() and d["dq"].shape == (0, 4, 64)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES + [(5000, 8, 2, 128, 3)], ids=str)
@pytest.mark.parametrize("normed", ["qk", "k", "none"])
def test_backward(case, dtype, normed):
    rows, H, Hkv, dh, axes = case
    print(f"\n[case] norm+rope backward {case} {dtype} {normed}", flush=True)
    q, k, _, pos, gq, gk, sec = inputs(rows, H, Hkv, dh, dtype, axes, rows + 1, packed=rows % 2 == 1)
    gq, gk = (gq if "q" in normed else None), (gk if "k" in normed else None)
    g = torch.Generator().manual_seed(7)
    dq, dk = (torch.randn(rows, n, dh, generator=g).to(DT[dtype]).cuda() for n in (H, Hkv))
    cfg = config(H, Hkv, dh, dtype=dtype)
    out = sas.qk_norm_rope_backward(cfg, q, k, pos, dq, dk, gq, gk, sections=sec)
    again = sas.qk_norm_rope_backward(cfg, q, k, pos, dq, dk, gq, gk, sections=sec)
    torch.cuda.synchronize()
    assert sorted(out) == sorted(["dq", "dk"] + (["dgain_q"] if gq is not None else []) + (["dgain_k"] if gk is not None else []))
    for f in out:
        assert torch.equal(out[f], again[f]), f
    for x, gain, dy, f in ((q, gq, dq, "q"), (k, gk, dk, "k")):
        args = (f64(x), None if gain is None else f64(gain), pos.cpu().numpy(), sec or (dh // 2,), BASE, EPS)
        dx, dg = oracle.chunk.norm_rope_backward(*args, f64(dy))
        if gain is None:
            close(out["d" + f], dx, HALF[dtype] * np.abs(dx) + 2.0 ** -20 * pairs(f64(dy)) + 1e-37, "d" + f)
            continue
        # r (g dn - x k): the pieces' sizes, k a mean over dh products
        xa = f64(x)
        r = 1.0 / np.sqrt(np.mean(xa * xa, axis=-1, keepdims=True) + EPS)
        dn = pairs(f64(dy)) * np.abs(f64(gain))
        size = r * (dn + np.abs(xa) * r * r * np.mean(dn * np.abs(xa), axis=-1, keepdims=True))
        close(out["d" + f], dx, HALF[dtype] * np.abs(dx) + 2.0 ** -19 * size + 1e-37, "d" + f)
        # a lane adds rows * heads / (its share) terms in fp32: at most `chain` of them in a row
        terms = np.abs(pairs(f64(dy)) * xa * r).sum(axis=(0, 1))
        chain = 16 + rows * (H + Hkv) / 1024
        close(out["dgain_" + f], dg, (2.0 ** -20 + chain * 2.0 ** -24) * terms + 1e-37, "dgain_" + f)


def test_gradients_against_differences():
    # the kernel's own forward, differenced in fp32 along random directions
    cfg = config(4, 2, 64, dtype="f32")
    q, k, _, pos, gq, gk, sec = inputs(6, 4, 2, 64, "f32", 3, 3, packed=False)
    g = torch.Generator().manual_seed(1)
    dq, dk = (torch.randn(6, n, 64, generator=g).cuda() for n in (4, 2))
    out = sas.qk_norm_rope_backward(cfg, q, k, pos, dq, dk, gq, gk, sections=sec)
    def loss(*a):
        y = sas.qk_norm_rope(cfg, a[0], a[1], pos, a[2], a[3], sections=sec)
        return float((y[0].double() * dq.double()).sum() + (y[1].double() * dk.double()).sum())
    args = [q, k, gq, gk]
    for n, f in enumerate(("dq", "dk", "dgain_q", "dgain_k")):
        d = torch.randn(args[n].shape, generator=g).cuda()
        h = 2.0 ** -7
        up, down = ([a if i != n else (a + s * h * d) for i, a in enumerate(args)] for s in (1, -1))
        # steps as they are after rounding
        step = (up[n].double() - down[n].double())
        want = float((out[f].double() * step).sum())
        diff = loss(*up) - loss(*down)
        # outputs round to 2^-24 of about |y| ~ 3 at each of the 6 * 6 * 64 places, against gradients of size 1;
        # the third-order term is some h^2 of the slope
        err = 2 * 2.0 ** -24 * 3 * 6 * 6 * 64 + 4 * h * h * float((out[f].abs().double() * step.abs()).sum())
        assert abs(diff - want) <= err, (f, diff, want, err)


# ---- append ------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", [
    ([0], [1], 4, 4, 64, 8, 16, 1), ([63, 5, 127], [1, 1, 1], 32, 32, 128, 16, 64, 1),
    ([0, 100, 63, 64], [64, 0, 200, 63], 28, 4, 128, 16, 64, 3), ([31, 2], [33, 300], 4, 2, 64, 1, 32, 2),
    ([100], [300], 8, 1, 128, 128, 128, 1)], ids=str)
@pytest.mark.parametrize("proj", [False, True])
def test_append(case, dtype, proj):
    ctx, new, H, Hkv, dh, ps, B, axes = case
    print(f"\n[case] append {case} {dtype} proj={proj}", flush=True)
    # holes: a page of the cached part and, in long chunks, one of the new part
    unmap = [(0, 1)] if ctx[0] + new[0] > 2 * ps else []
    c = Chunk(ctx, new, H, Hkv, dh, ps, B, dtype, seed=sum(new), unmap=unmap)
    cfg = config(H, Hkv, dh, B, dtype)
    rows = c.rows
    q, k, v, pos, gq, gk, sec = inputs(rows, H, Hkv, dh, dtype, axes, rows, packed=True)
    table = c.cache.block_table.cpu().numpy()
    num = c.cache.k_pages.shape[0]
    slot = np.array([(lambda pg, p: pg * ps + p % ps if pg >= 0 else -1)(oracle.chunk.page_of(table, i, p, ps, num), p)
                     for i in range(len(ctx)) for p in range(ctx[i], ctx[i] + new[i])], dtype=np.int64)
    if rows > 2:
        slot[2] = num * ps    # outside the pool: dropped
    w_gk = (torch.eye(dh)[None] + 0.05 * torch.randn(Hkv, dh, dh)).to(DT[dtype]).cuda() if proj else None
    kp0, vp0 = c.cache.k_pages.clone(), c.cache.v_pages.clone()
    ks0 = c.cache.k_summary.normal_().clone()
    qo = sas.cache_append(cfg, c.cache, q, k, v, pos, torch.tensor(slot, device="cuda"), c.ctx_len, c.kv_len, gq, gk,
                          sections=sec, w_gk=w_gk)
    torch.cuda.synchronize()
    wq, wk = sas.qk_norm_rope(cfg, q, k, pos, gq, gk, sections=sec)   # checked above
    assert torch.equal(qo, wq)
    ok = (slot >= 0) & (slot < num * ps)
    rr = torch.tensor(np.nonzero(ok)[0], device="cuda")
    pg, at = torch.tensor(slot[ok] // ps, device="cuda"), torch.tensor(slot[ok] % ps, device="cuda")
    kp0[pg, :, at] = wk[rr]
    vp0[pg, :, at] = v[rr]
    same = lambda a, b: torch.equal(torch.nan_to_num(a, nan=12345.0), torch.nan_to_num(b, nan=12345.0))  # noqa: E731
    assert same(c.cache.k_pages, kp0) and same(c.cache.v_pages, vp0)
    want = oracle.chunk.completed_summaries(f64(kp0), table, ctx, [a + b for a, b in zip(ctx, new)], B,
                                            ks0.shape[2], dtype, None if w_gk is None else f64(w_gk))
    for (i, m), s in want.items():
        np.testing.assert_array_equal(f64(c.cache.k_summary[i, :, m]), s)
        ks0[i, :, m] = c.cache.k_summary[i, :, m]
    assert torch.equal(c.cache.k_summary, ks0)


def test_append_of_many_sequences():
    b, ps, B = 700, 16, 16
    cfg = config(2, 1, 64, B)
    rng = np.random.default_rng(0)
    ctx, new = rng.integers(0, 40, size=b), rng.integers(0, 4, size=b)
    c = Chunk(ctx.tolist(), new.tolist(), 2, 1, 64, ps, B, "bf16", seed=1)
    q, k, v, pos, gq, gk, sec = inputs(c.rows, 2, 1, 64, "bf16", 1, 2, packed=False)
    seq = np.repeat(np.arange(b), new)
    p = np.concatenate([np.arange(a, a + m) for a, m in zip(ctx, new)])
    table = c.cache.block_table.cpu().numpy()
    slot = torch.tensor(table[seq, p // ps].astype(np.int64) * ps + p % ps, device="cuda")
    sas.cache_append(cfg, c.cache, q, k, v, pos, slot, c.ctx_len, c.kv_len, gq, gk, sections=sec)
    torch.cuda.synchronize()
    want = oracle.chunk.completed_summaries(f64(c.cache.k_pages), table, ctx, ctx + new, B, 10 ** 6, "bf16")
    assert want
    got = f64(c.cache.k_summary)
    for (i, m), s in want.items():
        np.testing.assert_array_equal(got[i, :, m], s)
        got[i, :, m] = 0
    assert (got == 0).all()
