"""Chunks of new tokens over the paged cache, in float64: pages and slots from
request lengths, per-head norm and multi-axis rotation with its backward, the
append to the cache, causal attention over the pages, and the verification of
drafted tokens.

The paper prefills densely and decodes block-sparsely (Sec. 5.1); it says
nothing of chunked prompts, drafts or image positions.  Parity status: the
attention over the pages is pinned against the contiguous causal oracle, the
rotation of one axis against ``numerics.rope``, the backward against central
differences, the summaries against ``selector.block_summaries``, the
verification against the distribution it has to leave (the target's), and the
plan against hand-worked lengths.

TEST INFRASTRUCTURE ONLY (see the package docstring).
"""
import math

import numpy as np

from .numerics import rho


def plan_chunk(ctx_len, new_len, held, free_pages, free_count, table, page_size, num_pages, rows):
    """Returns the outputs of the plan as a dict (table a new array)."""
    table = np.array(table)
    b, width = table.shape
    left = min(max(int(free_count), 0), len(free_pages))
    missing = 0
    start, kv, have = [0], [], []
    seq, pos, slot = [np.full(rows, -1, dtype=np.int64) for _ in range(3)]
    total = 0
    for i in range(b):
        c, m, h = max(int(ctx_len[i]), 0), max(int(new_len[i]), 0), min(max(int(held[i]), 0), width)
        want = min(-(-(c + m) // page_size), width) if m else h
        got = h
        for j in range(h, want):
            if left:
                left -= 1
                table[i, j] = free_pages[left]
                got += 1
            else:
                table[i, j] = -1
                missing += 1
        have.append(got)
        given = min(m, max(rows - total, 0))   # tokens past `rows` have no row, and are not in the chunk
        kv.append(min(c + given, 2 ** 31 - 1))
        for j in range(given):
            r, p = total + j, c + j
            page = int(table[i, p // page_size]) if p // page_size < width else -1
            seq[r], pos[r] = i, min(p, 2 ** 31 - 1)
            if 0 <= page < num_pages:
                slot[r] = page * page_size + p % page_size
        total += m
        start.append(min(total, rows))
    return {"row_start": np.array(start), "kv_len": np.array(kv), "seq": seq, "pos": pos, "slot": slot,
            "pages_held": np.array(have), "free_count": np.array([left]), "missing": np.array([missing]),
            "block_table": table}


def turns(pos, sections, dh, base):
    """cos and sin [rows, dh/2] of the pairs' angles; pos [axes, rows]."""
    pos = np.atleast_2d(np.asarray(pos, dtype=np.float64))
    axis = np.repeat(np.arange(len(sections)), sections)
    assert len(axis) == dh // 2
    freq = np.power(float(base), -2.0 * np.arange(dh // 2) / dh)
    ang = pos[axis].T * freq
    return np.cos(ang), np.sin(ang)


def norm_rope(x, gain, pos, sections, base, eps):
    """x [rows, heads, dh] normed (unless gain is None) and rotated, not rounded."""
    x = np.asarray(x, dtype=np.float64)
    dh = x.shape[-1]
    if gain is not None:
        x = x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps) * np.asarray(gain, dtype=np.float64)
    c, s = (a[:, None, :] for a in turns(pos, sections, dh, base))
    x0, x1 = x[..., :dh // 2], x[..., dh // 2:]
    return np.concatenate([x0 * c - x1 * s, x1 * c + x0 * s], axis=-1)


def norm_rope_backward(x, gain, pos, sections, base, eps, dy):
    """(dx, dgain or None) of norm_rope, not rounded."""
    x, dy = np.asarray(x, dtype=np.float64), np.asarray(dy, dtype=np.float64)
    dh = x.shape[-1]
    c, s = (a[:, None, :] for a in turns(pos, sections, dh, base))
    y0, y1 = dy[..., :dh // 2], dy[..., dh // 2:]
    dn = np.concatenate([y0 * c + y1 * s, y1 * c - y0 * s], axis=-1)
    if gain is None:
        return dn, None
    g = np.asarray(gain, dtype=np.float64)
    r = 1.0 / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps)
    dgain = (dn * x * r).sum(axis=(0, 1))
    dx = r * (g * dn - x * r * r * np.mean(g * dn * x, axis=-1, keepdims=True))
    return dx, dgain


def page_of(table, i, p, page_size, num_pages):
    """Page of position p of sequence i, -1 if unmapped."""
    j = p // page_size
    page = int(table[i, j]) if 0 <= j < table.shape[1] else -1
    return page if 0 <= page < num_pages else -1


def completed_summaries(k_pages, table, ctx_len, kv_len, B, max_blocks, dtype, w_gk=None):
    """{(i, block): summary [Hkv, dh]} of the blocks that positions ctx_len[i] ..
    kv_len[i] - 1 complete; k_pages [pages, Hkv, page_size, dh] after the append."""
    num_pages, Hkv, ps, dh = k_pages.shape
    out = {}
    for i in range(len(ctx_len)):
        for m in range(int(ctx_len[i]) // B, min(int(kv_len[i]) // B, max_blocks)):
            acc = np.zeros((Hkv, dh))
            for p in range(m * B, (m + 1) * B):
                page = page_of(table, i, p, ps, num_pages)
                if page >= 0:
                    acc = acc + np.asarray(k_pages[page, :, p % ps], dtype=np.float64)
            s = rho(acc / B, dtype)
            if w_gk is not None:
                s = rho(np.einsum("gkj,gj->gk", np.asarray(w_gk, dtype=np.float64), s), dtype)
            out[i, m] = s
    return out


def attention_chunk(q, k_pages, v_pages, table, row_start, kv_len, sm_scale=None):
    """o [rows, H, dh] and lse [rows, H] in fp64 (NaN rows outside every
    sequence), and for error bounds A = sum_p p |v| [rows, H, dh] and the largest
    sum |q||k| sm of a row's keys [rows, H]."""
    q = np.asarray(q, dtype=np.float64)
    rows, H, dh = q.shape
    num_pages, Hkv, ps, _ = k_pages.shape
    G = H // Hkv
    sm = sm_scale or 1.0 / math.sqrt(dh)
    o, A = np.full((2, rows, H, dh), np.nan)
    lse, Z = np.full((2, rows, H), np.nan)
    for i in range(len(kv_len)):
        r0, r1 = int(row_start[i]), int(row_start[i + 1])
        if r1 == r0:
            continue
        n = min(int(kv_len[i]), table.shape[1] * ps)
        at = np.array([p for p in range(n) if page_of(table, i, p, ps, num_pages) >= 0], dtype=np.int64)
        pg = np.array([page_of(table, i, int(p), ps, num_pages) for p in at], dtype=np.int64)
        K = np.asarray(k_pages[pg, :, at % ps], dtype=np.float64) if len(at) else np.zeros((0, Hkv, dh))
        V = np.asarray(v_pages[pg, :, at % ps], dtype=np.float64) if len(at) else np.zeros((0, Hkv, dh))
        for j in range(r1 - r0):
            t = int(kv_len[i]) - (r1 - r0) + j
            c = int(np.searchsorted(at, t, side="right"))
            for h in range(H):
                if c == 0:
                    o[r0 + j, h], lse[r0 + j, h], A[r0 + j, h], Z[r0 + j, h] = 0.0, -np.inf, 0.0, 0.0
                    continue
                Kh, Vh, qh = K[:c, h // G], V[:c, h // G], q[r0 + j, h]
                z = Kh @ qh * sm
                top = z.max()
                w = np.exp(z - top)
                den = w.sum()
                o[r0 + j, h] = w @ Vh / den
                A[r0 + j, h] = w @ np.abs(Vh) / den
                lse[r0 + j, h] = top + math.log(den)
                Z[r0 + j, h] = (np.abs(Kh) @ np.abs(qh)).max() * sm
    return o, lse, A, Z


def verify_drafts(target, draft, tokens, draft_start, u_accept, u_sample, max_draft):
    """(tokens [b, max_draft + 1], accepted [b])."""
    target = np.asarray(target, dtype=np.float64)
    V = target.shape[1]
    b = len(u_sample)
    out = np.full((b, max_draft + 1), -1, dtype=np.int64)
    acc = np.zeros(b, dtype=np.int64)
    pos = lambda x: np.where(x > 0, x, 0.0)  # noqa: E731  (NaN counts as zero)
    for i in range(b):
        r0, r1 = int(draft_start[i]), int(draft_start[i + 1])
        w = None
        for j in range(r1 - r0):
            x = int(tokens[r0 + j])
            p = target[r0 + i + j]
            qd = None if draft is None else np.asarray(draft[r0 + j], dtype=np.float64)
            if 0 <= x < V and float(u_accept[r0 + j]) * (1.0 if qd is None else qd[x]) < p[x]:
                out[i, j] = x
                acc[i] += 1
                continue
            if qd is None:
                w = pos(p)
                if 0 <= x < V:
                    w[x] = 0.0
            else:
                w = pos(p - qd)
            if not (w > 0).any():
                w = None
            break
        if w is None:
            w = pos(target[r0 + i + int(acc[i])])
        cum = np.cumsum(w)
        # a token of zero weight is never drawn
        hit = np.nonzero((cum > float(u_sample[i]) * cum[-1]) & (w > 0))[0]
        some = np.nonzero(w > 0)[0]
        out[i, acc[i]] = hit[0] if len(hit) else some[-1] if len(some) else -1
    return out, acc
