"""The oracle of the chunk operators against independent statements of the same
things (CPU)."""
import numpy as np
import pytest

import oracle
from oracle import chunk as ref


def test_attention_over_pages_equals_the_contiguous_causal_attention():
    rng = np.random.default_rng(0)
    n, m, H, Hkv, dh, ps = 37, 9, 4, 2, 8, 4
    K, V, Q = rng.standard_normal((3, n, H, dh))
    K, V = K[:, :Hkv], V[:, :Hkv]
    pages = rng.permutation(12)
    kp, vp = np.full((2, 12, Hkv, ps, dh), np.nan)
    for p in range(n):
        kp[pages[p // ps], :, p % ps], vp[pages[p // ps], :, p % ps] = K[p], V[p]
    table = np.full((1, 11), -1)
    table[0, :10] = pages[:10]
    o, lse, _, _ = ref.attention_chunk(Q[-m:], kp, vp, table, [0, m], [n])
    _, exact, L = oracle.sas_attention(Q[-m:], K, V, 4, "dense", "f32", rows=np.arange(n - m, n))
    np.testing.assert_allclose(o, exact, rtol=1e-12, atol=1e-14)
    np.testing.assert_allclose(lse, L.T, rtol=1e-12)


def test_one_axis_is_the_layers_rotation_and_axes_turn_their_own_pairs():
    rng = np.random.default_rng(1)
    x, pos = rng.standard_normal((5, 3, 16)), np.array([0, 1, 7, 300, 100000])
    np.testing.assert_allclose(ref.norm_rope(x, None, pos, (8,), 1e4, 0), oracle.rope(x, pos, 1e4), atol=1e-12)
    three = np.stack([pos, pos * 2 + 1, np.zeros(5, int)])
    y = ref.norm_rope(x, None, three, (2, 3, 3), 1e4, 0)
    full = [oracle.rope(x, p, 1e4) for p in three]
    for i in range(8):
        a = 0 if i < 2 else 1 if i < 5 else 2
        np.testing.assert_allclose(y[..., [i, i + 8]], full[a][..., [i, i + 8]], atol=1e-12)


@pytest.mark.parametrize("normed", [True, False])
def test_backward_against_differences(normed):
    rng = np.random.default_rng(2)
    x, dy = rng.standard_normal((2, 3, 2, 8))
    g = 1 + 0.3 * rng.standard_normal(8) if normed else None
    pos = np.array([[3, 50, 9], [1, 0, 4]])
    f = lambda x_, g_: (ref.norm_rope(x_, g_, pos, (1, 3), 1e4, 1e-3) * dy).sum()  # noqa: E731
    dx, dg = ref.norm_rope_backward(x, g, pos, (1, 3), 1e4, 1e-3, dy)
    h = 1e-6
    for idx in np.ndindex(x.shape):
        e = np.zeros_like(x)
        e[idx] = h
        assert abs((f(x + e, g) - f(x - e, g)) / (2 * h) - dx[idx]) < 1e-7
    if normed:
        for d in range(8):
            e = np.zeros(8)
            e[d] = h
            assert abs((f(x, g + e) - f(x, g - e)) / (2 * h) - dg[d]) < 1e-7
    else:
        assert dg is None


def test_summaries_are_the_selectors():
    rng = np.random.default_rng(3)
    K = oracle.rho(rng.standard_normal((32, 2, 8)), "bf16")
    kp = np.full((8, 2, 4, 8), np.nan)
    table = rng.permutation(8)[None]
    for p in range(32):
        kp[table[0, p // 4], :, p % 4] = K[p]
    s = ref.completed_summaries(kp, table, [9], [32], 8, 4, "bf16")
    assert sorted(s) == [(0, 1), (0, 2), (0, 3)]
    want = oracle.block_summaries(K, 8, "bf16")
    for (_, m), v in s.items():
        np.testing.assert_array_equal(v, want[:, m])


def test_plan_of_hand_worked_lengths():
    table = np.array([[5, -1, -1], [3, 4, -1], [-1, -1, -1]])
    out = ref.plan_chunk([3, 8, 0], [2, 0, 9], [1, 2, 0], [9, 8, 7, 6], 4, table, 4, 100, 13)
    # sequence 0: positions 3, 4 (one page, the top 6); 2: positions 0..8, three pages, 7, 8, 9
    np.testing.assert_array_equal(out["block_table"], [[5, 6, -1], [3, 4, -1], [7, 8, 9]])
    np.testing.assert_array_equal(out["row_start"], [0, 2, 2, 11])
    np.testing.assert_array_equal(out["pos"], [3, 4, 0, 1, 2, 3, 4, 5, 6, 7, 8, -1, -1])
    np.testing.assert_array_equal(out["slot"], [23, 24, 28, 29, 30, 31, 32, 33, 34, 35, 36, -1, -1])
    np.testing.assert_array_equal(out["pages_held"], [2, 2, 3])
    assert out["free_count"][0] == 0 and out["missing"][0] == 0
    short = ref.plan_chunk([3, 8, 0], [2, 0, 9], [1, 2, 0], [9, 8, 7, 6], 2, table, 4, 100, 13)
    np.testing.assert_array_equal(short["block_table"], [[5, 8, -1], [3, 4, -1], [9, -1, -1]])
    assert short["missing"][0] == 2 and (short["slot"][6:11] == -1).all()
    np.testing.assert_array_equal(short["pages_held"], [2, 2, 1])


def test_verified_tokens_follow_the_targets_distribution():
    # whatever the draft, the first token's distribution is the target's
    rng = np.random.default_rng(4)
    V, n = 5, 40000
    p, q = rng.dirichlet(np.ones(V)), rng.dirichlet(np.ones(V))
    x = rng.choice(V, size=n, p=q)
    target = np.broadcast_to(p, (2 * n, V))
    out, acc = ref.verify_drafts(target, np.broadcast_to(q, (n, V)), x, np.arange(n + 1), rng.random(n), rng.random(n), 1)
    freq = np.bincount(out[:, 0], minlength=V) / n
    # five standard deviations of a binomial share
    assert (np.abs(freq - p) < 5 * np.sqrt(p * (1 - p) / n)).all()
    assert abs(acc.mean() - np.minimum(p, q).sum()) < 5 * 0.5 / np.sqrt(n)
