"""sas_plan_chunk against the oracle: every output, and the rest of the block
table untouched."""
import numpy as np
import pytest
import torch

import oracle
from paper_2609_13141_amd import sas

pytestmark = pytest.mark.gpu


def make(ctx, new, held, ps, width, free, count, num_pages, seed=0):
    rng = np.random.default_rng(seed)
    b = len(ctx)
    table = rng.integers(-3, num_pages + 3, size=(b, width))
    dev = lambda a: torch.tensor(np.array(a), dtype=torch.int32, device="cuda")  # noqa: E731
    z = torch.zeros(num_pages, 1, ps, 8, dtype=torch.bfloat16, device="cuda")
    cache = sas.PagedCache(z, z, dev(table), torch.zeros(b, 1, 1, 8, dtype=torch.bfloat16, device="cuda"), ps)
    return cache, table, (dev(ctx), dev(new), dev(held), dev(free), dev([count]))


def check(ctx, new, held, ps, width, free, count, num_pages, rows):
    cache, table, args = make(ctx, new, held, ps, width, free, count, num_pages)
    want = oracle.chunk.plan_chunk(ctx, new, held, free, count, table, ps, num_pages, rows)
    got = sas.plan_chunk(cache, *args, rows)
    torch.cuda.synchronize()
    for k, v in want.items():
        g = (cache.block_table if k == "block_table" else got[k]).cpu().numpy()
        np.testing.assert_array_equal(g, v, err_msg=k)


def need(ctx, new, held, ps, width):
    return sum(max(0, min(-(-(c + m) // ps), width) - h) for c, m, h in zip(ctx, new, held) if m > 0)


@pytest.mark.parametrize("b,hi,ps", [(1, 1, 16), (3, 40, 16), (8, 1, 1), (64, 9, 4), (65, 200, 128), (300, 33, 16),
                                     (1025, 5, 8), (4096, 3, 16)])
@pytest.mark.parametrize("pad", [0, 1, 37])
def test_lengths(b, hi, ps, pad):
    rng = np.random.default_rng(b * 7 + hi)
    ctx = rng.integers(0, 500, size=b)
    new = rng.integers(0 if b > 1 else 1, hi + 1, size=b)
    new[rng.integers(0, b)] = hi
    held = -(-ctx // ps) + rng.integers(0, 2, size=b)
    width = -(-(500 + hi) // ps) + 2
    n = need(ctx, new, held, ps, width)
    free = rng.permutation(n + 5)
    print(f"\n[case] plan b={b} new<={hi} ps={ps} pad={pad} pages {n}", flush=True)
    check(ctx, new, held, ps, width, free, n + 5, n + 5, int(new.sum()) + pad)


@pytest.mark.parametrize("count", [0, 1, 7, 1000])
def test_the_stack_runs_out(count):
    ctx, new, held = [5, 0, 16, 3], [30, 20, 1, 2], [1, 0, 1, 1]
    check(ctx, new, held, 4, 12, np.arange(11)[::-1], count, 64, 60)


def test_tokens_past_the_rows_and_past_the_table():
    check([0, 10, 4], [9, 9, 9], [0, 3, 1], 4, 3, np.arange(30), 30, 30, 20)


def test_lengths_that_make_no_sense_stay_in_bounds():
    big = 2 ** 31 - 1
    check([-5, big, 3, big], [4, 3, -2, big], [-1, big, 2, 0], 16, 6, np.arange(40), 40, 40, 50)
    check([0, 0], [0, -4], [0, 1], 16, 6, np.arange(4), -3, 4, 5)


def test_no_free_list():
    cache, table, args = make([3], [2], [1], 16, 2, [0], 0, 8)
    got = sas.plan_chunk(cache, *args[:3], args[3][:0], args[4], 4)
    assert int(got["missing"]) == 0 and got["pos"].tolist() == [3, 4, -1, -1]


def test_captured_replays_follow_the_lengths():
    ps, width, rows = 16, 8, 24
    cache, table, (ctx, new, held, free, count) = make([0] * 4, [0] * 4, [0] * 4, ps, width, np.arange(20), 20, 20)
    sas.plan_chunk(cache, ctx, new, held, free, count, rows)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = sas.plan_chunk(cache, ctx, new, held, free, count, rows)
    rng = np.random.default_rng(1)
    for _ in range(4):
        c, m = rng.integers(0, 60, size=4), rng.integers(0, 9, size=4)
        h = -(-c // ps)
        t = rng.integers(0, 20, size=(4, width))
        for dst, a in ((ctx, c), (new, m), (held, h), (cache.block_table, t)):
            dst.copy_(torch.tensor(a, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        want = oracle.chunk.plan_chunk(c, m, h, np.arange(20), 20, t, ps, 20, rows)
        for k, v in want.items():
            np.testing.assert_array_equal((cache.block_table if k == "block_table" else out[k]).cpu().numpy(), v)


def test_the_binding_refuses_other_types_and_strides():
    cache, _, (ctx, new, held, free, count) = make([0] * 4, [1] * 4, [0] * 4, 16, 8, np.arange(20), 20, 20)
    for a in ((ctx.long(), new, held), (ctx, new[:3], held), (ctx, new, torch.stack([held, held], 1)[:, 0])):
        with pytest.raises(sas.SasError):
            sas.plan_chunk(cache, *a, free, count, 4)
    with pytest.raises(sas.SasError):
        sas.plan_chunk(cache, ctx, new, held, free, count, 0)
