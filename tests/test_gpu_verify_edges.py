"""sas_verify_drafts at the edges of its inputs in every way that the vocabulary is
divided: one cut (600 tokens), repeated cuts by one workgroup (20000), and sums taken
by a kernel before (100003, few sequences)."""
import numpy as np
import pytest
import torch

import oracle
from paper_2609_13141_amd import sas
from test_gpu_verify_drafts import case, check

pytestmark = pytest.mark.gpu
VOCABS = [600, 20000, 100003]


def holes(t, V):
    """Weights in a few narrow ranges only: whole pieces of every cut are empty."""
    keep = torch.zeros(V, dtype=torch.bool)
    for a in (V // 7, V // 2, V - V // 5):
        keep[a:a + max(V // 300, 2)] = True
    t[:, ~keep] = 0.0
    return keep


@pytest.mark.parametrize("V", VOCABS)
@pytest.mark.parametrize("us", [0.0, 2.0 ** -24, 0.5, 1.0 - 2.0 ** -24, 1.0, 2.0, -1.0, float("nan")])
def test_uniforms_at_and_past_the_borders(V, us):
    a = case([2, 0, 1], V, 4)
    keep = holes(a[0], V)
    a[1] = a[0][[0, 1, 4]].clone()
    a[5][:] = us
    want, acc = check(a, 2)
    assert keep[torch.tensor(want[np.arange(3), acc])].all()
    # nothing drafted with a distribution: the drafted token is left out
    a[1], a[4][:] = None, 1.0
    check(a, 2)


@pytest.mark.parametrize("V", VOCABS)
@pytest.mark.parametrize("at", ["the first token", "the last token", "the end of a piece"])
def test_all_weight_on_one_token(V, at):
    x = {"the first token": 0, "the last token": V - 1, "the end of a piece": min(V - 1, 64 * (V // 1100 + 1) - 1)}[at]
    for us in (0.0, 0.4, 1.0 - 2.0 ** -24, 1.0):
        a = case([1, 0, 2], V, 8)
        a[0][:] = 0.0
        a[0][:, x] = 0.7
        a[5][:] = us
        want, acc = check(a, 2)
        assert (want[np.arange(3), acc] == x).all()


@pytest.mark.parametrize("V", VOCABS)
def test_an_empty_rest_draws_from_the_target(V):
    a = case([3, 3, 1], V, 5)
    rows = [0, 1, 2, 4, 5, 6, 8]
    a[1] = a[0][rows].clone()
    a[2] = a[1].argmax(1).int()
    _, acc = check(a, 3)
    assert acc.tolist() == [3, 3, 1]
    a[1] = (a[0][rows] * 1.5).clone()    # p <= q everywhere: nothing is left over
    a[4][:] = 0.99
    for u in (0.0, 0.3, 0.999):
        a[5][:] = u
        _, acc = check(a, 3)
        assert (acc == 0).all()
    # all the target's weight is on the drafted token, which is left out: nothing remains either
    a[0][:] = 0.0
    a[0][torch.arange(len(a[0])), a[2][0]] = 1.0
    a[1], a[4][:] = None, 1.0
    check(a, 3)


@pytest.mark.parametrize("V", VOCABS)
def test_zero_and_nan_weights_and_tokens_outside_the_vocabulary(V):
    a = case([2, 2, 1], V, 6)
    a[2][0], a[2][2] = V, -1
    a[0][3:5] = 0.0
    a[0][0, ::3] = float("nan")
    a[0][6, V // 3:] = -1.0
    check(a, 2)
    a[1][:, :V // 2] = float("nan")
    check(a, 2)
    a[1] = None
    check(a, 2)
    z = case([1, 0, 1], V, 7)
    z[0][:] = 0.0
    z[0][1] = float("nan")
    want, acc = check(z, 1)
    assert (acc == 0).all() and (want[:, 0] == -1).all()


@pytest.mark.parametrize("V", VOCABS)
def test_captured_replays(V):
    a = [t.cuda() for t in case([2, 1, 0], V, 8)]
    sas.verify_drafts(*a, 2)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = sas.verify_drafts(*a, 2)
    for seed, drafts in ((9, [2, 1, 0]), (10, [0, 1, 2]), (11, [1, 1, 1]), (12, [1, 0, 2])):
        b = case(drafts, V, seed)
        if seed == 11:      # nothing left over: the sums taken before are not those that are used
            b[1] = (b[0][[0, 2, 4]] * 2).clone()
            b[4][:] = 0.99
        for dst, src in zip(a, b):
            dst.copy_(src)
        other = sas.verify_drafts(*[t.cuda() for t in case([2, 0, 1], V, seed + 20)], 2)
        graph.replay()
        torch.cuda.synchronize()
        del other
        want, acc = oracle.chunk.verify_drafts(*[t.numpy() for t in b], 2)
        np.testing.assert_array_equal(out["tokens"].cpu().numpy(), want)
        np.testing.assert_array_equal(out["accepted"].cpu().numpy(), acc)


@pytest.mark.parametrize("V,b,scratch", [(65536, 3, False), (65537, 127, True), (65537, 128, False), (131072, 129, False),
                                         (131073, 128, True), (131073, 1, True), (250001, 130, True)])
def test_both_sides_of_the_division(V, b, scratch):
    check(case([i % 2 for i in range(b)], V, b), 2)
    assert (sas.lib().sas_workspace_size(None, sas.OP_VERIFY_DRAFTS, b, V) > 0) == scratch
