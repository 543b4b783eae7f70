"""Beam search's selection and reordering on the GPU against the definitions in float64.

Scores are float32 sums and one logarithm: held to 2e-6 absolute for scores of up to 20 (an ulp there
is 2e-6). Tokens, parents and slots are exact; inputs whose candidates differ by less than that are
those with equal scores by construction."""

import numpy as np
import pytest
import torch

import gdr_ref as R
from paper_2609_07816_amd import kdn

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def select(logits, scores, done, end, dtype):
    """Runs the operator on float64 arrays that the type holds; returns host arrays."""
    out = kdn.beam_select(torch.from_numpy(logits).to(DT[dtype]).cuda(),
                          torch.from_numpy(scores).float().cuda(),
                          None if done is None else torch.from_numpy(done).cuda(), end)
    return [t.cpu().numpy() for t in out]


def check(logits, scores, done, end, dtype):
    got = select(logits, scores, done, end, dtype)
    want = R.beam_select(logits, scores, done, end)
    fine = np.isfinite(want[0])
    assert np.array_equal(fine, np.isfinite(got[0]))
    assert np.abs(got[0][fine] - want[0][fine]).max(initial=0.0) <= 4e-6
    for i in (1, 2, 3):
        assert np.array_equal(got[i], want[i]), ("token", "parent", "done")[i - 1]


def draw(seed, N, W, V, dtype):
    g = np.random.default_rng(seed)
    logits = (3 * g.standard_normal((N, W, V))).astype(np.float32).astype(np.float64)
    if dtype == "bf16":
        logits = R.to_bf16(logits)
    scores = -g.uniform(0, 8, (N, W)).astype(np.float32).astype(np.float64)
    return g, logits, scores


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,W,V", [(1, 1, 1), (1, 1, 7), (2, 3, 5), (3, 4, 512), (2, 4, 513),
                                   (1, 2, 1000), (5, 8, 4001), (2, 64, 2003), (1, 5, 40007),
                                   (40, 3, 9001), (1, 64, 65), (3, 16, 3)])
def test_select(N, W, V, dtype):
    g, logits, scores = draw(N + W + V, N, W, V, dtype)
    check(logits, scores, None, V - 1, dtype)
    check(logits, scores, g.random((N, W)) < 0.4, V // 2, dtype)
    check(logits, scores, np.ones((N, W), bool), 0, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_ties_take_the_lowest(dtype):
    """Equal logits within a beam and equal beams: the lowest beam, then the lowest token; across
    tiles and pieces, and -0 as 0."""
    V = 3001
    logits = np.zeros((2, 4, V))
    logits[0, :, 1::2] = -0.0
    logits[1, :, [5, 600, 601, 2999]] = 2.0
    scores = np.zeros((2, 4))
    check(logits, scores, None, 0, dtype)
    got = select(logits, scores, None, 0, dtype)
    assert got[1].tolist() == [[0, 1, 2, 3], [5, 600, 601, 2999]]
    assert got[2].tolist() == [[0] * 4] * 2


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masks_and_values_that_are_not_finite(dtype):
    g, logits, scores = draw(4, 6, 4, 1030, dtype)
    low = float(torch.finfo(DT[dtype]).min)
    logits[0, 1] = -np.inf                      # a beam with no token left
    logits[0, 2, g.random(1030) < 0.999] = -np.inf
    logits[1] = -np.inf                         # a batch element with none
    logits[2, :, 3:] = low                      # masked by the type's lowest value
    logits[3, 0, 17] = np.inf                   # a forced token
    logits[3, 1, :40] = np.nan
    logits[4, :, :] = np.nan
    scores[5, 1:] = -np.inf                     # the first step: one beam
    check(logits, scores, None, 2, dtype)


def test_first_index_past_a_row_start_of_any_alignment():
    """Rows of odd length start at any alignment; the neighbours' values stay out."""
    for V in (1, 2, 3, 5, 9, 511, 519, 1025):
        logits = np.full((3, 2, V), -5.0)
        logits[:, 1] = 60.0
        check(logits, np.zeros((3, 2)), None, 0, "bf16")
        check(logits, np.zeros((3, 2)), None, 0, "f32")
    base = torch.randn(4 * 101 + 3, device="cuda").bfloat16()
    view = base[3:].view(2, 2, 101)             # logits off a 16-byte boundary
    sc = torch.zeros(2, 2, device="cuda")
    a, b = kdn.beam_select(view, sc), kdn.beam_select(view.clone(), sc)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("N,W,slots,shape,pshape", [
    (1, 1, 1, (4,), None), (1, 4, 9, (2, 16, 16), (2, 16)), (6, 5, 40, (3, 32, 64), (3,)),
    (2, 64, 130, (1, 16, 16), (1, 16)), (3, 8, 24, (2, 128, 128), (2, 128))])
def test_reorder(N, W, slots, shape, pshape):
    g = np.random.default_rng(N * W)
    S = g.standard_normal((slots,) + shape).astype(np.float32)
    P = None if pshape is None else g.standard_normal((slots,) + pshape).astype(np.float32)
    slot = g.permutation(slots)[:N * W].reshape(N, W).astype(np.int32)
    for trial in range(4):
        parent = g.integers(0, W, (N, W)).astype(np.int32)
        if trial == 0:
            parent[:] = np.arange(W)            # nothing moves
        if trial == 1:
            parent[:] = W - 1                   # one survivor
        if trial == 2 and W > 1:
            parent[0, 0], parent[0, 1] = -1, W  # no parent
            slot[0, W - 1] = -1                 # no state
        dS = torch.from_numpy(S).cuda()
        dP = None if P is None else torch.from_numpy(P).cuda()
        got = kdn.beam_reorder(torch.from_numpy(parent).cuda(), torch.from_numpy(slot).cuda(), dS,
                               dP)
        want, pools = R.beam_reorder(parent, slot, [S] if P is None else [S, P])
        assert np.array_equal(got.cpu().numpy(), want)
        assert np.array_equal(dS.cpu().numpy(), pools[0])
        if P is not None:
            assert np.array_equal(dP.cpu().numpy(), pools[1])


def test_stream_and_graph():
    g = torch.Generator(device="cuda").manual_seed(1)
    logits = torch.randn(3, 4, 5003, generator=g, device="cuda")
    scores = torch.zeros(3, 4, device="cuda")
    slot = torch.arange(12, device="cuda").view(3, 4).int()
    S = torch.randn(12, 2, 16, 16, generator=g, device="cuda")

    def step(pool):
        out = kdn.beam_select(logits, scores, end_token=1)
        return out + (kdn.beam_reorder(out[2], slot, pool), pool)

    want = step(S.clone())
    pool = S.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(pool)
    for _ in range(3):
        pool.copy_(S)
        for t in out[:5]:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(out, want))


def test_refusals():
    logits = torch.zeros(2, 3, 10, device="cuda")
    scores = torch.zeros(2, 3, device="cuda")
    with pytest.raises(ValueError):
        kdn.beam_select(logits[0], scores)
    with pytest.raises(ValueError):
        kdn.beam_select(logits, scores[:1])
    with pytest.raises(TypeError):
        kdn.beam_select(logits.half(), scores)
    with pytest.raises(TypeError):
        kdn.beam_select(logits, scores.double())
    with pytest.raises(kdn.KdnError):
        kdn.beam_select(logits, scores, end_token=10)
    with pytest.raises(kdn.KdnError):
        kdn.beam_select(torch.zeros(1, 65, 10, device="cuda"), torch.zeros(1, 65, device="cuda"))
    slot = torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        kdn.beam_reorder(slot, slot[:1], torch.zeros(6, 4, device="cuda"))
    with pytest.raises(TypeError):
        kdn.beam_reorder(slot.long(), slot, torch.zeros(6, 4, device="cuda"))
    with pytest.raises(ValueError):
        kdn.beam_reorder(slot, slot, torch.zeros(6, 4, device="cuda"),
                         torch.zeros(5, 4, device="cuda"))
