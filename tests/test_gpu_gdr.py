"""Gated delta rule on the GPU against the float64 recurrences.

Tolerances (rel-L2 against float64 on the stored inputs). float32 outputs: float32 sums over up to a
few hundred tokens lose some 2^-24 sqrt(terms) each, and products from operands in two halves 2^-22:
below 1e-6 together, held to 3e-6. bf16 outputs: operands rounded to 11 bits give 2^-12 each, held to
8e-4, beside the final rounding, which is that of the exact result (1.7e-3 over many values; a single
value's is up to 2^-8)."""

import numpy as np
import pytest
import torch

import gdr_ref as R
from gpu_util import host_f64, rel_l2
from paper_2609_07816_amd import kdn

pytestmark = pytest.mark.gpu
TOL = {"f32": 3e-6, "bf16": 2.5e-3}
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
NAMES = ("q", "k", "v", "alpha", "beta")


def dev(x, dtype):
    t = {n: torch.from_numpy(x[n]).to(DT[dtype]).cuda() for n in NAMES + ("dO",)}
    for n in ("S0", "dS_T"):
        t[n] = None if x[n] is None else torch.from_numpy(x[n]).cuda()
    return t


def near(got, want, dtype):
    """Whether an output in the call's type is as near as it has to be."""
    tol = TOL["f32"] if dtype == "f32" else 8e-4 + rel_l2(R.to_bf16(want), want)
    return rel_l2(host_f64(got), want) <= tol


def cu_of(lens):
    return None if lens is None else np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


# (B or packed lengths, T, H, Hk, dk, dv, initial state, gates)
SHAPES = [
    (1, 1, 1, 1, 128, 128, False, "usual"),
    (2, 3, 2, 1, 16, 16, True, "usual"),
    (1, 64, 2, 2, 32, 64, False, "usual"),
    (2, 65, 3, 1, 64, 32, True, "usual"),
    (1, 127, 2, 2, 128, 128, True, "zeros"),
    (1, 200, 4, 2, 128, 64, False, "strong"),
    (1, 150, 2, 1, 16, 128, True, "one"),
    (1, 190, 2, 2, 128, 16, True, "scaled"),
    (2, 333, 2, 2, 128, 128, False, "usual"),
    (1, 300, 2, 1, 64, 64, True, "jumps"),
    ([0, 1, 63, 0, 64, 65, 130, 2, 0], None, 2, 1, 64, 128, True, "usual"),
    ([5], None, 1, 1, 32, 32, False, "usual"),
    ([100, 28, 300], None, 3, 3, 128, 128, True, "zeros"),
]


def case(shape, dtype, seed):
    B, T, H, Hk, dk, dv, state, gates = shape
    lens = B if isinstance(B, list) else None
    N = len(lens) if lens else None
    x = R.draw(seed, 1 if lens else B, sum(lens) if lens else T, H, Hk, dk, dv, dtype, N, state,
               gates)
    return x, cu_of(lens)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_forward(shape, dtype):
    x, cu = case(shape, dtype, 11)
    d = dev(x, dtype)
    o, S = kdn.forward_gdr(*[d[n] for n in NAMES], S0=d["S0"],
                           cu_seqlens=None if cu is None else torch.from_numpy(cu).cuda())
    want_o, want_S = R.forward(x, cu)
    assert o.dtype == DT[dtype] and S.dtype == torch.float32
    assert near(o, want_o, dtype)
    assert near(S, want_S, "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_backward(shape, dtype):
    """Every gradient against the adjoint recurrence in float64. The gradients of a chunk sum some
    hundred products whose operands were rounded once (bf16 calls) on the way: 2^-12 each beside the
    final rounding; the state's gradient keeps float32 accuracy."""
    x, cu = case(shape, dtype, 12)
    d = dev(x, dtype)
    got = kdn.backward_gdr(*[d[n] for n in NAMES], S0=d["S0"], dO=d["dO"], dS_T=d["dS_T"],
                           cu_seqlens=None if cu is None else torch.from_numpy(cu).cuda())
    want = R.backward(x, cu)
    for n in ("dq", "dk", "dv", "dalpha", "dbeta"):
        assert got[n].dtype == DT[dtype] and got[n].shape == d[n[1:]].shape
        assert near(got[n], want[n], dtype), n
    assert got["dS0"].dtype == torch.float32
    assert near(got["dS0"], want["dS0"], "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("given", ["dO", "dS_T"])
def test_backward_of_one_output(given, dtype):
    """The other output's gradient is left out (None)."""
    x = R.draw(13, 2, 100, 4, 2, 64, 64, dtype, state=True)
    d = dev(x, dtype)
    x = dict(x, **{"dO": 0 * x["dO"]} if given == "dS_T" else {"dS_T": None})
    got = kdn.backward_gdr(*[d[n] for n in NAMES], S0=d["S0"], **{given: d[given]})
    want = R.backward(x)
    for n in want:
        assert near(got[n], want[n], "f32" if n == "dS0" else dtype), n


def test_backward_is_the_same_every_time_and_on_another_stream():
    x = R.draw(14, 1, 300, 4, 1, 128, 128, "bf16", state=True)
    d = dev(x, "bf16")
    kw = dict(S0=d["S0"], dO=d["dO"], dS_T=d["dS_T"])
    args = [d[n] for n in NAMES]
    first = kdn.backward_gdr(*args, **kw)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        again = kdn.backward_gdr(*args, **kw)
    torch.cuda.synchronize()
    assert all(torch.equal(first[n], again[n]) for n in first)


def test_backward_leaves_tokens_outside_the_sequences():
    x = R.draw(5, 1, 200, 2, 2, 32, 32)
    d = dev(x, "f32")
    cu = torch.tensor([0, 70, 130], dtype=torch.int32).cuda()
    args = [d[n] for n in NAMES]
    inside = kdn.backward_gdr(*args, dO=d["dO"], cu_seqlens=cu)
    for n in NAMES + ("dO",):
        d[n][:, 130:] = float("nan")
    again = kdn.backward_gdr(*args, dO=d["dO"], cu_seqlens=cu)
    for n in ("dq", "dk", "dv", "dalpha", "dbeta"):
        assert torch.equal(inside[n][:, :130], again[n][:, :130]), n


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_forward_in_place_state_and_no_state_out(dtype):
    """S_T may be S0 itself, and may be left out; twice in halves is once in whole."""
    x = R.draw(3, 2, 160, 2, 1, 64, 64, dtype, state=True)
    d = dev(x, dtype)
    args = [d[n] for n in NAMES]
    o, S = kdn.forward_gdr(*args, S0=d["S0"])
    half = [[t[:, :96].contiguous() for t in args], [t[:, 96:].contiguous() for t in args]]
    S1 = d["S0"].clone()
    outs = []
    for h in half:
        q, k, v, a, b = h
        y = torch.empty_like(v)
        L = kdn.lib()
        need = L.kdn_forward_gdr_workspace_bytes(2, 2, v.shape[1], 2, 1, 64, 64,
                                                 kdn._dtype_code(v), 0)
        ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        st = L.kdn_forward_gdr(*kdn._ptrs(q, k, v, a, b, S1, y, S1), None, 2, 2, v.shape[1], 2, 1,
                               64, 64, kdn._dtype_code(v), 0.125, kdn._ptr(ws), need,
                               kdn._stream(v.device))
        assert st == kdn.KDN_OK
        outs.append(y)
    assert rel_l2(host_f64(S1), host_f64(S)) <= TOL["f32"]
    assert rel_l2(host_f64(torch.cat(outs, 1)), host_f64(o)) <= TOL[dtype]


def test_forward_leaves_tokens_outside_the_sequences():
    """Tokens after the last sequence are not written."""
    x = R.draw(5, 1, 200, 2, 2, 32, 32)
    d = dev(x, "f32")
    cu = torch.tensor([0, 70, 130], dtype=torch.int32).cuda()
    o = torch.full_like(d["v"], 7.0)
    S = torch.empty(2, 2, 32, 32, device="cuda")
    L = kdn.lib()
    need = L.kdn_forward_gdr_workspace_bytes(2, 1, 200, 2, 2, 32, 32, 0, 1)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    st = L.kdn_forward_gdr(*kdn._ptrs(*[d[n] for n in NAMES], None, o, S, cu), 2, 1, 200, 2, 2, 32,
                           32, 0, 1.0, kdn._ptr(ws), need, kdn._stream(o.device))
    assert st == kdn.KDN_OK
    assert bool((o[:, 130:] == 7.0).all()) and bool((o[:, :130] != 7.0).any())


def test_infinities_past_a_sequence_stay_out():
    """What stands after a sequence's end reaches nothing of it."""
    x = R.draw(6, 1, 100, 2, 1, 64, 64, "bf16")
    d = dev(x, "bf16")
    cu = torch.tensor([0, 40, 90], dtype=torch.int32).cuda()
    o, S = kdn.forward_gdr(*[d[n] for n in NAMES], cu_seqlens=cu)
    for n in NAMES:
        d[n][:, 90:] = float("nan")
    o2, S2 = kdn.forward_gdr(*[d[n] for n in NAMES], cu_seqlens=cu)
    assert torch.equal(o[:, :90], o2[:, :90]) and torch.equal(S, S2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,slots,H,Hk,dk,dv", [(1, 1, 1, 1, 16, 16), (3, 7, 2, 1, 16, 32),
                                                   (5, 5, 4, 4, 32, 16), (7, 20, 6, 2, 64, 128),
                                                   (9, 16, 4, 1, 128, 64), (33, 40, 2, 2, 128, 128)])
def test_decode(rows, slots, H, Hk, dk, dv, dtype):
    x = R.draw(21, 1, rows, H, Hk, dk, dv, dtype)
    d = {n: y[0] for n, y in dev(x, dtype).items() if y is not None}
    g = np.random.default_rng(5)
    S = g.standard_normal((slots, H, dk, dv)).astype(np.float32)
    slot = g.permutation(slots)[:rows].astype(np.int32)
    if rows > 3:
        slot[1], slot[2] = -1, slots + 3  # skipped rows
    pool = torch.from_numpy(S).cuda()
    o = torch.full((rows, H, dv), 9.0, dtype=DT[dtype], device="cuda")
    kdn.decode_step_gdr(*[d[n] for n in NAMES], pool, slot_idx=torch.from_numpy(slot).cuda(), o=o)
    want, want_o = S.astype(np.float64), np.full((rows, H, dv), 9.0)
    for i, s in enumerate(slot):
        if 0 <= s < slots:
            y = {n: x[n][:, i:i + 1] for n in NAMES}
            y["S0"] = S[s:s + 1]
            oo, SS = R.forward(y)
            want[s], want_o[i] = SS[0], oo[0, 0]
    assert near(pool, want, "f32")
    assert near(o, want_o, dtype)


def test_decode_continues_the_forward():
    """A prefill, then single tokens, is the forward of all."""
    x = R.draw(8, 2, 140, 4, 2, 128, 128, "bf16")
    d = dev(x, "bf16")
    o, S = kdn.forward_gdr(*[d[n] for n in NAMES])
    o1, S1 = kdn.forward_gdr(*[d[n][:, :137].contiguous() for n in NAMES])
    for t in range(137, 140):
        y = kdn.decode_step_gdr(*[d[n][:, t].contiguous() for n in NAMES], S1)
        assert rel_l2(host_f64(y), host_f64(o[:, t])) <= 2 * TOL["bf16"]
    assert rel_l2(host_f64(S1), host_f64(S)) <= TOL["f32"]


def test_other_stream_and_graph():
    """On a stream of the caller's, and captured: every replay gives the eager result."""
    x = R.draw(9, 1, 130, 2, 1, 64, 64, "bf16", state=True)
    d = dev(x, "bf16")
    args = [d[n] for n in NAMES]
    o, S = kdn.forward_gdr(*args, S0=d["S0"])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        o1, S1 = kdn.forward_gdr(*args, S0=d["S0"])
    torch.cuda.synchronize()
    assert torch.equal(o, o1) and torch.equal(S, S1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o2, S2 = kdn.forward_gdr(*args, S0=d["S0"])
    for _ in range(3):
        o2.zero_()
        S2.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, o2) and torch.equal(S, S2)


def test_refusals():
    x = R.draw(1, 1, 8, 2, 1, 32, 32)
    d = dev(x, "f32")
    q, k, v, a, b = [d[n] for n in NAMES]
    with pytest.raises(TypeError):
        kdn.forward_gdr(q, k, v.bfloat16(), a, b)
    with pytest.raises(ValueError):
        kdn.forward_gdr(q[:, :4], k, v, a, b)
    with pytest.raises(ValueError):
        kdn.forward_gdr(q, k, v, a[..., :1], b)
    with pytest.raises(ValueError):  # a view that is not contiguous
        kdn.forward_gdr(q, k, v.transpose(0, 1).contiguous().transpose(0, 1)[:, ::2],
                        a[:, ::2], b[:, ::2])
    with pytest.raises(ValueError):
        kdn.forward_gdr(q, k, v, a, b, S0=torch.zeros(1, 2, 32, 16, device="cuda"))
    with pytest.raises(ValueError):
        kdn.forward_gdr(q.cpu(), k, v, a, b)
    with pytest.raises(kdn.KdnError):
        kdn.forward_gdr(q, k, v, a, b, scale=-1.0)
    with pytest.raises(ValueError):
        kdn.backward_gdr(q, k, v, a, b, dO=v[:, :4])
    with pytest.raises(TypeError):
        kdn.backward_gdr(q, k, v, a, b, dS_T=torch.zeros(1, 2, 32, 32, device="cuda").bfloat16())
    with pytest.raises(ValueError):
        kdn.decode_step_gdr(q[0], k[0], v[0], a[0], b[0], torch.zeros(9, 1, 32, 32, device="cuda"))


def test_too_many_heads():
    """32-bit offsets within a chunk and the grid bound the heads of a call."""
    H = 65552
    z = [torch.zeros(1, 9, n, 16, dtype=torch.bfloat16, device="cuda") for n in (16, 16, H)]
    g = torch.zeros(1, 9, H, dtype=torch.bfloat16, device="cuda")
    for f in (kdn.forward_gdr, kdn.backward_gdr):
        with pytest.raises(kdn.KdnError):
            f(*z, g, g)
    R = (1 << 19) // 16 + 1  # rows of 16 heads
    z = [torch.zeros(R, 1, 16, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    v = torch.zeros(R, 16, 16, dtype=torch.bfloat16, device="cuda")
    g = torch.zeros(R, 16, dtype=torch.bfloat16, device="cuda")
    slots = torch.zeros(R, dtype=torch.int32, device="cuda")
    with pytest.raises(kdn.KdnError):
        kdn.decode_step_gdr(*z, v, g, g, torch.zeros(1, 16, 16, 16, device="cuda"), slots)


@pytest.mark.parametrize("B,T,H", [(1, 12, 2), (1, 13, 2), (64, 32, 8), (64, 33, 8), (63, 32, 8)])
def test_either_side_of_the_short_rows(B, T, H):
    """The forms that run token by token and over chunks, where one takes over from the other."""
    x = R.draw(T, B, T, H, H, 16, 32, state=True)
    d = dev(x, "f32")
    o, S = kdn.forward_gdr(*[d[n] for n in NAMES], S0=d["S0"])
    want_o, want_S = R.forward(x)
    assert near(o, want_o, "f32") and near(S, want_S, "f32")
