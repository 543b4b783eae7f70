"""The float64 references of the gated delta rule and of beam search against other forms of the same
definitions (CPU), and the host-side refusals of their entry points."""

import ctypes

import numpy as np
import pytest

import gdr_ref as R
from paper_2609_07816_amd import kdn

F = ctypes.c_float


@pytest.mark.parametrize("cu", [None, [0, 3, 3, 9]])
def test_backward_against_differences(cu):
    """Central differences of the loss in every input: h = 1e-5 leaves h^2 = 1e-10 of curvature and
    1e-16 / h = 1e-11 of rounding."""
    x = R.draw(2, 1 if cu else 2, 9, 2, 1, 3, 2, N=3 if cu else None, state=True, gates="usual")
    x["S0"], x["dS_T"] = (x[n].astype(np.float64) for n in ("S0", "dS_T"))
    got = R.backward(x, cu)

    def loss():
        o, S = R.forward(x, cu)
        return (o * x["dO"]).sum() + (S * x["dS_T"]).sum()

    h = 1e-5
    for name in ("q", "k", "v", "alpha", "beta", "S0"):
        num = np.zeros(x[name].shape)
        for i in np.ndindex(*x[name].shape):
            keep = x[name][i]
            x[name][i] = keep + h
            up = loss()
            x[name][i] = keep - h
            num[i] = (up - loss()) / (2 * h)
            x[name][i] = keep
        err = np.abs(num - got["d" + name]).max()
        assert err <= 1e-8 * max(1.0, np.abs(num).max()), name


def test_beam_select_is_the_best_of_all_candidates():
    g = np.random.default_rng(0)
    logits, scores = g.standard_normal((4, 3, 11)), g.standard_normal((4, 3))
    got = R.beam_select(logits, scores, None, 0)
    lp = logits - np.log(np.exp(logits).sum(-1, keepdims=True))
    total = (scores[..., None] + lp).reshape(4, -1)
    at = np.argsort(-total, axis=-1)[:, :3]
    assert np.array_equal(got[2] * 11 + got[1], at)
    assert np.allclose(got[0], np.take_along_axis(total, at, -1))


def P(i):
    return ctypes.c_void_p(0x1000000 * (i + 1))


@pytest.fixture(scope="module")
def L():
    return kdn.lib()


def fwd(L, ptrs=None, S0=None, S_T=None, cu=None, N=1, B=1, T=8, H=2, Hk=2, dk=64, dv=64, dtype=1,
        scale=0.125, ws=None, ws_bytes=0):
    p = [P(i) for i in range(6)] if ptrs is None else ptrs
    return L.kdn_forward_gdr(*p[:5], S0, p[5], S_T, cu, N, B, T, H, Hk, dk, dv, dtype, F(scale), ws,
                             ws_bytes, None)


def test_gdr_argument_errors(L):
    p = [P(i) for i in range(6)]
    bad = kdn.KDN_ERR_INVALID_ARG
    for i in range(6):
        assert fwd(L, ptrs=p[:i] + [None] + p[i + 1:]) == bad
    assert fwd(L, T=0) == bad
    assert fwd(L, N=2) == bad
    assert fwd(L, cu=P(20), N=2, B=2) == bad
    assert fwd(L, Hk=0) == bad
    assert fwd(L, H=3, Hk=2) == bad
    assert fwd(L, scale=0.0) == bad
    assert fwd(L, scale=float("nan")) == bad
    assert fwd(L, dtype=3) == bad
    assert fwd(L, dk=48) == kdn.KDN_ERR_UNSUPPORTED
    assert fwd(L, ptrs=p[:5] + [p[2]]) == bad                    # o is v
    assert fwd(L, ptrs=[ctypes.c_void_p(0x1000008)] + p[1:]) == bad
    assert "q must be 16-byte aligned" in L.kdn_last_error().decode()
    base = 0x7000000
    assert fwd(L, S0=ctypes.c_void_p(base), S_T=ctypes.c_void_p(base + 64)) == bad
    assert fwd(L, S_T=p[1]) == bad
    g = [P(i) for i in range(10, 16)]

    def bwd(ins=p[:5], S0=None, dO=P(6), dST=None, outs=g, ws=P(40), n=1 << 40, H=2, Hk=1, dk=64):
        return L.kdn_backward_gdr(*ins, S0, None, 1, 1, 8, H, Hk, dk, 64, 1, F(1.0), dO, dST, *outs,
                                  ws, n, None)

    need = L.kdn_backward_gdr_workspace_bytes(1, 1, 8, 2, 1, 64, 64, 1, 0)
    assert need > 0 and L.kdn_backward_gdr_workspace_bytes(1, 1, 8, 3, 2, 64, 64, 1, 0) == 0
    assert bwd(ins=[None] + p[1:5]) == bad
    assert bwd(outs=g[:3] + [None] + g[4:]) == bad
    assert bwd(outs=[P(0)] + g[1:]) == bad and bwd(outs=[g[1]] + g[1:]) == bad
    assert bwd(dO=P(12)) == bad                                  # dO is dv
    assert bwd(Hk=3) == bad and bwd(dk=8) == kdn.KDN_ERR_UNSUPPORTED
    assert bwd(n=need - 1) == kdn.KDN_ERR_WORKSPACE and bwd(ws=None) == kdn.KDN_ERR_WORKSPACE
    dec = [P(i) for i in range(5)]

    def step(ptrs=dec, S=P(8), slot=None, o=P(9), R=4, slots=4, H=2, Hk=1, dk=64, dv=64):
        return L.kdn_decode_step_gdr(*ptrs, S, slot, o, R, slots, H, Hk, dk, dv, 1, F(1.0), None)

    assert step(S=None) == bad
    assert step(R=5) == bad                                      # no slot table, too many rows
    assert step(R=-1) == bad
    assert step(Hk=3) == bad
    assert step(o=P(8)) == bad
    assert step(S=P(2)) == bad
    assert step(dv=8) == kdn.KDN_ERR_UNSUPPORTED


def test_beam_argument_errors(L):
    bad, most = kdn.KDN_ERR_INVALID_ARG, kdn.KDN_ERR_UNSUPPORTED
    need = L.kdn_beam_select_workspace_bytes(2, 4, 1000)
    assert need > 0 and L.kdn_beam_select_workspace_bytes(2, 65, 1000) == 0
    assert L.kdn_beam_select_workspace_bytes(2, 4, 0) == 0

    def sel(logits=P(0), scores=P(1), done=None, N=2, W=4, V=1000, dtype=1, end=3, so=P(3), tok=P(4),
            par=P(5), do=None, ws=P(7), n=need):
        return L.kdn_beam_select(logits, scores, done, N, W, V, dtype, end, so, tok, par, do, ws, n,
                                 None)

    assert sel(logits=None) == bad and sel(par=None) == bad
    assert sel(N=0) == bad and sel(V=0) == bad and sel(dtype=5) == bad
    assert sel(W=65) == most and sel(N=40000) == most
    assert sel(end=-1) == bad and sel(end=1000) == bad
    assert sel(logits=ctypes.c_void_p(0x1000001)) == bad
    assert sel(so=P(1)) == bad and sel(tok=P(3)) == bad          # scores in place; shared outputs
    assert sel(ws=None) == kdn.KDN_ERR_WORKSPACE and sel(n=need - 1) == kdn.KDN_ERR_WORKSPACE

    def reo(par=P(0), slot=P(1), out=P(2), N=2, W=4, slots=8, S=P(3), sb=1024, Pp=None, pb=0):
        return L.kdn_beam_reorder(par, slot, out, N, W, slots, S, sb, Pp, pb, None)

    assert reo(S=None) == bad and reo(out=P(1)) == bad and reo(sb=0) == bad
    assert reo(Pp=P(3), pb=16) == bad and reo(Pp=P(4), pb=0) == bad and reo(sb=1022) == bad
    assert reo(W=65) == most
