"""The C entry points of the gated delta rule and of beam search refuse bad arguments on the host, with the
documented status, before anything runs."""

import ctypes

import pytest

from paper_2609_07816_amd import kdn

F = ctypes.c_float
INVALID, UNSUPPORTED = kdn.KDN_ERR_INVALID_ARG, kdn.KDN_ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def L():
    return kdn.lib()


# addresses that nothing reads: the checks run before any launch; 4 GiB apart
def P(i):
    return (i + 1) << 32


BASE = dict(q=P(0), k=P(1), v=P(2), alpha=P(3), beta=P(4), S0=None, o=P(6), S_T=P(7), cu=None, N=1,
            B=1, T=100, H=4, Hk=2, dk=64, dv=64, dtype=1, scale=0.125, ws=P(9), ws_bytes=1 << 30)


def forward(L, **kw):
    c = dict(BASE, **kw)
    return L.kdn_forward_gdr(*[c[n] for n in ("q", "k", "v", "alpha", "beta", "S0", "o", "S_T", "cu",
                                              "N", "B", "T", "H", "Hk", "dk", "dv", "dtype")],
                             F(c["scale"]), c["ws"], c["ws_bytes"], None)


def backward(L, **kw):
    c = dict(BASE, dO=P(20), dS_T=None, dq=P(21), dk_out=P(22), dv_out=P(23), dalpha=P(24),
             dbeta=P(25), dS0=P(26))
    c.update(kw)
    return L.kdn_backward_gdr(*[c[n] for n in ("q", "k", "v", "alpha", "beta", "S0", "cu", "N", "B",
                                               "T", "H", "Hk", "dk", "dv", "dtype")], F(c["scale"]),
                              *[c[n] for n in ("dO", "dS_T", "dq", "dk_out", "dv_out", "dalpha",
                                               "dbeta", "dS0", "ws", "ws_bytes")], None)


COMMON = [
    (dict(q=None), INVALID), (dict(v=None), INVALID), (dict(beta=None), INVALID),
    (dict(T=0), INVALID), (dict(N=2), INVALID), (dict(cu=P(12), N=3, B=2), INVALID),
    (dict(Hk=3), INVALID), (dict(Hk=0), INVALID), (dict(H=0), INVALID), (dict(dtype=2), INVALID),
    (dict(scale=0.0), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(dk=48), UNSUPPORTED), (dict(dv=256), UNSUPPORTED),
    (dict(H=65536, Hk=1), UNSUPPORTED), (dict(cu=P(12), N=1 << 18), UNSUPPORTED),
    (dict(T=(1 << 22) + 1), INVALID),
    (dict(q=P(0) + 2), INVALID), (dict(ws_bytes=64), kdn.KDN_ERR_WORKSPACE),
    (dict(ws=None), kdn.KDN_ERR_WORKSPACE), (dict(ws=P(9) + 4), INVALID),
]


@pytest.mark.parametrize("call", [forward, backward])
@pytest.mark.parametrize("kw,status", COMMON, ids=str)
def test_refusals_of_both_directions(L, call, kw, status):
    assert call(L, **kw) == status
    assert L.kdn_last_error()


@pytest.mark.parametrize("kw", [dict(o=None), dict(o=P(2)), dict(o=P(7)), dict(S_T=P(3)),
                                dict(S0=P(7) + 16), dict(S0=P(6)), dict(ws=P(6)), dict(ws=P(7))],
                         ids=str)
def test_forward_overlaps(L, kw):
    assert forward(L, **kw) == INVALID


@pytest.mark.parametrize("kw", [dict(dq=None), dict(dbeta=None), dict(dq=P(0)), dict(dv_out=P(20)),
                                dict(dalpha=P(25)), dict(dS0=P(9)), dict(dk_out=P(21))], ids=str)
def test_backward_overlaps(L, kw):
    assert backward(L, **kw) == INVALID


def test_workspace_queries(L):
    fw, bw = L.kdn_forward_gdr_workspace_bytes, L.kdn_backward_gdr_workspace_bytes
    ok = (1, 1, 100, 4, 2, 64, 64, 1, 0)
    assert fw(*ok) > 0 and bw(*ok) > fw(*ok)
    assert fw(1, 1, 8, 4, 2, 64, 64, 1, 0) == 0  # token by token: none needed
    assert bw(1, 1, 1, 4, 2, 64, 64, 1, 0) > 0
    for bad in ((0, 1, 100, 4, 2, 64, 64, 1, 0), (1, 1, 100, 4, 3, 64, 64, 1, 0),
                (1, 1, 100, 4, 2, 48, 64, 1, 0), (1, 1, 100, 4, 2, 64, 64, 5, 0)):
        assert fw(*bad) == 0 and bw(*bad) == 0
    # a packed batch has at most one chunk more per sequence
    assert fw(9, 1, 6400, 4, 2, 64, 64, 1, 1) == fw(1, 1, 109 * 64, 4, 2, 64, 64, 1, 0)


DECODE = dict(q=P(0), k=P(1), v=P(2), alpha=P(3), beta=P(4), S=P(5), slot=None, o=P(7), R=4, slots=8, H=4,
              Hk=2, dk=64, dv=64, dtype=1)


@pytest.mark.parametrize("kw,status", [
    (dict(S=None), INVALID), (dict(R=-1), INVALID), (dict(slots=0), INVALID), (dict(R=9), INVALID),
    (dict(Hk=3), INVALID), (dict(dk=24), UNSUPPORTED), (dict(o=P(2)), INVALID), (dict(o=P(5)), INVALID),
    (dict(S=P(5) + 4), INVALID), (dict(S=P(1)), INVALID), (dict(R=(1 << 17) + 1, slots=1 << 18),
                                                          UNSUPPORTED)], ids=str)
def test_decode_refusals(L, kw, status):
    c = dict(DECODE, **kw)
    assert L.kdn_decode_step_gdr(*c.values(), F(0.125), None) == status


SELECT = dict(logits=P(0), scores=P(1), done=None, N=2, W=4, V=100, dtype=1, end=2, out=P(4), token=P(5),
              parent=P(6), done_out=P(7), ws=P(8), ws_bytes=1 << 24)


@pytest.mark.parametrize("kw,status", [
    (dict(logits=None), INVALID), (dict(parent=None), INVALID), (dict(W=0), INVALID),
    (dict(W=65), UNSUPPORTED), (dict(N=65536, W=1), UNSUPPORTED), (dict(V=(1 << 30) + 1), UNSUPPORTED),
    (dict(end=-1), INVALID), (dict(end=100), INVALID), (dict(dtype=9), INVALID),
    (dict(logits=P(0) + 1), INVALID), (dict(out=P(1)), INVALID), (dict(token=P(6)), INVALID),
    (dict(done=P(7)), INVALID), (dict(ws_bytes=8), kdn.KDN_ERR_WORKSPACE), (dict(ws=P(8) + 8), INVALID)],
    ids=str)
def test_select_refusals(L, kw, status):
    assert L.kdn_beam_select(*dict(SELECT, **kw).values(), None) == status


REORDER = dict(parent=P(0), slot=P(1), out=P(2), N=2, W=4, slots=16, S=P(3), s_bytes=4096, P=P(4),
               p_bytes=64)


@pytest.mark.parametrize("kw,status", [
    (dict(S=None), INVALID), (dict(out=P(1)), INVALID), (dict(slots=0), INVALID),
    (dict(s_bytes=0), INVALID), (dict(p_bytes=0), INVALID), (dict(s_bytes=4098), INVALID),
    (dict(S=P(3) + 2), INVALID), (dict(W=65), UNSUPPORTED), (dict(N=0), INVALID),
    (dict(out=P(3) + 64), INVALID), (dict(P=P(3) + 4096), INVALID), (dict(slot=P(4) + 64), INVALID)], ids=str)
def test_reorder_refusals(L, kw, status):
    assert L.kdn_beam_reorder(*dict(REORDER, **kw).values(), None) == status
