"""Gated delta rule and beam search in float64 numpy, from their definitions: the references of the
operators' tests, and their seeded inputs."""

from __future__ import annotations

import numpy as np
import torch


def to_bf16(x):
    """float64 values as bf16 stores them."""
    return torch.from_numpy(np.asarray(x, dtype=np.float32)).to(torch.bfloat16).double().numpy()


def draw(seed, B, T, H, Hk, dk, dv, dtype="f32", N=None, state=False, gates="usual"):
    """Inputs as float64 arrays of values that the stored type holds exactly. N: sequences of a
    packed batch (else B)."""
    g = np.random.default_rng(seed)
    x = {}
    for name in ("q", "k"):
        y = g.standard_normal((B, T, Hk, dk))
        x[name] = y / np.linalg.norm(y, axis=-1, keepdims=True)
    x["v"] = g.standard_normal((B, T, H, dv))
    x["dO"] = g.standard_normal((B, T, H, dv))
    x["beta"] = 1 / (1 + np.exp(-g.standard_normal((B, T, H))))
    if gates == "usual":
        x["alpha"] = np.exp(-np.exp(g.uniform(-4.6, 0, H)) * np.log1p(np.exp(
            g.standard_normal((B, T, H)))))
    elif gates == "one":      # nothing decays
        x["alpha"] = np.ones((B, T, H))
    elif gates == "strong":   # decays of up to 1e-6 per token
        x["alpha"] = 10.0 ** g.uniform(-6, 0, (B, T, H))
    elif gates == "zeros":    # the memory is cleared now and then, also twice in a row
        x["alpha"] = np.where(g.random((B, T, H)) < 0.1, 0.0, g.uniform(0.5, 1, (B, T, H)))
        x["beta"] = np.where(g.random((B, T, H)) < 0.2, 0.0, 2 * x["beta"])
    elif gates == "scaled":   # keys, values and queries of very different size from row to row
        x["alpha"] = g.uniform(0.8, 1, (B, T, H))
        s = 2.0 ** g.integers(-6, 1, (B, T, Hk, 1))
        x["k"] = x["k"] * s
        x["q"] = x["q"] * 2.0 ** g.integers(-20, 20, (B, T, Hk, 1))
        x["v"] = x["v"] * 2.0 ** g.integers(-10, 10, (B, T, H, 1))
    elif gates == "jumps":    # columns whose values change by up to 2^40 from one stretch to the next
        x["alpha"] = np.full((B, T, H), 0.25)
        for name in ("v", "dO"):
            s = 2.0 ** g.integers(-20, 21, (B, T // 40 + 1, H, dv))
            x[name] = x[name] * np.repeat(s, 40, axis=1)[:, :T]
    else:
        raise ValueError(gates)
    x = {n: (to_bf16(y) if dtype == "bf16" else y.astype(np.float32).astype(np.float64))
         for n, y in x.items()}
    n = B if N is None else N
    x["S0"] = g.standard_normal((n, H, dk, dv)).astype(np.float32) * np.float32(0.1)
    x["dS_T"] = g.standard_normal((n, H, dk, dv)).astype(np.float32)
    if not state:
        x["S0"] = x["dS_T"] = None
    return x


def spans(x, cu):
    B, T = x["v"].shape[:2]
    if cu is None:
        return [(b, 0, T) for b in range(B)]
    return [(0, int(cu[i]), int(cu[i + 1])) for i in range(len(cu) - 1)]


def forward(x, cu=None, scale=None):
    """(o [B,T,H,dv], S_T [N,H,dk,dv]) token by token."""
    B, T, H, dv = x["v"].shape
    Hk, dk = x["k"].shape[2:]
    scale = dk ** -0.5 if scale is None else scale
    sp = spans(x, cu)
    o = np.zeros((B, T, H, dv))
    S_T = np.zeros((len(sp), H, dk, dv))
    for n, (b, t0, t1) in enumerate(sp):
        S = np.zeros((H, dk, dv)) if x["S0"] is None else x["S0"][n].astype(np.float64)
        for t in range(t0, t1):
            k = np.repeat(x["k"][b, t], H // Hk, 0)
            q = np.repeat(x["q"][b, t], H // Hk, 0)
            S = x["alpha"][b, t][:, None, None] * S
            u = x["beta"][b, t][:, None] * (x["v"][b, t] - np.einsum("hij,hi->hj", S, k))
            S = S + k[:, :, None] * u[:, None, :]
            o[b, t] = scale * np.einsum("hij,hi->hj", S, q)
        S_T[n] = S
    return o, S_T


def backward(x, cu=None, scale=None):
    """Gradients of sum(o dO) + sum(S_T dS_T): the adjoint recurrence, token by token, with every
    state kept."""
    B, T, H, dv = x["v"].shape
    Hk, dk = x["k"].shape[2:]
    scale = dk ** -0.5 if scale is None else scale
    sp = spans(x, cu)
    g = {n: np.zeros(x[n].shape) for n in ("q", "k", "v", "alpha", "beta")}
    dS0 = np.zeros((len(sp), H, dk, dv))
    for n, (b, t0, t1) in enumerate(sp):
        S = np.zeros((H, dk, dv)) if x["S0"] is None else x["S0"][n].astype(np.float64)
        kept = []
        for t in range(t0, t1):
            k = np.repeat(x["k"][b, t], H // Hk, 0)
            a, be = x["alpha"][b, t][:, None], x["beta"][b, t][:, None]
            e = x["v"][b, t] - a * np.einsum("hij,hi->hj", S, k)
            S1 = a[:, :, None] * S + k[:, :, None] * (be * e)[:, None, :]
            kept.append((S, e, S1))
            S = S1
        dS = np.zeros((H, dk, dv)) if x["dS_T"] is None else x["dS_T"][n].astype(np.float64)
        for t in reversed(range(t0, t1)):
            S, e, S1 = kept[t - t0]
            k = np.repeat(x["k"][b, t], H // Hk, 0)
            q = np.repeat(x["q"][b, t], H // Hk, 0)
            a, be, dO = x["alpha"][b, t][:, None], x["beta"][b, t][:, None], scale * x["dO"][b, t]
            dq = np.einsum("hij,hj->hi", S1, dO)
            dS = dS + q[:, :, None] * dO[:, None, :]
            du = np.einsum("hij,hi->hj", dS, k)
            dkk = np.einsum("hij,hj->hi", dS, be * e)
            de = be * du
            Sk = np.einsum("hij,hi->hj", S, k)
            dkk -= a * np.einsum("hij,hj->hi", S, de)
            g["v"][b, t] = de
            g["beta"][b, t] = (du * e).sum(-1)
            g["alpha"][b, t] = (dS * S).sum((-1, -2)) - (de * Sk).sum(-1)
            g["q"][b, t] = dq.reshape(Hk, H // Hk, dk).sum(1)
            g["k"][b, t] = dkk.reshape(Hk, H // Hk, dk).sum(1)
            dS = a[:, :, None] * (dS - k[:, :, None] * de[:, None, :])
        dS0[n] = dS
    return {**{"d" + m: y for m, y in g.items()}, "dS0": dS0}


def beam_select(logits, scores, done, end_token):
    """(scores, token, parent, done) of one batch of [N,W,V] float64 logits."""
    N, W, V = logits.shape
    out = [np.zeros((N, W)), np.zeros((N, W), int), np.zeros((N, W), int), np.zeros((N, W), bool)]
    big = float(np.finfo(np.float32).max)
    for n in range(N):
        cand = []
        for w in range(W):
            if done is not None and done[n, w]:
                cand.append((scores[n, w], w, 0.0, end_token))
                cand += [(-np.inf, w, -np.inf, y) for y in range(V) if y != end_token]
                continue
            x = np.where(np.isnan(logits[n, w]), -np.inf, np.minimum(logits[n, w], big))
            m = x.max()
            norm = 0.0 if m == -np.inf else np.log(np.exp(x - m).sum())
            # the W best of a beam are its W largest logits
            for y in np.argsort(-x, kind="stable")[:W]:
                s = -np.inf if x[y] == -np.inf else scores[n, w] + ((x[y] - m) - norm)
                cand.append((s, w, x[y], int(y)))
        cand.sort(key=lambda c: (-c[0], c[1], -c[2], c[3]))
        for i, (s, w, _, y) in enumerate(cand[:W]):
            out[0][n, i], out[1][n, i], out[2][n, i] = s, y, w
            out[3][n, i] = y == end_token or (done is not None and bool(done[n, w]))
    return out


def beam_reorder(parent, slot_idx, pools):
    """(slots, moved copies of the pools): first children keep, later ones take free slots."""
    pools = [p.copy() for p in pools]
    slots = np.zeros_like(slot_idx)
    for n in range(parent.shape[0]):
        W = parent.shape[1]
        free = [b for b in range(W) if b not in parent[n]]
        seen, moves = set(), []
        for w in range(W):
            p = int(parent[n, w])
            if 0 <= p < W and p not in seen:
                seen.add(p)
                slots[n, w] = slot_idx[n, p]
            else:
                slots[n, w] = slot_idx[n, free.pop(0)]
                if 0 <= p < W:
                    moves.append((int(slot_idx[n, p]), int(slots[n, w])))
        for pool in pools:
            for a, b in moves:
                if 0 <= a < len(pool) and 0 <= b < len(pool):
                    pool[b] = pool[a]
    return slots, pools
