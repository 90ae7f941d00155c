"""Tolerances of the gated-delta layer's tests that count an error from what a
head held when it was made, not from the largest numbers of the whole call."""
from __future__ import annotations

import numpy as np

from layer_testutil import HALF


def _unit(x, norm, eps):
    return x / np.sqrt((x * x).sum(-1, keepdims=True) + eps) if norm else x


def sizes(d, lens, h0=None, norm=False, eps=1e-6):
    """Bounds of the terms of every o and of the last states, token after token
    in fp64: with M_t = max(e^{g_t} M_{t-1}, |S_t|) of a state's column (an error
    made while the column was M large has since decayed as the column has),
    K^-1/2 |q_t| M_t for o [T, Hv, V] and M_T for the states [B, Hv, V]."""
    q, k, v, g, beta = (None if d[n] is None else d[n].double().numpy() for n in ("q", "k", "v", "g", "beta"))
    (T, Hk, K), (Hv, V) = k.shape, v.shape[1:]
    head = np.arange(Hv) // (Hv // Hk)
    k = _unit(k, norm, eps)[:, head]
    qn = np.ones((T, Hv)) if q is None else np.linalg.norm(_unit(q, norm, eps), axis=-1)[:, head]
    o, last, at = np.zeros((T, Hv, V)), [], 0
    for b, n in enumerate(lens):
        S = np.zeros((Hv, K, V)) if h0 is None else h0[b].double().numpy().copy()
        M = np.sqrt((S * S).sum(1))
        for t in range(at, at + n):
            a = np.ones(Hv) if g is None else np.exp(g[t])
            bt = np.ones(Hv) if beta is None else beta[t]
            S *= a[:, None, None]
            u = bt[:, None] * (v[t] - np.matmul(k[t][:, None], S)[:, 0])
            S += k[t][:, :, None] * u[:, None]
            M = np.maximum(a[:, None] * M, np.sqrt((S * S).sum(1)))
            o[t] = K ** -0.5 * qn[t][:, None] * M
        last.append(M)
        at += n
    return o, np.stack(last)


def near(got, ref, size, bar, what=""):
    """|got - ref| <= half a step of got's type + bar * max(|ref|, size)."""
    g, r = got.detach().cpu().double().numpy(), np.asarray(ref)
    assert g.shape == r.shape and np.isfinite(r).all() and np.isfinite(g).all(), what
    tol = HALF[got.dtype] * (1 + 2.0 ** -7) * np.abs(r) + bar * np.maximum(np.abs(r), size)
    worst = np.max(np.abs(g - r) / np.maximum(tol, 1e-300))
    assert worst <= 1.0, "%s: %.3g times the tolerance" % (what, worst)
