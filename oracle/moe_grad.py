"""Backward pass of the expert block (second half of the pre-norm block).

TEST INFRASTRUCTURE (part of the CPU oracle): only tests use it.  It shares no
code with the GPU path.

Forward (``layer.moe``): n = act(Norm(x~; g2)); per slot with expert e != 0 and
gate p, y = p Wd_e (silu(Wg_e n) * (Wu_e n)), added to x~.  What is returned is
the gradient of <dx, x'> with the choice of experts held constant and the
rounding of n passed through.

``bounds`` follows the roundings of an implementation that sums products in
fp32 and rounds dG, dU and p h once to the activation type before the
products that follow, to first order, as a largest error of every element.
"""
from __future__ import annotations

import numpy as np

from .layer import EPS, rmsnorm, to_native

U32 = 2.0 ** -24
UNIT = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def _sigmoid(G):
    return 0.5 * (1.0 + np.tanh(0.5 * G))


def moe_backward(xt, L, eidx, egate, dx, act, bounds=False):
    """Gradients {dxt, dg2, g_gate, dWgate, dWup, dWdown}; with ``bounds`` also
    the largest error of each element for operands and outputs held in ``act``."""
    x, dx = np.asarray(xt, np.float64), np.asarray(dx, np.float64)
    g2 = np.asarray(L["g2"], np.float64)
    N, d = x.shape
    k = eidx.shape[1]
    r = 1.0 / np.sqrt(np.mean(x * x, axis=1, keepdims=True) + EPS)
    n = to_native(rmsnorm(x, g2), act).astype(np.float64)
    dn, edn = np.zeros((N, d)), np.zeros((N, d))
    out = dict(g_gate=np.zeros((N, k)))
    err = dict(g_gate=np.zeros((N, k)))
    for name, w in (("dWgate", "Wg"), ("dWup", "Wu"), ("dWdown", "Wd")):
        out[name] = np.zeros(np.shape(L[w]))
        err[name] = np.zeros(np.shape(L[w]))
    u_op = UNIT.get(act, U32)

    def gam(K):  # a sum of K products in fp32, in any order
        return 2.0 * (K + 4) * U32

    c = 32 * U32  # a handful of fp32 steps, exp and reciprocal among them
    for e in range(1, np.shape(L["Wg"])[0] + 1):
        i, s = np.nonzero(np.asarray(eidx) == e)
        if not len(i):
            continue
        Wg, Wu, Wd = (np.asarray(L[w][e - 1], np.float64) for w in ("Wg", "Wu", "Wd"))
        f = Wg.shape[0]
        ni, di, p = n[i], dx[i], np.asarray(egate, np.float64)[i, s][:, None]
        G, U, q = ni @ Wg.T, ni @ Wu.T, di @ Wd
        sg = _sigmoid(G)
        a = G * sg
        h, t = a * U, sg * (1.0 + G * (1.0 - sg))
        dG, dU = p * q * U * t, p * q * a
        out["g_gate"][i, s] = (q * h).sum(axis=1)
        out["dWgate"][e - 1], out["dWup"][e - 1] = dG.T @ ni, dU.T @ ni
        out["dWdown"][e - 1] = di.T @ (p * h)
        np.add.at(dn, i, dG @ Wg + dU @ Wu)
        if not bounds:
            continue
        A = np.abs
        eG, eU = gam(d) * (A(ni) @ A(Wg).T), gam(d) * (A(ni) @ A(Wu).T)
        eq = gam(d) * (A(di) @ A(Wd))
        ea = A(t) * eG + c * A(a) + eG * eG
        eh = ea * A(U) + A(a) * eU + c * A(h)
        err["g_gate"][i, s] = (eq * A(h) + A(q) * eh).sum(axis=1) + gam(f) * (A(q * h)).sum(axis=1)
        et = 0.5 * eG + c * sg * (1.0 + A(G) * (1.0 - sg))
        edG = A(p) * (eq * A(U * t) + A(q * t) * eU + A(q * U) * et) + (c + u_op) * A(dG)
        edU = A(p) * (eq * A(a) + A(q) * ea) + (c + u_op) * A(dU)
        ehp = A(p) * eh + (c + u_op) * A(p * h)
        rows = gam(len(i))
        err["dWgate"][e - 1] = edG.T @ A(ni) + rows * (A(dG).T @ A(ni))
        err["dWup"][e - 1] = edU.T @ A(ni) + rows * (A(dU).T @ A(ni))
        err["dWdown"][e - 1] = A(di).T @ ehp + rows * (A(di).T @ A(p * h))
        np.add.at(edn, i, edG @ A(Wg) + edU @ A(Wu)
                  + gam(2 * f + k) * (A(dG) @ A(Wg) + A(dU) @ A(Wu)))
    gx = dn * g2
    dot = (gx * x).sum(axis=1, keepdims=True)
    out["dxt"] = dx + r * gx - r ** 3 * x * dot / d
    out["dg2"] = (dn * x * r).sum(axis=0)
    if not bounds:
        return out
    A = np.abs
    egx = edn * A(g2)
    err["dxt"] = r * egx + r ** 3 * A(x) * (egx * A(x)).sum(axis=1, keepdims=True) / d \
        + c * (A(dx) + r * A(gx) + r ** 3 * A(x) * (A(gx) * A(x)).sum(axis=1, keepdims=True) / d)
    err["dg2"] = (edn * A(x) * r).sum(axis=0) + gam(N) * (A(dn * x) * r).sum(axis=0)
    for name in out:
        err[name] = err[name] + (U32 if name == "g_gate" else u_op) * A(out[name]) + 1e-37
    return out, err
