"""fp64 reference of the layer's products in 8-bit integers (triroute_i8_quantize,
triroute_linear_i8, triroute_qkv_i8, triroute_moe_i8).  TEST INFRASTRUCTURE.

Weights are (codes [rows, cols], scale [rows]); tokens are quantised row by row.  The functions
return the exact result and, for every element, a bound on the error of an implementation with
exact integer sums, fp32 scaling and the stated roundings (U = 2^-24, half a step of fp32;
u = half a step of the activation dtype).
"""
from __future__ import annotations

import numpy as np

from .layer import EPS, ROPE_THETA, rmsnorm

U = 2.0 ** -24
HALF_STEP = {"bf16": 2.0 ** -8, "f32": U}


def quantize(x):
    """Codes and fp32 scales of the rows of x (fp32 values): 127 x / a rounded half to even.
    The fp64 quotient of 127 x (exact) and a lies on a border of two codes only if the
    exact one does, and is a border itself then: borders are k + 1/2 with k <= 126, and a quotient
    of two 24-bit numbers times 127 that is none keeps at least 2^-33 away from it."""
    x = np.asarray(x, np.float32)
    bits = np.abs(x)
    a = bits.max(axis=1)                      # NaN if one is there
    bad = ~np.isfinite(a)
    safe = np.where(bad | (a == 0), np.float32(1), a)
    clean = np.where(bad[:, None], np.float32(0), x).astype(np.float64)
    codes = np.rint(127.0 * clean / safe.astype(np.float64)[:, None])
    with np.errstate(invalid="ignore"):
        scale = np.where(bad, np.float32(np.nan), (a / np.float32(127)).astype(np.float32))
    return codes.astype(np.int8), scale.astype(np.float32)


def matrix(codes, scale):
    return codes.astype(np.float64) * np.asarray(scale, np.float64)[:, None]


def product(q, s, w, t):
    """Sums of products of codes times both scales, and the error of forming it in fp32: the
    sum's rounding and two products."""
    y = (q.astype(np.float64) @ w.astype(np.float64).T) * np.asarray(s, np.float64)[:, None] \
        * np.asarray(t, np.float64)[None]
    return y, 3.01 * U * np.abs(y) + 2.0 ** -148


def linear(x, w, t, act, residual=None):
    q, s = quantize(x)
    y, err = product(q, s, w, t)
    if residual is not None:
        y = y + np.asarray(residual, np.float64)
    # the sum with the residual in fp32, then the rounding to act
    return y, err + (1.01 * U + 1.01 * HALF_STEP[act]) * np.abs(y) + 1e-38


def rotate(y, err, pos, dh, act):
    """Rotate-half RoPE.  cos and sin are fp32 values of an angle reduced in fp64 and rounded to
    fp32: off by pi U, and an ulp or two of the functions, 2^-21 in all; then two products and a sum."""
    h = dh // 2
    ang = np.asarray(pos, np.float64)[:, None, None] * ROPE_THETA ** (-2.0 * np.arange(h) / dh)
    c, s = np.cos(ang), np.sin(ang)
    y, err = y.reshape(len(pos), -1, dh), err.reshape(len(pos), -1, dh)
    a, b, ea, eb = y[..., :h], y[..., h:], err[..., :h], err[..., h:]
    out = np.concatenate([a * c - b * s, a * s + b * c], axis=-1)
    slack = (np.abs(a) + np.abs(b)) * (2.0 ** -21 + 2 * U) + ea + eb
    e = np.concatenate([slack, slack], axis=-1) + (1.01 * U + 1.01 * HALF_STEP[act]) * np.abs(out)
    return out.reshape(len(pos), -1), e.reshape(len(pos), -1)


def qkv(n1, Wq, Wk, Wv, pos, dh, act):
    """[(value, bound)] of q, k, v; W*: (codes, scale)."""
    q, s = quantize(n1)
    out = []
    for w, turned in ((Wq, True), (Wk, True), (Wv, False)):
        y, err = product(q, s, *w)
        out.append(rotate(y, err, pos, dh, act) if turned
                   else (y, err + 1.01 * HALF_STEP[act] * np.abs(y)))
    return out


def _uncertain(h, rel, off):
    """Codes of rows that an implementation whose h is off by up to rel |h| + off may set one step
    elsewhere; and the relative error of its scales."""
    a = np.abs(h).max(axis=1, keepdims=True)
    with np.errstate(divide="ignore", invalid="ignore"):
        top = np.where((np.abs(h) >= a * (1 - 2 * rel)) & (a > 0), rel + off / a, 0.0).max(axis=1, keepdims=True)
        t = np.where(a > 0, 127.0 * np.abs(h) / np.where(a > 0, a, 1), 0.0)
        t_off = np.where(a > 0, 127.0 * off / np.where(a > 0, a, 1), 0.0)
    near = np.abs(np.abs(t - np.floor(t)) - 0.5) <= 1.01 * (t * (rel + top) + t_off)
    return near, top[:, 0] + U


def moe(xt, g2, Wg, Wu, Wd, eidx, egate, act, eps=EPS):
    """x_out of triroute_moe_i8 and its bound; Wg, Wu: (codes [E, f, d], scale [E, f]), Wd:
    (codes [E, d, f], scale [E, d]).  The normalised token is an fp32 value before it is
    quantised, and so is h; h of bf16 layers is formed in fp32: the exponential's argument
    (a sum, three products, a constant) is off by 5 U |G| and moves silu by that much at most; the sums, the
    other products, exponential and quotient are off by 20 U together, so that h is off by less than
    5 (|G| + 8) U; and a sigmoid below 2^-126 (the quotient's smallest) may be 0."""
    xt = np.asarray(xt, np.float64)
    n2 = rmsnorm(xt, g2, eps).astype(np.float32)
    # (an fp64 norm that is a last place elsewhere rounds one n2 in 2^29 to its neighbour)
    nq, ns = quantize(n2)
    y = np.zeros_like(xt)
    err = np.zeros_like(xt)
    for e in range(1, Wg[0].shape[0] + 1):
        i, slot = np.nonzero(np.asarray(eidx) == e)
        if not len(i):
            continue
        g = np.asarray(egate, np.float64)[i, slot][:, None]
        G, _ = product(nq[i], ns[i], Wg[0][e - 1], Wg[1][e - 1])
        V, _ = product(nq[i], ns[i], Wu[0][e - 1], Wu[1][e - 1])
        with np.errstate(over="ignore"):
            h = (G / (1.0 + np.exp(-G)) * V).astype(np.float32)
        rel = 5 * (np.abs(G) + 8) * U if act == "bf16" else np.full(h.shape, 1.01 * 2 * U)
        hq, hs = quantize(h)
        off = np.zeros_like(G)
        if act == "bf16":
            off = 2.0 ** -125 * np.abs(G * V) * (G < -80) + 2.0 ** -148
        moved, hrel = _uncertain(h.astype(np.float64), rel, off)
        Y, eY = product(hq, hs, Wd[0][e - 1], Wd[1][e - 1])
        wd = np.abs(matrix(Wd[0][e - 1], Wd[1][e - 1]))
        eY = eY + np.abs(Y) * hrel[:, None] + (moved * np.asarray(hs, np.float64)[:, None]) @ wd.T
        np.add.at(y, i, g * Y)
        np.add.at(err, i, g * eY + 3 * U * (eidx.shape[1] + 1) * np.abs(g * Y))
    out = xt + y
    # (what is rounded at the end is the sum as formed, up to err further out: half its step)
    return out, err + (2 * U + 1.01 * HALF_STEP[act]) * (np.abs(out) + err) + 2 * U * np.abs(y)
