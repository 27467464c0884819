"""Pins of the 8-bit oracle (CPU)."""
from fractions import Fraction

import numpy as np
import pytest
import torch

import gen
import oracle
from oracle import i8

from _i8 import awkward_rows, experts, routing, tokens, weight


def nearest_even(q):
    lo = q.numerator // q.denominator
    rest = q - lo
    return lo + (rest > Fraction(1, 2) or (rest == Fraction(1, 2) and lo % 2 == 1))


@pytest.mark.parametrize("act", ["bf16", "f32"])
def test_codes_are_the_exact_quotients(act):
    x = np.concatenate([awkward_rows(act), tokens(3, "x", 20, 128, act)])
    q, s = i8.quantize(x)
    for row, c, t in zip(x, q, s):
        if not np.isfinite(row).all():
            assert np.isnan(t) and (c == 0).all()
            continue
        a = max(Fraction(float(abs(v))) for v in row)
        if a == 0:
            assert t == 0 and (c == 0).all()
            continue
        assert t == np.float32(np.float32(a) / np.float32(127))
        assert [nearest_even(127 * Fraction(float(v)) / a) for v in row] == c.tolist()
        assert np.abs(c.astype(int)).max() == 127


def test_values_are_within_half_a_step():
    x = tokens(4, "x", 50, 333, "f32")
    q, s = i8.quantize(x)
    assert (np.abs(i8.matrix(q, s) - x) <= s[:, None] * (0.5 + 127 * 2.0 ** -23)).all()


def test_linear_is_the_product_of_the_values():
    x, (w, t) = tokens(5, "x", 9, 200, "bf16"), weight(5, "W", 17, 200)
    r = gen.normal(5, "r", (9, 17))
    y, err = i8.linear(x, w, t, "f32", r)
    want = torch.nn.functional.linear(torch.from_numpy(i8.matrix(*i8.quantize(x))),
                                      torch.from_numpy(i8.matrix(w, t))).numpy() + r
    np.testing.assert_allclose(y, want, rtol=1e-12, atol=1e-12)
    full = x.astype(np.float64) @ i8.matrix(w, t).T + r
    assert np.linalg.norm(y - full) < 0.05 * np.linalg.norm(full)
    # the same in fp32, as an implementation forms it, keeps the bound
    q, s = i8.quantize(x)
    S = (q.astype(np.int64) @ w.astype(np.int64).T).astype(np.float32)
    f32 = S * s[:, None] * t[None] + r.astype(np.float32)
    assert (np.abs(f32 - y) <= err).all()


def test_rotation_is_the_layer_s():
    y = gen.normal(6, "y", (5, 2 * 64)).astype(np.float64)
    pos = np.array([0, 1, 7, 4095, 100000])
    got, _ = i8.rotate(y, np.zeros_like(y), pos, 64, "f32")
    want = oracle.layer.rope(y.reshape(5, 2, 64), pos)
    np.testing.assert_allclose(got, np.asarray(want).reshape(5, -1), rtol=0, atol=1e-9)


def test_experts_are_near_the_unquantised_ones():
    d, f, E, k, N = 128, 192, 4, 2, 40
    W = experts(7, d, f, E)
    xt, g2 = tokens(7, "xt", N, d, "f32"), (1 + gen.normal(7, "g2", (d,), 0.1))
    eidx, gate = routing(7, N, E, k)
    out, err = i8.moe(xt, g2, *W, eidx, gate, "f32")
    L = dict(cfg=dict(E=E, k=k, d=d, d_ff=f, act="f64"), g2=g2,
             **{n: np.stack([i8.matrix(w[0][e], w[1][e]) for e in range(E)])
                for n, w in zip(("Wg", "Wu", "Wd"), W)})
    want = oracle.moe(xt, L, eidx, gate, "f64")[0]
    y, wy = out - xt, want - xt
    assert np.linalg.norm(y - wy) < 0.05 * np.linalg.norm(wy) and np.linalg.norm(wy) > 1
    # an implementation in fp32 keeps the bf16 bound (its h is formed in fp32)
    _, berr = i8.moe(xt, g2, *W, eidx, gate, "bf16")
    nq, ns = i8.quantize(oracle.layer.rmsnorm(xt, g2).astype(np.float32))
    x32 = xt.copy()
    for i in range(N):
        for s in range(k):
            e = eidx[i, s] - 1
            if e < 0:
                continue
            def prod(q, sc, w):
                S = (w[0][e].astype(np.int64) @ q.astype(np.int64)).astype(np.float32)
                return S * np.float32(sc) * w[1][e]
            G, V = prod(nq[i], ns[i], W[0]), prod(nq[i], ns[i], W[1])
            h = (G / (np.float32(1) + np.exp(-G)) * V).astype(np.float32)
            hq, hs = i8.quantize(h[None])
            x32[i] += np.float32(gate[i, s]) * prod(hq[0], hs[0], W[2])
    assert (np.abs(x32 - out) <= berr).all()
    assert berr.max() < 0.05 * np.abs(y).max()


def test_null_tokens_pass_through():
    d, f, E = 64, 64, 2
    xt = tokens(8, "xt", 3, d, "bf16")
    eidx, gate = routing(8, 3, E, 2, "null")
    out, _ = i8.moe(xt, np.ones(d, np.float32), *experts(8, d, f, E), eidx, gate, "bf16")
    np.testing.assert_array_equal(out, xt)
