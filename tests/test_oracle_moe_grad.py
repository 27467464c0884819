"""Pins of the oracle's expert backward pass: central differences of the scalar
it differentiates, and torch's autograd of the same block in fp64."""
import numpy as np
import pytest
import torch

import oracle
from oracle.moe_grad import moe_backward

from _moe_grad import forward, moe_case


def scalar(L, xt, dx, eidx, egate):
    return float((np.asarray(dx, np.float64) * forward(xt, L, eidx, egate)).sum())


@pytest.mark.parametrize("k,choice", [(1, "random"), (2, "random"), (4, "random"), (1, "null")])
def test_central_differences(k, choice):
    L, xt, dx, eidx, egate = moe_case(3, "f64", 5, 64, 64, 3, k, choice)
    L = {n: v if n == "cfg" else np.asarray(v, np.float64) for n, v in L.items()}
    xt, egate = np.asarray(xt, np.float64), egate.astype(np.float64)
    g = moe_backward(xt, L, eidx, egate, dx, "f64")
    rng = np.random.default_rng(0)
    h = 1e-5
    for name, t in (("dxt", xt), ("dg2", L["g2"]), ("dWgate", L["Wg"]), ("dWup", L["Wu"]),
                    ("dWdown", L["Wd"]), ("g_gate", egate)):
        for _ in range(3):
            v = rng.standard_normal(t.shape)
            if name == "g_gate":
                v = v * (eidx != 0)
            t += h * v
            hi = scalar(L, xt, dx, eidx, egate)
            t -= 2 * h * v
            lo = scalar(L, xt, dx, eidx, egate)
            t += h * v
            want = float((g[name] * v).sum())
            # differences of step h: h^2 of curvature and 2^-52 / h of rounding
            assert abs((hi - lo) / (2 * h) - want) <= 1e-7 * (1 + abs(want)), name


def test_matches_autograd():
    L, xt, dx, eidx, egate = moe_case(4, "f64", 9, 64, 128, 4, 2)
    t = {n: torch.tensor(np.asarray(v, np.float64), requires_grad=True) for n, v in L.items()
         if n != "cfg"}
    x = torch.tensor(np.asarray(xt, np.float64), requires_grad=True)
    p = torch.tensor(egate.astype(np.float64), requires_grad=True)
    n = x * torch.rsqrt((x * x).mean(1, keepdim=True) + oracle.layer.EPS) * t["g2"]
    y = x
    for i in range(9):
        for s in range(2):
            e = int(eidx[i, s])
            if e:
                h = torch.nn.functional.silu(t["Wg"][e - 1] @ n[i]) * (t["Wu"][e - 1] @ n[i])
                row = torch.zeros(9, 64, dtype=torch.float64)
                row[i] = 1.0
                y = y + row * (p[i, s] * (t["Wd"][e - 1] @ h))
    (y * torch.tensor(np.asarray(dx, np.float64))).sum().backward()
    g = moe_backward(xt, L, eidx, egate, dx, "f64")
    for name, leaf in (("dxt", x), ("g_gate", p), ("dg2", t["g2"]), ("dWgate", t["Wg"]),
                       ("dWup", t["Wu"]), ("dWdown", t["Wd"])):
        want = np.zeros(leaf.shape) if leaf.grad is None else leaf.grad.numpy()
        np.testing.assert_allclose(g[name], want, rtol=1e-10, atol=1e-12, err_msg=name)


def test_bounds_cover_a_rounded_run():
    """An emulation that rounds where the bounds say (fp32 products, bf16
    operands) stays inside them, and they are not loose by orders."""
    L, xt, dx, eidx, egate = moe_case(5, "bf16", 33, 64, 192, 3, 2)
    g, err = moe_backward(xt, L, eidx, egate, dx, "bf16", bounds=True)

    def bf(a):
        return torch.tensor(a).float().bfloat16().double().numpy()
    n = bf(oracle.rmsnorm(xt, L["g2"]))
    dW = np.zeros_like(g["dWgate"])
    for e in range(1, 4):
        i, s = np.nonzero(eidx == e)
        Wg, Wu, Wd = (np.asarray(L[w][e - 1], np.float32) for w in ("Wg", "Wu", "Wd"))
        n32 = n[i].astype(np.float32)
        G, U, q = n32 @ Wg.T, n32 @ Wu.T, dx[i].astype(np.float32) @ Wd
        sg = 1 / (1 + np.exp(-G))
        dG = bf(egate[i, s][:, None] * q * U * sg * (1 + G * (1 - sg))).astype(np.float32)
        dW[e - 1] = bf(dG.T @ n32)
    ratio = np.abs(dW - g["dWgate"]) / err["dWgate"]
    assert 0.05 < ratio.max() <= 1.0
