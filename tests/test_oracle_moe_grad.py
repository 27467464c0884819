"""Pins of the oracle's expert backward pass: central differences of the scalar
it differentiates, and torch's autograd of the same block in fp64."""
import numpy as np
import pytest
import torch

import oracle
from oracle.moe_grad import moe_backward

from _moe_grad import forward, moe_case, reference, whole_tensor_ratios


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


def tensors(L, xt, dx, eidx, egate, dtype):
    t = {n: torch.tensor(np.asarray(v, np.float32)).to(dtype)
         for n, v in dict(xt=xt, dx=dx, **{n: L[n] for n in ("g2", "Wg", "Wu", "Wd")}).items()}
    return dict(t, eidx=torch.tensor(eidx), egate=torch.tensor(egate))


@pytest.mark.parametrize("act,dtype", [("bf16", torch.bfloat16), ("f32", torch.float32)])
def test_torch_reference_equals_the_oracle(act, dtype):
    case = moe_case(6, act, 300, 64, 128, 4, 2)
    want = moe_backward(case[1], case[0], case[3], case[4], case[2], act)
    got = reference(tensors(*case, dtype))
    for name in want:
        np.testing.assert_allclose(got[name].numpy(), want[name], rtol=1e-9, atol=1e-11, err_msg=name)


@pytest.mark.parametrize("N,d,f", [(49200, 64, 64), (8200, 128, 320)])
def test_whole_tensors_show_lost_work(N, d, f):
    """Rounded once they pass; a step of 64 rows that the weight gradients of one expert miss, or
    a block's tokens that dg2 misses, do not (each element may stay inside its own
    bound, which grows with the rows while the sum grows with their root)."""
    case = moe_case(7, "bf16", N, d, f, 2, 2)
    t = tensors(*case, torch.bfloat16)
    ref = reference(t)

    def ratios(g):
        return whole_tensor_ratios({n: v if n == "g_gate" else v.bfloat16() for n, v in g.items()}, ref,
                                   t["eidx"], "bf16")
    right = ratios(ref)
    assert len(right) == 9 and 0 < max(right.values()) <= 1
    rows = int((t["eidx"] == 2).sum())
    for lo in (0, rows // 128 * 64):
        bad = ratios(reference(t, skip_rows=(2, lo, lo + 64)))
        assert {k for k, v in bad.items() if v > 1} == {(n, 2) for n in ("dWgate", "dWup", "dWdown")}
    block = torch.arange(N) // 4 % 512 == 77
    assert {k for k, v in ratios(reference(t, skip_tokens=block)).items() if v > 1} == {"dg2"}
