"""A training step of the routed experts as it runs: the relaxed controller's
forward, the experts, their backward pass, whose gate gradients go into the
controller's backward pass, and one clipping over all gradients."""
import math

import numpy as np
import pytest
import torch

import gen
import oracle
import paper_2607_06601_amd as tr
from oracle import relax, relax_grad
from oracle.moe_grad import moe_backward
from oracle.ties import enforce_relaxed_margins
from paper_2607_06601_amd.device import DeviceLayer, to_dev

from _common import assert_close, layer, npy
from test_gpu_relax import GRAD_KEYS, run_relaxed, run_relaxed_backward

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("k", [1, 2])
def test_step_of_the_small_fp32_layer(k):
    L = layer("tiny_f32_prefill")
    L["cfg"] = cfg = dict(L["cfg"], k=k)
    R = gen.relax_inputs(L, white=True)
    enforce_relaxed_margins(L, R)
    fwd = run_relaxed(L, R)
    D = DeviceLayer(L)
    c, N, d, E, act = D.cfg, cfg["B"] * cfg["T"], cfg["d"], cfg["E"], cfg["act"]
    cmp = fwd["cmp"].struct
    eidx, egate = to_dev(fwd["eidx"], torch.int32), to_dev(fwd["egate"], torch.float32)
    xt = to_dev(gen.to_act(gen.normal(21, "xt", (N, d)), act), D.act)
    dx = to_dev(gen.to_act(gen.normal(22, "dx", (N, d)), act), D.act)
    # the experts, forward and backward
    xo = torch.empty_like(xt)
    tr.moe(c, N, xt, D.dw, D.mw, eidx, egate, cmp, xo, tr.workspace(c, tr.OP_MOE, N, 1))
    out = dict(dxt=torch.empty_like(xt), dWgate=torch.empty_like(D.t["Wg"]),
               dWup=torch.empty_like(D.t["Wu"]), dWdown=torch.empty_like(D.t["Wd"]),
               dg2=torch.empty_like(D.t["g2"]), g_gate=torch.empty(N, k, device=DEV))
    tr.moe_backward(c, N, xt, D.dw, D.mw, eidx, egate, cmp, dx,
                    tr.MoeGradOut(**{n: t.data_ptr() for n, t in out.items()}),
                    tr.workspace(c, tr.OP_MOE_BACKWARD, N, 1))
    ref_x = oracle.moe(npy(xt), L, fwd["eidx"], fwd["egate"].astype(np.float64), act)[0]
    assert_close(npy(xo), ref_x, act, "x_out")
    ref = moe_backward(npy(xt), L, fwd["eidx"], fwd["egate"], npy(dx), act)
    for n in out:
        assert_close(npy(out[n]), ref[n], act, n)
    # ... its gate gradients into the controller's backward pass
    A = fwd["y_attn"].shape[1]
    up = dict(g_ya=gen.normal(23, "ga", (N, A, 3)), g_yb=gen.normal(24, "gb", (N, 4)))
    rho = (1.5, 0.8, 2.5)
    got = run_relaxed_backward(L, R, fwd, dict(up, g_gate=npy(out["g_gate"])), rho, 0.0)
    f64 = relax.relaxed_forward(L, R)
    np.testing.assert_array_equal(fwd["eidx"], f64["S"])
    want = relax_grad.relaxed_backward(
        L, R, f64, dict({n: np.asarray(v, np.float64) for n, v in up.items()},
                        g_gate=ref["g_gate"]), rho=rho)
    for n in [n for n, _ in GRAD_KEYS] + ["dx", "dpsi"]:
        assert_close(got[n], want[n], "f32", n)
    # one norm over the controller's and the experts' gradients, all scaled by it
    names = [n for n, _ in GRAD_KEYS]
    grads = [to_dev(got[n], torch.float32) for n in names] + \
        [out[n] for n in ("dWgate", "dWup", "dWdown", "dg2")]
    total = math.sqrt(sum(float((npy(t).astype(np.float64) ** 2).sum()) for t in grads))
    exact = math.sqrt(sum(float((np.asarray(w, np.float64) ** 2).sum()) for w in
                          [want[n] for n in names] + [ref[n] for n in ("dWgate", "dWup", "dWdown", "dg2")]))
    before = [t.clone() for t in grads]
    norm = torch.zeros(1, dtype=torch.float64, device=DEV)
    tr.grad_clip(tr.GradList(grads), 0.25 * total, norm, tr.grad_workspace())
    torch.cuda.synchronize()
    assert abs(norm.item() - total) <= 1e-12 * total
    assert abs(norm.item() - exact) <= 2e-5 * exact
    for a, b in zip(before, grads):
        assert torch.equal(b, a * np.float32(0.25)) or \
            ((b - 0.25 * a).abs() <= 2.0 ** -23 * a.abs()).all()


@pytest.mark.parametrize("k", [1, 2])
def test_step_of_the_small_layer_in_bf16(k):
    """bf16 tokens and experts, the controller in fp32: each part against its oracle on what
    the part before it left, and one clipping over gradients of both types."""
    L = layer("tiny_f32_prefill", act="bf16")
    L["cfg"] = cfg = dict(L["cfg"], k=k)
    assert cfg["act"] == "bf16"
    R = gen.relax_inputs(L, white=True)
    enforce_relaxed_margins(L, R)
    fwd = run_relaxed(L, R)
    D = DeviceLayer(L)
    c, N, d, act = D.cfg, cfg["B"] * cfg["T"], cfg["d"], cfg["act"]
    cmp = fwd["cmp"].struct
    eidx, egate = to_dev(fwd["eidx"], torch.int32), to_dev(fwd["egate"], torch.float32)
    xt = to_dev(gen.to_act(gen.normal(21, "xt", (N, d)), act), D.act)
    dx = to_dev(gen.to_act(gen.normal(22, "dx", (N, d)), act), D.act)
    xo = torch.empty_like(xt)
    tr.moe(c, N, xt, D.dw, D.mw, eidx, egate, cmp, xo, tr.workspace(c, tr.OP_MOE, N, 1))
    out = dict(dxt=torch.empty_like(xt), dWgate=torch.empty_like(D.t["Wg"]),
               dWup=torch.empty_like(D.t["Wu"]), dWdown=torch.empty_like(D.t["Wd"]),
               dg2=torch.empty_like(D.t["g2"]), g_gate=torch.empty(N, k, device=DEV))
    tr.moe_backward(c, N, xt, D.dw, D.mw, eidx, egate, cmp, dx,
                    tr.MoeGradOut(**{n: t.data_ptr() for n, t in out.items()}),
                    tr.workspace(c, tr.OP_MOE_BACKWARD, N, 1))
    ref_x = oracle.moe(npy(xt), L, fwd["eidx"], fwd["egate"].astype(np.float64), act)[0]
    assert_close(npy(xo), ref_x, act, "x_out")
    ref, err = moe_backward(npy(xt), L, fwd["eidx"], fwd["egate"], npy(dx), act, bounds=True)
    for n in out:
        assert (np.abs(npy(out[n]).astype(np.float64) - ref[n]) <= err[n]).all(), n
    A = fwd["y_attn"].shape[1]
    up = dict(g_ya=gen.normal(23, "ga", (N, A, 3)), g_yb=gen.normal(24, "gb", (N, 4)),
              g_gate=npy(out["g_gate"]))
    rho = (1.5, 0.8, 2.5)
    got = run_relaxed_backward(L, R, fwd, up, rho, 0.0)
    f64 = relax.relaxed_forward(L, R)
    np.testing.assert_array_equal(fwd["eidx"], f64["S"])
    want = relax_grad.relaxed_backward(L, R, f64, {n: np.asarray(v, np.float64) for n, v in up.items()},
                                       rho=rho)
    names = [n for n, _ in GRAD_KEYS]
    for n in names + ["dx", "dpsi"]:
        assert_close(got[n], want[n], "f32", n)
    grads = [to_dev(got[n], torch.float32) for n in names] + \
        [out[n] for n in ("dWgate", "dWup", "dWdown", "dg2")]
    total = math.sqrt(sum(float((npy(t).astype(np.float64) ** 2).sum()) for t in grads))
    before = [npy(t).astype(np.float64) for t in grads]
    norm = torch.zeros(1, dtype=torch.float64, device=DEV)
    tr.grad_clip(tr.GradList(grads), 0.3 * total, norm, tr.grad_workspace())
    torch.cuda.synchronize()
    assert abs(norm.item() - total) <= 1e-12 * total
    for a, b in zip(before, grads):
        # the coefficient's and the product's rounding to fp32, and one to bf16
        u = (2.0 ** -8 if b.dtype == torch.bfloat16 else 0.0) + 3 * 2.0 ** -24
        assert (np.abs(npy(b) - 0.3 * a) <= u * np.abs(0.3 * a) + 1e-40).all()
