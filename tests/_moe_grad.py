"""Inputs of the expert backward tests, shared by the CPU and GPU ones."""
import numpy as np
import torch

import gen
import oracle


def moe_case(seed, act, N, d, f, E, k, choice="random"):
    """Weights, tokens, routing and an upstream gradient, rounded to ``act``.
    choice: random top-k sets; null (every slot the null expert where k is 1);
    or a list of row counts, one expert after another (k 1)."""
    L = dict(cfg=dict(E=E, act=act, k=k, d=d, d_ff=f), g2=gen.to_act(1.0 + gen.normal(seed, "g2", (d,), 0.1), act),
             Wg=gen.to_act(gen.normal(seed, "Wg", (E, f, d), d ** -0.5), act),
             Wu=gen.to_act(gen.normal(seed, "Wu", (E, f, d), d ** -0.5), act),
             Wd=gen.to_act(gen.normal(seed, "Wd", (E, d, f), f ** -0.5), act))
    xt = gen.to_act(gen.normal(seed, "xt", (N, d)), act)
    dx = gen.to_act(gen.normal(seed, "dx", (N, d)), act)
    z = gen.normal(seed, "z", (N, E + 1)).astype(np.float64)
    if choice == "random":
        eidx = np.sort(np.argsort(-z, axis=1, kind="stable")[:, :k], axis=1)
    elif choice == "null":
        eidx = np.zeros((N, k), np.int64)
    else:
        eidx = np.repeat(np.arange(len(choice)), choice).reshape(N, 1)
    p = np.exp(z)
    p = np.take_along_axis(p / p.sum(axis=1, keepdims=True), eidx, axis=1)
    egate = (p / p.sum(axis=1, keepdims=True)).astype(np.float32)
    return L, xt, dx, eidx.astype(np.int32), egate


def lists(eidx, E):
    """exp_cnt, exp_off, exp_rows of a routing (brute force)."""
    flat = eidx.reshape(-1)
    cnt = np.array([(flat == e).sum() for e in range(E + 1)], np.int32)
    off = np.concatenate([[0], np.cumsum(cnt[1:])]).astype(np.int32)
    rows = np.concatenate([np.nonzero(flat == e)[0] for e in range(1, E + 1)]).astype(np.int32)
    return cnt, off, rows


def forward(xt, L, eidx, egate, act="f64"):
    return oracle.moe(xt, L, eidx, egate, act)[0]


def reference(t, skip_rows=None, skip_tokens=None):
    """The gradients from fp64 products on the device of ``t`` (xt, dx, g2, Wg, Wu, Wd, eidx,
    egate; n rounded as the operator does).  skip_rows (e, from, to): rows of expert e's list
    that the weight gradients miss; skip_tokens: tokens that dg2 misses."""
    D = {n: t[n].double() for n in ("xt", "dx", "g2", "Wg", "Wu", "Wd")}
    x, eidx = D["xt"], t["eidx"]
    r = 1.0 / torch.sqrt((x * x).mean(1, keepdim=True) + oracle.layer.EPS)
    n = (x * r * D["g2"]).to(t["xt"].dtype).double()
    dn = torch.zeros_like(x)
    ref = dict(g_gate=torch.zeros(eidx.shape, dtype=torch.float64, device=x.device))
    for name, w in (("dWgate", "Wg"), ("dWup", "Wu"), ("dWdown", "Wd")):
        ref[name] = torch.zeros_like(D[w])
    for e in range(1, D["Wg"].shape[0] + 1):
        i, s = torch.nonzero(eidx == e, as_tuple=True)
        if not len(i):
            continue
        p, dx = t["egate"][i, s].double()[:, None], D["dx"][i]
        G, U, q = n[i] @ D["Wg"][e - 1].T, n[i] @ D["Wu"][e - 1].T, dx @ D["Wd"][e - 1]
        sg = torch.sigmoid(G)
        dG, dU, h = p * q * U * sg * (1 + G * (1 - sg)), p * q * G * sg, G * sg * U
        ref["g_gate"][i, s] = (q * h).sum(1)
        on = torch.ones(len(i), 1, dtype=torch.float64, device=x.device)
        if skip_rows and skip_rows[0] == e:
            on[skip_rows[1]:skip_rows[2]] = 0
        ref["dWgate"][e - 1], ref["dWup"][e - 1] = (on * dG).T @ n[i], (on * dU).T @ n[i]
        ref["dWdown"][e - 1] = dx.T @ (on * p * h)
        dn.index_add_(0, i, dG @ D["Wg"][e - 1] + dU @ D["Wu"][e - 1])
    gx = dn * D["g2"]
    ref["dxt"] = D["dx"] + r * gx - r ** 3 * x * (gx * x).mean(1, keepdim=True)
    on = torch.ones(len(x), 1, dtype=torch.float64, device=x.device)
    if skip_tokens is not None:
        on[skip_tokens] = 0
    ref["dg2"] = (on * dn * x * r).sum(0)
    return ref


def whole_tensor_ratios(got, ref, eidx, act):
    """||got - ref|| / ||ref|| of every output, the weight gradients expert by expert, over its
    tolerance.  A rounding to bf16 is off by 2^-8 / sqrt(3) of the value in the mean square at
    most; operands and results have one each, which add in squares.  A sum of K fp32
    products is off by about sqrt(K / 6) 2^-24 of its size in the mean square: eight sqrt(terms)
    2^-24, with all terms that lead to an output, covers the sums on the way and the few
    steps between them.
    Tensors of few rows are left out: the elements' bounds are close to their errors, and
    their roundings too few to speak of a mean.  A step of 64 rows missing among R is off by
    8 / sqrt(R)."""
    d, f = ref["dWdown"].shape[1:]
    N = eidx.shape[0]
    out = {}

    def add(name, key, a, b, terms):
        tol = 8 * terms ** 0.5 * 2.0 ** -24 if act == "f32" or name == "g_gate" else 2.0 ** -7.5 / 3 ** 0.5
        out[key] = float((a.double() - b).norm() / b.norm()) / tol

    for e in range(1, ref["dWgate"].shape[0] + 1):
        rows = int((eidx == e).sum())
        if rows >= 64:
            for name in ("dWgate", "dWup", "dWdown"):
                add(name, (name, e), got[name][e - 1], ref[name][e - 1], 2 * d + rows)
    if N >= 256 and bool((eidx != 0).any()):
        add("dxt", "dxt", got["dxt"], ref["dxt"], 3 * d + 2 * f)
        add("dg2", "dg2", got["dg2"], ref["dg2"], 2 * d + 2 * f + N)
        add("g_gate", "g_gate", got["g_gate"], ref["g_gate"], 2 * d + f)
    return out
