"""Inputs of the expert backward tests, shared by the CPU and GPU ones."""
import numpy as np

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
