"""Timed cases of the training operators: the backward pass of the experts' gated
feed-forward block, and the global gradient norm with clipping.

  listed()            the cases, from the smallest call to a full batch
  draw(rng)           one more case of the same ranges
  prepare(case, s)    device inputs of seed s, and what a training program keeps beside them
  run(state)          one pass: the plain form, or (own) the library's calls
  work(case)          bytes and operations that one pass cannot do without
  exact(case, s)      the outputs from the definition, in 64 bits

Shapes are those of the layers in gen/ (160M to 1.3B classes) and generic ones.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
EPS = 1e-6
ACT = {"bf16": torch.bfloat16, "f32": torch.float32}
# (d, d_ff, E, top-k) of the layers in gen/
SHAPES = {"tiny": (256, 512, 4, 1), "160m": (768, 2048, 8, 2), "410m": (1024, 2816, 8, 2),
          "1p3b": (2048, 5632, 16, 2)}


# ------------------------------------------------------------------- cases
def _moe(name, shape, N, act="bf16", skew=False, frozen=False):
    d, f, E, k = SHAPES[shape]
    return dict(name=name, kind="moe", d=d, f=f, E=E, k=k, N=N, act=act, skew=skew, frozen=frozen)


def _layer(name, shape, ratio, norm=2, act="bf16", frozen=False):
    d, f, E, _ = SHAPES[shape]
    return dict(name=name, kind="clip", layout="layer", d=d, f=f, E=E, act=act, frozen=frozen,
                ratio=ratio, norm=norm)


def listed():
    return [
        # one token through the 160M layer's experts: the latency of the call
        _moe("experts 160m, 1 token", "160m", 1),
        # the small fp32 layer that gradients are checked on
        _moe("experts tiny fp32, 128 tokens", "tiny", 128, act="f32"),
        # a short odd batch, most experts with a part of a tile
        _moe("experts 410m, 333 tokens", "410m", 333),
        # an fp32 training step of the 160M layer
        _moe("experts 160m fp32, 2000 tokens", "160m", 2000, act="f32"),
        # two hot experts, as a router makes them before the balance loss bites
        _moe("experts 410m, 4000 tokens, skewed", "410m", 4000, skew=True),
        # the controller trained on frozen experts: no weight gradients
        _moe("experts 1.3B, 8192 tokens, frozen", "1p3b", 8192, frozen=True),
        # the full batches of the 160M and 1.3B layers
        _moe("experts 160m, 16384 tokens", "160m", 16384),
        _moe("experts 1.3B, 16384 tokens", "1p3b", 16384),
        # the controller's own twelve gradients: latency
        _layer("clip router 160m", "160m", 3.7, frozen=True),
        # 480 small and middling gradients in a flat bucket, odd sizes, largest value
        dict(name="clip 480 odd tensors, max norm", kind="clip", layout="bucket", tensors=480,
             most=1 << 17, split=7, ratio=2.0, norm=0),
        # all gradients of a 160M layer, below the threshold (copied as they are)
        _layer("clip layer 160m, no scaling", "160m", 0.5),
        # all gradients of a 1.3B layer
        _layer("clip layer 1.3B", "1p3b", 3.7),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    if rng.random() < 0.35:
        norm = rng.choice((2, 2, 0))
        ratio = round(math.exp(rng.uniform(math.log(0.2), math.log(50.0))), 3)
        if rng.random() < 0.5:
            return dict(kind="clip", layout="bucket", tensors=_log_int(rng, 1, 600),
                        most=_log_int(rng, 16, 1 << 20), split=rng.randrange(1 << 20),
                        ratio=ratio, norm=norm)
        return dict(kind="clip", layout="layer", d=64 * _log_int(rng, 1, 32),
                    f=64 * _log_int(rng, 1, 88), E=_log_int(rng, 1, 16),
                    act=rng.choice(("bf16", "f32")), frozen=rng.random() < 0.2, ratio=ratio,
                    norm=norm)
    f32 = rng.random() < 0.25
    top = SHAPES["160m" if f32 else "1p3b"]
    while True:
        E = _log_int(rng, 1, 24)
        c = dict(kind="moe", d=64 * _log_int(rng, 1, 16 if f32 else 32),
                 f=64 * _log_int(rng, 1, 44 if f32 else 88), E=E,
                 k=rng.randint(1, min(4, E + 1)), N=_log_int(rng, 1, 4000 if f32 else 16384),
                 act="f32" if f32 else "bf16", skew=rng.random() < 0.3,
                 frozen=rng.random() < 0.2)
        most = top[0] * top[1] * 2 * (2000 if f32 else 16384)
        if c["d"] * c["f"] * c["N"] * c["k"] <= most and E * c["d"] * c["f"] <= top[0] * top[1] * 16:
            return c


# ------------------------------------------------------------------ inputs
def _gen(seed, tag):
    g = torch.Generator(device=DEV)
    g.manual_seed((seed * 1000003 + tag) % (1 << 62))
    return g


def _normal(g, shape, std, dtype):
    return (torch.randn(shape, generator=g, device=DEV, dtype=torch.float32) * std).to(dtype)


def _shares(c):
    """Target share of each option 0..E (0 = null)."""
    E = c["E"]
    if not c["skew"] or E < 4:
        return [1.0 / (E + 1)] * (E + 1)
    return [0.15, 0.30, 0.30] + [0.25 / (E - 2)] * (E - 2)


def _moe_inputs(c, seed):
    N, d, f, E, k, act = c["N"], c["d"], c["f"], c["E"], c["k"], ACT[c["act"]]
    g = _gen(seed, 1)
    xt = _normal(g, (N, d), 1.0, act)
    dx = _normal(g, (N, d), 1.0, act)
    g2 = (1.0 + 0.1 * torch.randn(d, generator=g, device=DEV)).to(act)
    Wg = _normal(g, (E, f, d), d ** -0.5, act)
    Wu = _normal(g, (E, f, d), d ** -0.5, act)
    Wd = _normal(g, (E, d, f), f ** -0.5, act)
    # the router's choice: the k largest logits, in ascending expert id, gates
    # renormalised over them (the null's share among them)
    z = torch.randn(N, E + 1, generator=g, device=DEV)
    z = z + torch.log(torch.tensor(_shares(c), device=DEV))
    eidx = torch.topk(z, k, dim=1).indices.sort(dim=1).values
    p = torch.softmax(z, dim=1).gather(1, eidx)
    gate = (p / p.sum(dim=1, keepdim=True)).float().contiguous()
    return xt, dx, g2, Wg, Wu, Wd, eidx.to(torch.int32).contiguous(), gate


def _prepare_moe(c, seed):
    xt, dx, g2, Wg, Wu, Wd, eidx, gate = _moe_inputs(c, seed)
    N, d, f, E, k = c["N"], c["d"], c["f"], c["E"], c["k"]
    # the expert lists that the router's forward left: assignments by expert
    flat = eidx.reshape(-1).long()
    order = torch.sort(flat, stable=True).indices
    cnt = torch.bincount(flat, minlength=E + 1)
    off = torch.cumsum(cnt, 0) - cnt[0]
    nulls = int(cnt[0])
    rows = torch.cat([order[nulls:], order[:nulls]])
    st = dict(c=c, xt=xt, dx=dx, g2=g2, Wg=Wg, Wu=Wu, Wd=Wd, eidx=eidx, gate=gate,
              cnt=cnt.to(torch.int32), off=off.to(torch.int32), rows=rows.to(torch.int32),
              cap=max(1, int(cnt[1:].max())))
    if own:
        _plan_moe(st)
    return st


def _plan_moe(st):
    """The structs, gradient buffers and workspace that a training program keeps."""
    import paper_2607_06601_amd as tr
    c = st["c"]
    N, d, f, E, k, act = c["N"], c["d"], c["f"], c["E"], c["k"], ACT[c["act"]]
    cfg = tr.make_cfg(d, 4, 1, 64, 128, E, k, f, 64, c["act"], rms_eps=EPS)
    out = dict(dxt=torch.empty_like(st["xt"]), dg2=torch.empty_like(st["g2"]),
               g_gate=torch.empty(N, k, device=DEV))
    if not c["frozen"]:
        out.update(dWgate=torch.empty_like(st["Wg"]), dWup=torch.empty_like(st["Wu"]),
                   dWdown=torch.empty_like(st["Wd"]))
    st.update(tr=tr, cfg=cfg, out=out, dw=tr.DenseW(g2=st["g2"].data_ptr()),
              mw=tr.MoeW(*(st[n].data_ptr() for n in ("Wg", "Wu", "Wd"))),
              cmp=tr.Compaction(exp_cnt=st["cnt"].data_ptr(), exp_off=st["off"].data_ptr(),
                                exp_rows=st["rows"].data_ptr()),
              gout=tr.MoeGradOut(**{n: t.data_ptr() for n, t in out.items()}),
              ws=tr.workspace(cfg, tr.OP_MOE_BACKWARD, N, 1))


def _sizes(c):
    """(elements, bf16?) of each gradient."""
    if c["layout"] == "bucket":
        r = random.Random(c["split"])
        return [(_log_int(r, 1, c["most"]), r.random() < 0.5) for _ in range(c["tensors"])]
    d, f, E, R = c["d"], c["f"], c["E"], 128
    s = [(n, False) for n in (R * (d + 8), R, R * R, R, R, 36 * R, 36, (E + 1) * R, E + 1, 4 * R,
                              4, d)]  # the controller's, fp32
    if not c["frozen"]:
        s += [(n, c["act"] == "bf16") for n in (d, E * f * d, E * f * d, E * f * d)]
    return s


def _clip_inputs(c, seed):
    """Two flat buffers (fp32, bf16), and where each gradient lies: a layer's
    gradients as an allocator places them, a bucket's one behind the other."""
    step = 1 if c["layout"] == "bucket" else 128
    at, views = [0, 0], []
    for n, half in _sizes(c):
        views.append((int(half), at[half], n))
        at[half] += (n + step - 1) // step * step
    total = sum(n for _, _, n in views)
    # values of a spread of magnitudes, as gradients of different weights have;
    # their norm is about `ratio` times the threshold of 1
    scale = c["ratio"] / (math.sqrt(total) if c["norm"] == 2 else 4.0)
    g = _gen(seed, 2)
    flat = []
    for half in (0, 1):
        t = torch.randn(max(1, at[half]), generator=g, device=DEV)
        t *= scale * (0.5 + torch.rand(1, generator=g, device=DEV))
        flat.append(t.to(torch.bfloat16 if half else torch.float32))
    if step > 1:  # what lies between two gradients belongs to none
        for half, lo, n in views:
            flat[half][lo + n:lo + (n + step - 1) // step * step] = 0
    for half in (0, 1):
        if at[half] == 0:
            flat[half].zero_()
    return flat, views


def _prepare_clip(c, seed):
    flat, views = _clip_inputs(c, seed)
    st = dict(c=c, flat=flat, views=views)
    if own:
        import paper_2607_06601_amd as tr
        dst = [torch.zeros_like(t) for t in flat]
        pick = lambda bufs: [bufs[h][lo:lo + n] for h, lo, n in views]  # noqa: E731
        st.update(tr=tr, dst=dst, plan=tr.GradList(pick(flat), pick(dst)),
                  norm=torch.empty((), dtype=torch.float64, device=DEV),
                  ws=tr.grad_workspace())
    return st


def prepare(case, seed):
    return _prepare_moe(case, seed) if case["kind"] == "moe" else _prepare_clip(case, seed)


# --------------------------------------------------------------- plain forms
def _plain_moe(st):
    """Rows of every expert padded to the longest list, products batched over
    the experts, fp32 throughout; n2 is the operator's own rounding."""
    c = st["c"]
    N, d, f, E, k, act, cap = c["N"], c["d"], c["f"], c["E"], c["k"], ACT[c["act"]], st["cap"]
    pos = torch.arange(cap, device=DEV)
    live = pos[None, :] < st["cnt"][1:, None]
    a = st["rows"].long()[(st["off"][:-1, None].long() + pos[None, :]).clamp(max=N * k - 1)]
    tok, on = a // k, live[..., None]
    x64 = st["xt"].double()
    r64 = torch.rsqrt(x64.square().mean(1, keepdim=True) + EPS)
    # (a value next to the border of two bf16 numbers: the norm in 64 bits)
    n2 = (x64 * r64 * st["g2"].double()).float().to(act).float()
    x, r, g2, dx = st["xt"].float(), r64.float(), st["g2"].float(), st["dx"].float()
    X = torch.where(on, n2[tok], 0.0)
    DY = torch.where(on, dx[tok], 0.0)
    p = torch.where(live, st["gate"].reshape(-1)[a], 0.0)[..., None]
    Wg, Wu, Wd = st["Wg"].float(), st["Wu"].float(), st["Wd"].float()
    G, U = torch.bmm(X, Wg.transpose(1, 2)), torch.bmm(X, Wu.transpose(1, 2))
    Q = torch.bmm(DY, Wd)
    s = torch.sigmoid(G)
    A = G * s
    H = A * U
    gq = (Q * H).sum(-1)
    Q = Q * p
    DG = Q * U * (s * (1.0 + G * (1.0 - s)))
    DU = Q * A
    dX = torch.bmm(DG, Wg) + torch.bmm(DU, Wu)
    # back to the tokens: the padded row of each assignment, the last (zero) one for nulls
    where = torch.full((N * k,), E * cap, dtype=torch.long, device=DEV)
    spare = torch.where(live, a, N * k)
    where = torch.cat([where, where[:1]]).scatter(
        0, spare.reshape(-1), torch.arange(E * cap, device=DEV))[:N * k]
    nul = st["eidx"].reshape(-1) == 0
    where = torch.where(nul, E * cap, where)
    dXz = torch.cat([dX.reshape(E * cap, d), torch.zeros(1, d, device=DEV)])
    dn = dXz[where.reshape(N, k)].sum(1)
    g_gate = torch.cat([gq.reshape(-1), torch.zeros(1, device=DEV)])[where].reshape(N, k)
    gx = dn * g2
    dxt = dx + r * gx - r ** 3 * x * ((gx * x).sum(1, keepdim=True) / d)
    dg2 = (dn.double() * x64 * r64).sum(0)
    out = dict(dxt=dxt.to(act), dg2=dg2.float().to(act), g_gate=g_gate)
    if not c["frozen"]:
        out.update(dWgate=torch.bmm(DG.transpose(1, 2), X).to(act),
                   dWup=torch.bmm(DU.transpose(1, 2), X).to(act),
                   dWdown=torch.bmm(DY.transpose(1, 2), p * H).to(act))
    return out


def _plain_clip(st):
    c, (a, b) = st["c"], st["flat"]
    if c["norm"] == 2:
        norm = torch.sqrt(a.double().square().sum() + b.double().square().sum())
    else:
        norm = torch.maximum(a.abs().max().double(), b.abs().max().double())
    coef = torch.clamp(1.0 / norm, max=1.0).float()
    return dict(norm=norm, f32=a * coef, bf16=(b.float() * coef).to(torch.bfloat16))


# --------------------------------------------------------------- one pass
def run(st):
    c = st["c"]
    if not own:
        return _plain_moe(st) if c["kind"] == "moe" else _plain_clip(st)
    tr = st["tr"]
    if c["kind"] == "moe":
        tr.moe_backward(st["cfg"], c["N"], st["xt"], st["dw"], st["mw"], st["eidx"], st["gate"],
                        st["cmp"], st["dx"], st["gout"], st["ws"])
        return st["out"]
    tr.grad_clip(st["plan"], 1.0, st["norm"], st["ws"], norm_type=c["norm"] or math.inf)
    return dict(norm=st["norm"], f32=st["dst"][0], bf16=st["dst"][1])


def work(case):
    c = case
    if c["kind"] == "clip":
        size = sum(n * (2 if half else 4) for n, half in _sizes(c))
        return {"bytes": 2 * size, "flops": 3 * sum(n for n, _ in _sizes(c))}
    b = 2 if c["act"] == "bf16" else 4
    real = c["N"] * c["k"] * (1.0 - _shares(c)[0])
    used = min(c["E"], real)  # experts whose weights are read
    w = 3 * c["d"] * c["f"] * b
    wr = 0 if c["frozen"] else c["E"] * w
    return {"bytes": used * w + wr + 3 * c["N"] * c["d"] * b + 12 * c["N"] * c["k"],
            "flops": (10 if c["frozen"] else 16) * c["d"] * c["f"] * real}


# ------------------------------------------------------- 64-bit reference
def _exact_moe(c, seed):
    xt, dx, g2, Wg, Wu, Wd, eidx, gate = _moe_inputs(c, seed)
    N, d, E, k = c["N"], c["d"], c["E"], c["k"]
    x, up, g = xt.double(), dx.double(), g2.double()
    inv = 1.0 / torch.sqrt((x * x).sum(1) / d + EPS)
    n2 = (x * inv[:, None] * g).float().to(ACT[c["act"]]).double()
    dn = torch.zeros(N, d, dtype=torch.float64, device=DEV)
    g_gate = torch.zeros(N, k, dtype=torch.float64, device=DEV)
    dW = [torch.zeros(w.shape, dtype=torch.float64, device=DEV) for w in (Wg, Wu, Wd)]
    for e in range(1, E + 1):
        i, s = (eidx == e).nonzero(as_tuple=True)
        if i.numel() == 0:
            continue
        wg, wu, wd = Wg[e - 1].double(), Wu[e - 1].double(), Wd[e - 1].double()
        pre, lin = n2[i] @ wg.T, n2[i] @ wu.T
        sig = 1.0 / (1.0 + torch.exp(-pre))
        hid = pre * sig * lin
        dhid = up[i] @ wd
        g_gate[i, s] = (dhid * hid).sum(1)
        pr = gate[i, s].double()[:, None]
        d_pre = pr * dhid * lin * (sig + pre * sig * (1.0 - sig))
        d_lin = pr * dhid * pre * sig
        dn.index_put_((i,), d_pre @ wg + d_lin @ wu, accumulate=True)
        dW[0][e - 1] = d_pre.T @ n2[i]
        dW[1][e - 1] = d_lin.T @ n2[i]
        dW[2][e - 1] = (pr * up[i]).T @ hid
    xhat = x * inv[:, None]
    dxh = dn * g
    dxt = up + inv[:, None] * (dxh - xhat * (dxh * xhat).mean(1, keepdim=True))
    out = dict(dxt=dxt, dg2=(dn * xhat).sum(0), g_gate=g_gate)
    if not c["frozen"]:
        out.update(dWgate=dW[0], dWup=dW[1], dWdown=dW[2])
    return out


def _exact_clip(c, seed):
    flat, views = _clip_inputs(c, seed)
    parts = [flat[h][lo:lo + n].double() for h, lo, n in views]
    if c["norm"] == 2:
        norm = math.sqrt(math.fsum(float(torch.dot(t, t)) for t in parts))
    else:
        norm = max(float(t.abs().max()) for t in parts)
    coef = min(1.0, 1.0 / norm)
    return dict(norm=torch.tensor(norm, dtype=torch.float64), f32=flat[0].double() * coef,
                bf16=flat[1].double() * coef)


def exact(case, seed):
    return _exact_moe(case, seed) if case["kind"] == "moe" else _exact_clip(case, seed)
