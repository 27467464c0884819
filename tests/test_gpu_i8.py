"""The 8-bit operators against the oracle: each element within a bound that follows from the roundings."""
import numpy as np
import pytest
import torch

import gen
import paper_2607_06601_amd as tr
from oracle import i8
from paper_2607_06601_amd.device import to_dev

from _common import note, npy, torch_act
from _i8 import awkward_rows, experts, padded, routing, tokens, weight
from _moe_grad import lists

pytestmark = pytest.mark.gpu
DEV = "cuda"


def within(got, want, err, name=""):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    assert got.shape == want.shape
    d = np.abs(got - want)
    note(name, float((d / err).max()))
    bad = ~(d <= err)
    assert not bad.any(), (name, int(bad.sum()), d[bad][:4], err[bad][:4], np.argwhere(bad)[:4])


def matrix(q, s):
    cols = q.shape[-1]
    q = q.reshape(-1, cols)
    return tr.I8Matrix(to_dev(padded(q), torch.int8), to_dev(s.reshape(-1), torch.float32), cols)


def dirty(n):
    """A workspace that holds NaNs."""
    return torch.full((max(n, 256),), 0xFF, dtype=torch.uint8, device=DEV)


# ------------------------------------------------------------------ codes
def check_codes(x, xt):
    rows, cols = x.shape
    guard = torch.full((rows + 2, tr.i8_pitch(cols)), 77, dtype=torch.int8, device=DEV)
    scale = torch.full((rows + 2,), -5.0, device=DEV)
    tr.i8_quantize(xt, guard[1:-1], scale[1:-1])
    q, s = i8.quantize(x)
    got, gs = guard.cpu().numpy(), scale.cpu().numpy()
    np.testing.assert_array_equal(got[1:-1], padded(q))
    np.testing.assert_array_equal(gs[1:-1], s)
    assert (got[0] == 77).all() and (got[-1] == 77).all() and gs[0] == gs[-1] == -5


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("cols", [1, 2, 7, 8, 100, 127, 128, 129, 768, 1000, 2048, 2049, 2056, 5632, 9001])
def test_codes(cols, act):
    x = tokens(11, "x", 13, cols, act)
    x[3] = 0
    check_codes(x, to_dev(x, torch_act(act)))


@pytest.mark.parametrize("act", ["bf16", "f32"])
def test_codes_of_awkward_rows(act):
    x = awkward_rows(act)
    check_codes(x, to_dev(x, torch_act(act)))
    wide = np.tile(x, (1, 20))                       # four waves a row
    check_codes(wide, to_dev(wide, torch_act(act)))


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("cols,ld,off", [(768, 800, 0), (768, 801, 0), (768, 800, 3), (333, 999, 1),
                                         (2304, 2305, 1), (1, 9, 4)])
def test_codes_of_strided_rows(cols, ld, off, act):
    x = tokens(12, "x", 9, ld, act)
    check_codes(x[:, off:off + cols], to_dev(x, torch_act(act))[:, off:off + cols])


def test_codes_of_many_rows_and_one():
    x = tokens(13, "x", 20000, 40, "bf16")
    check_codes(x, to_dev(x, torch.bfloat16))
    x = tokens(14, "x", 1, 131072, "f32")
    check_codes(x, to_dev(x, torch.float32))


@pytest.mark.parametrize("cols", [8, 520, 1032, 1544, 2048])
def test_codes_of_long_batches(cols):
    """Rows enough for several a wave; an awkward row among them."""
    x = tokens(16, "x", 12321, cols, "bf16")
    x[100] = 0
    x[12320] *= np.float32(2.0 ** -120)
    x[6000, 3] = np.nan
    check_codes(x, to_dev(x, torch.bfloat16))
    if cols > 8:
        check_codes(x[:, :cols - 8], to_dev(x, torch.bfloat16)[:, :cols - 8])


def test_matrix_of_a_weight():
    x = gen.normal(15, "w", (3, 5, 300))
    m = tr.I8Matrix.quantize(to_dev(x, torch.float32))
    q, s = i8.quantize(x.reshape(15, 300))
    np.testing.assert_array_equal(npy(m.codes), padded(q))
    np.testing.assert_array_equal(npy(m.dequantize()), q.astype(np.float32) * s[:, None])


# ------------------------------------------------------------------ linear
def run_linear(x, W, act, residual=None, guard=3):
    """y in the middle columns of a wider buffer, whose other columns have to stay."""
    N, k = x.shape
    m = W.rows
    buf = torch.full((N + 1, m + 2 * guard), 7.0, dtype=torch_act(act), device=DEV)
    y = buf[:N, guard:guard + m]
    n = tr.linear_i8_workspace(N, k).numel()
    ws = dirty(n + 256)
    tr.linear_i8(x, W, y, ws[:n], residual=residual)
    torch.cuda.synchronize()
    assert (ws[n:] == 0xFF).all()
    out = npy(buf)
    assert (out[N] == 7).all() and (out[:, :guard] == 7).all() and (out[:, guard + m:] == 7).all()
    return out[:N, guard:guard + m]


LINEAR = [(1, 1, 1), (1, 768, 768), (2, 3, 5), (31, 64, 63), (32, 128, 64), (33, 129, 65),
          (64, 1000, 300), (65, 256, 1024), (127, 512, 129), (128, 128, 128), (130, 1001, 517),
          (100, 640, 300), (40, 1150, 70), (70, 1200, 64), (50, 300, 130), (60, 8000, 200),
          (200, 2048, 2048), (257, 384, 256), (300, 96, 1537), (1000, 5632, 128), (513, 640, 1280)]


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("N,k,m", LINEAR)
def test_linear(N, k, m, act):
    x, (w, t) = tokens(21, "x", N, k, act), weight(21, "W", m, k)
    r = gen.to_act(gen.normal(21, "r", (N, m)), act)
    W, xt, rt = matrix(w, t), to_dev(x, torch_act(act)), to_dev(r, torch_act(act))
    rows = np.unique(np.concatenate([[0, N - 1], np.arange(0, N, max(1, N // 48))]))
    plain, err = i8.linear(x[rows], w, t, act)
    full, rerr = i8.linear(x[rows], w, t, act, r[rows])
    within(run_linear(xt, W, act)[rows], plain, err, "y")
    aligned = run_linear(xt, W, act, guard=16)
    within(aligned[rows], plain, err, "y aligned")
    within(run_linear(xt, W, act, residual=rt)[rows], full, rerr, "y + residual")
    both = run_linear(xt, W, act, residual=rt, guard=16)
    within(both[rows], full, rerr, "y + residual aligned")
    # a token's result does not depend on the others: the first rows alone
    few = min(N, 5)
    np.testing.assert_array_equal(run_linear(xt[:few], W, act), aligned[:few])


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("N,k,m", [(2100, 512, 768), (2100, 520, 770), (4097, 256, 2048), (3000, 130, 517),
                                   (8200, 768, 1024)])
def test_linear_of_many_tokens(N, k, m, act):
    """The large tiles: whole results against integer products on the device."""
    x, (w, t) = tokens(22, "x", N, k, act), weight(22, "W", m, k)
    r = to_dev(gen.to_act(gen.normal(22, "r", (N, m)), act), torch_act(act))
    W, xt = matrix(w, t), to_dev(x, torch_act(act))
    q, s = (to_dev(a, torch.float64) for a in i8.quantize(x))
    y = (q @ to_dev(w, torch.float64).T) * s[:, None] * to_dev(t, torch.float64)
    u = i8.HALF_STEP[act]
    for res in (None, r):
        for guard in (3, 16):
            got = torch.from_numpy(run_linear(xt, W, act, residual=res, guard=guard)).to(DEV).double()
            want = y if res is None else y + res.double()
            err = 3.01 * i8.U * y.abs() + (1.01 * i8.U + 1.01 * u) * want.abs() + 1e-38
            assert ((got - want).abs() <= err).all()
            # the small tiles give the same bits
            for lo in range(0, N, 499):
                part = run_linear(xt[lo:lo + 40], W, act, residual=None if res is None else res[lo:lo + 40])
                assert (torch.from_numpy(part).to(DEV).double() == got[lo:lo + 40]).all()


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("N,k,m", [(3, 129, 9001), (8, 256, 16392), (15, 2048, 2101), (16, 2112, 8200)])
def test_linear_of_few_tokens_and_many_columns(N, k, m, act):
    x, (w, t) = tokens(25, "x", N, k, act), weight(25, "W", m, k)
    r = gen.to_act(gen.normal(25, "r", (N, m)), act)
    W, xt, rt = matrix(w, t), to_dev(x, torch_act(act)), to_dev(r, torch_act(act))
    for guard in (3, 16):
        within(run_linear(xt, W, act, guard=guard), *i8.linear(x, w, t, act), "y")
        within(run_linear(xt, W, act, residual=rt, guard=guard), *i8.linear(x, w, t, act, r), "y + residual")


def test_linear_of_codes_past_32_bits():
    """2^24 rows of 256 codes: more than 4 GB of them.  Rows here and there, and at each end."""
    N, k, m = 1 << 24, 256, 8
    x0 = to_dev(tokens(26, "x", 4099, k, "bf16"), torch.bfloat16)
    W = matrix(*weight(26, "W", m, k))
    x = torch.empty(N, k, dtype=torch.bfloat16, device=DEV)
    for lo in range(0, N, 4099):
        x[lo:lo + 4099] = x0[:N - lo]
    y = torch.full((N, m), float("nan"), dtype=torch.bfloat16, device=DEV)
    tr.linear_i8(x, W, y, tr.linear_i8_workspace(N, k))
    y0 = torch.empty(4099, m, dtype=torch.bfloat16, device=DEV)
    tr.linear_i8(x0, W, y0, tr.linear_i8_workspace(4099, k))
    at = torch.arange(N, device=DEV) % 4099
    assert torch.equal(y, y0[at])


def test_linear_in_place_and_strided():
    N, k, m = 70, 300, 256
    x, (w, t) = tokens(23, "x", N, k + 9, "bf16"), weight(23, "W", m, k)
    r = gen.to_act(gen.normal(23, "r", (N, m)), "bf16")
    W = matrix(w, t)
    y = to_dev(r, torch.bfloat16)
    tr.linear_i8(to_dev(x, torch.bfloat16)[:, 5:5 + k], W, y, tr.linear_i8_workspace(N, k), residual=y)
    within(npy(y), *i8.linear(x[:, 5:5 + k], w, t, "bf16", r), "in place")


@pytest.mark.parametrize("N", [40, 3000])
def test_linear_keeps_bad_tokens_apart(N):
    k, m = 256, 512
    x, (w, t) = tokens(24, "x", N, k, "bf16"), weight(24, "W", m, k)
    want, err = i8.linear(x, w, t, "bf16")
    x[3, 7], x[N - 2, 0], x[N // 2] = np.nan, -np.inf, 0
    got = run_linear(to_dev(x, torch.bfloat16), matrix(w, t), "bf16")
    assert np.isnan(got[[3, N - 2]]).all() and (got[N // 2] == 0).all()
    keep = np.setdiff1d(np.arange(N), [3, N - 2, N // 2])
    within(got[keep], want[keep], err[keep], "others")


def test_linear_sums_are_exact_at_the_longest_rows():
    """Codes of +-127 all along 2^17 channels: sums next to 2^31 and of both signs."""
    k, m = 131072, 6
    x = np.ones((3, k), np.float32)
    x[1] = -1
    x[2, 1::2] = -1
    w = np.full((m, k), 127, np.int8)
    w[1], w[2, 1::2], w[3, ::2], w[4, :] = -127, -127, 0, np.where(np.arange(k) % 4 < 2, 1, -127)
    w[5, k // 2:] = -126
    t = np.full(m, 2.0 ** -20, np.float32)
    y, err = i8.linear(x, w, t, "f32")
    got = run_linear(to_dev(x, torch.float32), matrix(w, t), "f32")
    within(got, y, err + 1e-12, "y")
    assert np.abs(y).max() > 127 * 127 * 131072 * (1 / 127) * 2.0 ** -20 * 0.99


# ------------------------------------------------------------------ QKV
@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("d,H,Hkv,dh,B,T,far", [
    (64, 1, 1, 64, 1, 1, 0), (64, 1, 1, 128, 1, 1, 7), (768, 12, 3, 64, 3, 5, 100000),
    (1024, 16, 4, 64, 64, 1, 8192), (192, 5, 1, 64, 2, 33, 50), (320, 3, 3, 128, 1, 130, 1 << 20),
    (576, 8, 2, 64, 40, 1, 9), (1152, 2, 1, 128, 50, 1, 9), (1088, 2, 2, 64, 33, 1, 9),
    (2048, 16, 4, 128, 2, 100, 4096), (256, 6, 2, 64, 1, 700, 0), (512, 2, 1, 128, 3, 300, 3)])
def test_qkv(d, H, Hkv, dh, B, T, far, act):
    cfg = tr.make_cfg(d, H, Hkv, dh, 32, 4, 1, 64, 32, act)
    N, dt = B * T, torch_act(act)
    n1 = tokens(31, "n1", N, d, act)
    W = [weight(31, n, r * dh, d) for n, r in (("Wq", H), ("Wk", Hkv), ("Wv", Hkv))]
    pos0 = gen.stream(31, "pos").integers(0, far + 1, B).astype(np.int32)
    mats = [matrix(*w) for w in W]
    dw = tr.DenseI8W(*(m.w for m in mats))

    def call(tok, b, t, p):
        out = [torch.full((b * t + 1, r * dh), 7.0, dtype=dt, device=DEV) for r in (H, Hkv, Hkv)]
        ws = dirty(tr.workspace_bytes(cfg, tr.OP_QKV_I8, b, t))
        tr.qkv_i8(cfg, b, t, tok, dw, *out, ws, pos0=p)
        torch.cuda.synchronize()
        assert all((o[-1] == 7).all() for o in out)
        return [npy(o[:-1]) for o in out]

    tok = to_dev(n1, dt)
    got = call(tok, B, T, to_dev(pos0, torch.int32) if far else None)
    pos = ((pos0 if far else 0 * pos0)[:, None] + np.arange(T)).reshape(-1)
    rows = np.unique(np.concatenate([[0, N - 1], np.arange(0, N, max(1, N // 32))]))
    for name, g, (want, err) in zip("qkv", got, i8.qkv(n1[rows], *W, pos[rows], dh, act)):
        within(g[rows], want, err, name)
    # a token's keys and values do not depend on the other tokens
    alone = call(tok[N - 1:], 1, 1, to_dev(pos[-1:].astype(np.int32), torch.int32))
    for a, g in zip(alone, got):
        np.testing.assert_array_equal(a[0], g[-1])


@pytest.mark.parametrize("d,H,Hkv,dh", [(768, 12, 3, 64), (2048, 16, 4, 128), (256, 6, 1, 128), (320, 4, 2, 64)])
def test_qkv_of_many_tokens(d, H, Hkv, dh):
    B, T = 2, 2200
    cfg = tr.make_cfg(d, H, Hkv, dh, 32, 4, 1, 64, 32, "bf16")
    n1 = tokens(32, "n1", B * T, d, "bf16")
    W = [weight(32, n, r * dh, d) for n, r in (("Wq", H), ("Wk", Hkv), ("Wv", Hkv))]
    mats = [matrix(*w) for w in W]
    out = [torch.full((B * T, r * dh), float("nan"), dtype=torch.bfloat16, device=DEV)
           for r in (H, Hkv, Hkv)]
    tok = to_dev(n1, torch.bfloat16)
    tr.qkv_i8(cfg, B, T, tok, tr.DenseI8W(*(m.w for m in mats)), *out,
              dirty(tr.workspace_bytes(cfg, tr.OP_QKV_I8, B, T)))
    rows = np.unique(np.concatenate([np.arange(0, B * T, 61), [T - 1, T, B * T - 1]]))
    for name, g, (want, err) in zip("qkv", out, i8.qkv(n1[rows], *W, rows % T, dh, "bf16")):
        within(npy(g)[rows], want, err, name)
    # every row: the small tiles give the same bits
    for lo in range(0, B * T, 440):
        part = [torch.empty(40, r * dh, dtype=torch.bfloat16, device=DEV) for r in (H, Hkv, Hkv)]
        at = (torch.arange(lo, lo + 40, device=DEV) % T).to(torch.int32)
        tr.qkv_i8(cfg, 40, 1, tok[lo:lo + 40].contiguous(), tr.DenseI8W(*(m.w for m in mats)), *part,
                  tr.workspace(cfg, tr.OP_QKV_I8, 40, 1), pos0=at)
        for a, b in zip(part, out):
            assert torch.equal(a, b[lo:lo + 40])


def far_apart(mats):
    """Copies of matrices more than 4 GB from each other, and the memory that holds them."""
    step = 4352 << 20
    mem = torch.empty(step * (len(mats) - 1) + mats[-1].codes.numel(), dtype=torch.int8, device=DEV)
    out = []
    for i, m in enumerate(mats):
        codes = mem[i * step:i * step + m.codes.numel()].view(m.codes.shape)
        codes.copy_(m.codes)
        out.append(tr.I8Matrix(codes, m.scale, m.cols))
    return out, mem


@pytest.mark.parametrize("N", [7, 300, 4400])
@pytest.mark.parametrize("d,H,Hkv,dh", [(768, 12, 3, 64), (512, 8, 2, 128)])
def test_qkv_of_matrices_far_apart(d, H, Hkv, dh, N):
    cfg = tr.make_cfg(d, H, Hkv, dh, 32, 4, 1, 64, 32, "bf16")
    tok = to_dev(tokens(33, "n1", N, d, "bf16"), torch.bfloat16)
    mats = [matrix(*weight(33, n, r * dh, d)) for n, r in (("Wq", H), ("Wk", Hkv), ("Wv", Hkv))]
    far, mem = far_apart(mats)
    res = []
    for ms in (mats, far):
        out = [torch.full((N, r * dh), 7.0, dtype=torch.bfloat16, device=DEV) for r in (H, Hkv, Hkv)]
        tr.qkv_i8(cfg, 1, N, tok, tr.DenseI8W(*(m.w for m in ms)), *out,
                  dirty(tr.workspace_bytes(cfg, tr.OP_QKV_I8, 1, N)))
        res.append(out)
    for a, b in zip(*res):
        assert torch.equal(a, b)


def test_qkv_of_very_many_long_tokens():
    """More blocks of rows than one launch has: each block takes several."""
    N, d, many = (1 << 20) + 5, 2112, 4099
    cfg = tr.make_cfg(d, 1, 1, 64, 32, 4, 1, 64, 32, "bf16")
    tok0 = to_dev(tokens(34, "n1", many, d, "bf16"), torch.bfloat16)
    tok = torch.empty(N, d, dtype=torch.bfloat16, device=DEV)
    for lo in range(0, N, many):
        tok[lo:lo + many] = tok0[:N - lo]
    mats = [matrix(*weight(34, n, 64, d)) for n in ("Wq", "Wk", "Wv")]
    res = []
    for t in (tok, tok0):
        out = [torch.full((len(t), 64), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(3)]
        tr.qkv_i8(cfg, len(t), 1, t, tr.DenseI8W(*(m.w for m in mats)), *out,
                  tr.workspace(cfg, tr.OP_QKV_I8, len(t), 1))
        res.append(out)
    at = torch.arange(N, device=DEV) % many
    for a, b in zip(*res):
        assert torch.equal(a, b[at])


# ------------------------------------------------------------------ experts
def device_lists(eidx, E):
    """exp_cnt, exp_off, exp_rows (of at least one entry: an empty tensor has no address)."""
    cnt, off, rows = lists(eidx, E)
    return [to_dev(a, torch.int32) for a in (cnt, off, np.append(rows, 0))]


class Experts:
    def __init__(self, seed, act, N, d, f, E, k, choice="random"):
        self.act, self.N, self.d, self.E, self.k = act, N, d, E, k
        self.W = experts(seed, d, f, E)
        self.xt = tokens(seed, "xt", N, d, act)
        self.g2 = gen.to_act(1 + gen.normal(seed, "g2", (d,), 0.1), act)
        self.eidx, self.gate = routing(seed, N, E, k, choice)
        self.cfg = tr.make_cfg(d, 1, 1, 64, 32, E, k, f, 32, act)
        self.mats = [matrix(*w) for w in self.W]
        self.t = [to_dev(self.g2, torch_act(act)), to_dev(self.eidx, torch.int32),
                  to_dev(self.gate, torch.float32)] + device_lists(self.eidx, E)
        self.x = to_dev(self.xt, torch_act(act))
        self.dw = tr.DenseI8W(g2=self.t[0].data_ptr())
        self.mw = tr.MoeI8W(*(m.w for m in self.mats))
        self.cmp = tr.Compaction(exp_cnt=self.t[3].data_ptr(), exp_off=self.t[4].data_ptr(),
                                 exp_rows=self.t[5].data_ptr())
        self.ws = dirty(tr.workspace_bytes(self.cfg, tr.OP_MOE_I8, N, 1))

    def run(self, x=None, out=None, stream=None):
        x = self.x if x is None else x
        out = torch.full_like(x, float("nan")) if out is None else out
        tr.moe_i8(self.cfg, self.N, x, self.dw, self.mw, self.t[1], self.t[2], self.cmp, out, self.ws,
                  stream=stream)
        return out

    def check(self, got, rows=None, name="x_out"):
        rows = np.arange(self.N) if rows is None else rows
        want, err = i8.moe(self.xt[rows], self.g2, *self.W, self.eidx[rows], self.gate[rows], self.act)
        within(npy(got)[rows], want, err, name)


MOE = [(2, 256, 320, 4, 2), (4, 128, 192, 3, 1), (1, 2112, 2304, 3, 4), (2, 768, 2048, 8, 2),
       (1, 64, 64, 1, 1), (1, 768, 512, 8, 2), (3, 128, 192, 4, 3), (32, 256, 512, 4, 1),
       (20, 576, 1152, 3, 1), (60, 960, 2112, 8, 2), (33, 192, 64, 2, 2), (100, 320, 448, 6, 4), (128, 256, 512, 4, 1), (333, 512, 704, 8, 2),
       (700, 128, 128, 2, 1), (1100, 192, 320, 5, 2), (64, 2112, 192, 3, 2), (1100, 2112, 192, 3, 2)]


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("N,d,f,E,k", MOE)
def test_experts(N, d, f, E, k, act):
    c = Experts(41, act, N, d, f, E, k)
    c.check(c.run(), np.unique(np.linspace(0, N - 1, 128).astype(int)))


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("counts", [[5, 0, 0, 40], [0, 1, 0, 31, 32, 33], [3, 0, 700, 1], [0, 257, 255, 0, 256]])
def test_experts_of_uneven_lists(counts, act):
    c = Experts(42, act, sum(counts), 256, 320, len(counts) - 1, 1, counts)
    got = c.run()
    c.check(got)
    n = counts[0]
    assert torch.equal(got[:n], c.x[:n])                 # null tokens pass through


@pytest.mark.parametrize("act", ["bf16", "f32"])
def test_experts_without_a_real_one(act):
    c = Experts(43, act, 37, 128, 64, 3, 2, "null")
    assert torch.equal(c.run(), c.x)


@pytest.mark.parametrize("N,d,f,E,k", [(6000, 256, 512, 4, 2), (9000, 512, 832, 8, 2), (5000, 128, 1408, 2, 1),
                                       (12400, 64, 64, 7, 3), (14000, 768, 256, 8, 2), (12289, 1088, 128, 3, 2),
                                       (12300, 2048, 64, 4, 1)])
def test_experts_of_many_tokens(N, d, f, E, k):
    """The large tiles; a token's result does not depend on the other tokens, so small batches
    give the same bits."""
    c = Experts(44, "bf16", N, d, f, E, k)
    got = c.run()
    rows = np.unique(np.linspace(0, N - 1, 200).astype(int))
    c.check(got, rows)
    for lo in range(0, N, 997):
        n = min(60, N - lo)
        small = Experts(44, "bf16", n, d, f, E, k)
        small.eidx, small.gate = c.eidx[lo:lo + n], c.gate[lo:lo + n]
        small.t[1:] = [to_dev(small.eidx, torch.int32), to_dev(small.gate, torch.float32)] + \
            device_lists(small.eidx, E)
        small.cmp = tr.Compaction(exp_cnt=small.t[3].data_ptr(), exp_off=small.t[4].data_ptr(),
                                  exp_rows=small.t[5].data_ptr())
        assert torch.equal(small.run(c.x[lo:lo + n].contiguous()), got[lo:lo + n])


@pytest.mark.parametrize("N", [2, 200, 3000])
def test_experts_of_matrices_far_apart(N):
    c = Experts(51, "bf16", N, 256, 512, 3, 2)
    want = c.run()
    far, mem = far_apart(c.mats)
    c.mw = tr.MoeI8W(*(m.w for m in far))
    assert torch.equal(c.run(), want)


def test_experts_of_very_many_tiles():
    """More than 64 tiles of the large kernels to each CU, and hidden rows of more than 1 GB."""
    c = Experts(52, "bf16", 34000, 256, 16448, 2, 1)
    c.check(c.run(), np.unique(np.linspace(0, 33999, 40).astype(int)))


@pytest.mark.parametrize("N", [50, 3000])
def test_experts_keep_bad_tokens_apart(N):
    c = Experts(45, "bf16", N, 128, 192, 3, 2)
    good = c.run()
    x = c.x.clone()
    x[7, 3], x[N - 1, 0], x[11] = float("nan"), float("inf"), 0
    bad = c.run(x)
    keep = torch.tensor([i for i in range(N) if i not in (7, 11, N - 1)], device=DEV)
    assert torch.equal(bad[keep], good[keep])
    assert (bad[11] == 0).all()
    for i in (7, N - 1):
        if (c.eidx[i] != 0).any():
            assert torch.isnan(bad[i]).all()


@pytest.mark.parametrize("N", [1, 40, 1500])
def test_experts_of_a_weight_that_is_not_finite(N):
    """A gate row whose scale is NaN (it held one): every token of that expert is NaN, no other."""
    c = Experts(49, "bf16", N, 128, 192, 3, 1, [0, N // 3, N // 3, N - N // 3 * 2])
    good = c.run()
    c.mats[0].scale[2 * 192 + 77] = float("nan")
    bad = c.run()
    at = torch.from_numpy(c.eidx[:, 0] == 3).to(DEV)
    assert torch.isnan(bad[at]).all() and torch.equal(bad[~at], good[~at])


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("N", [2, 30])
def test_experts_twice_the_same(N, act):
    """One expert in both slots of a token."""
    c = Experts(50, act, N, 128, 192, 3, 2)
    c.eidx[:, 1] = c.eidx[:, 0] = np.maximum(c.eidx[:, 1], 1)
    c.t[1] = to_dev(c.eidx, torch.int32)
    c.t[3:] = device_lists(c.eidx, 3)
    c.cmp = tr.Compaction(exp_cnt=c.t[3].data_ptr(), exp_off=c.t[4].data_ptr(), exp_rows=c.t[5].data_ptr())
    c.check(c.run())


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("N,d", [(1, 128), (60, 128), (2600, 128), (13000, 128), (1, 8256), (2, 4224), (60, 8256),
                                 (1100, 2112)])
def test_experts_of_the_largest_and_smallest_tokens(N, d, act):
    """Tokens whose products with the gains leave the range of fp32 on the way, or whose squares
    are far below eps: n2 itself is an ordinary number, or 1000 times the token."""
    if act == "f32" and N > 60:
        N = 333
    c = Experts(53, act, N, d, 192, 3, 2)
    g2 = gen.to_act(np.where(np.arange(d) % 2, 8.0, -1.5).astype(np.float32), act)
    c.g2, c.t[0] = g2, to_dev(g2, torch_act(act))
    c.dw = tr.DenseI8W(g2=c.t[0].data_ptr())
    for i, f in {N - 1: 2.0 ** -100, N // 2: 2.0 ** 110, 0: 2.0 ** 122}.items():
        c.xt[i] = gen.to_act(c.xt[i] * np.float32(f), act)
    assert np.isfinite(c.xt).all()
    c.x = to_dev(c.xt, torch_act(act))
    c.check(c.run(), np.unique(np.concatenate([[0, N // 2, N - 1], np.linspace(0, N - 1, 60).astype(int)])))


def test_experts_in_place():
    c = Experts(46, "bf16", 90, 128, 192, 3, 2)
    want = c.run()
    x = c.x.clone()
    c.run(x, x)
    assert torch.equal(x, want)


def test_experts_with_saturated_and_zero_gates():
    """Gates far out on both sides of silu, and weights of zero rows (scale 0)."""
    c = Experts(47, "f32", 40, 64, 128, 2, 1)
    s = c.mats[0].scale
    s[:64] *= 3000.0
    s[64:80] = 0
    c.W[0] = (c.W[0][0], npy(s).reshape(2, 128))
    c.check(c.run())


# ------------------------------------------------------------------ streams and graphs
def test_on_another_stream_and_in_graphs():
    """Each operator on a side stream, and captured once and replayed with new inputs between
    eager calls of the same buffers; two graphs share a workspace."""
    c = Experts(48, "bf16", 200, 256, 320, 4, 2)
    w, t = weight(48, "W", 256, 256)
    W, ws = matrix(w, t), tr.linear_i8_workspace(200, 256)
    x, y, z = c.x.clone(), torch.empty_like(c.x), torch.empty_like(c.x)

    def chain():
        c.run(x, y)
        tr.linear_i8(y, W, z, ws, residual=x)

    chain()
    want = (y.clone(), z.clone())
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    y.fill_(0), z.fill_(0)
    st.wait_stream(torch.cuda.current_stream())
    c.run(x, y, stream=st)
    tr.linear_i8(y, W, z, ws, residual=x, stream=st)
    torch.cuda.current_stream().wait_stream(st)
    assert torch.equal(y, want[0]) and torch.equal(z, want[1])
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            chain()
        graphs.append(g)
    for k in range(6):
        x.copy_(c.x.roll(k, 0) * (1 + 0.25 * k))
        graphs[k % 2].replay()
        torch.cuda.synchronize()
        got = (y.clone(), z.clone())
        y.fill_(float("nan")), z.fill_(float("nan"))
        chain()
        assert torch.equal(y, got[0]) and torch.equal(z, got[1])


# ------------------------------------------------------------------ the layer
def layer_i8(L):
    """A layer's device weights with the dense and experts' ones in 8 bits."""
    from paper_2607_06601_amd.device import DeviceLayer
    D = DeviceLayer(L)
    mats = {n: tr.I8Matrix.quantize(D.t[n]) for n in ("Wq", "Wk", "Wv", "Wo", "Wg", "Wu", "Wd")}
    dw = tr.DenseI8W(*(mats[n].w for n in ("Wq", "Wk", "Wv", "Wo")), g2=D.t["g2"].data_ptr())
    return D, mats, dw, tr.MoeI8W(*(mats[n].w for n in ("Wg", "Wu", "Wd")))


@pytest.mark.parametrize("name,B,T", [("tiny_f32_prefill", 1, 128), ("160m_bf16_prefill", 2, 300),
                                      ("160m_bf16_prefill", 40, 9), ("160m_bf16_prefill", 1, 5),
                                      ("160m_bf16_prefill", 3, 4)])
@pytest.mark.parametrize("paged", [False, True])
def test_layer_is_the_chain_of_its_stages(name, B, T, paged):
    """Prefill and decode steps of the composites equal the stage calls bit for bit, over contiguous
    and paged caches; decisions are those of the unquantised layer."""
    L = gen.make_layer(name, 1)
    L["cfg"] = cfg = dict(L["cfg"], B=B, T=T)
    D, mats, dw, mw = layer_i8(L)
    c, act = D.cfg, D.act
    H, Hkv, dh, d, k = (cfg[n] for n in ("H", "Hkv", "dh", "d", "k"))
    pages = (1, [64 * B] * 4) if paged else None
    one, two = (tr.KVCache(c, B, T + 8, pages=pages) for _ in range(2))
    steps = [T, 1, 1, 1]
    for step, t in enumerate(steps):
        N = B * t
        x = to_dev(gen.to_act(gen.normal(60 + step, "x", (N, d)), cfg["act"]), act)
        psi = to_dev(gen.normal(60 + step, "psi", (N, 8)), torch.float32)
        op = tr.OP_LAYER_PREFILL_I8 if t > 1 else tr.OP_LAYER_DECODE_I8
        xo = torch.full((N, d), float("nan"), dtype=act, device=DEV)
        ws = dirty(tr.workspace_bytes(c, op, B, t))
        if t > 1:
            tr.layer_prefill_i8(c, B, t, x, psi, D.rw, dw, mw, one, xo, ws)
        else:
            tr.layer_decode_i8(c, B, x, psi, D.rw, dw, mw, one, xo, ws)
        # the stages
        n1, o, xt, x2 = (torch.empty(N, n, dtype=act, device=DEV) for n in (d, H * dh, d, d))
        q, kk, v = (torch.empty(N, r * dh, dtype=act, device=DEV) for r in (H, Hkv, Hkv))
        mode = torch.empty(N, H, dtype=torch.uint8, device=DEV)
        bit = torch.empty(N, dtype=torch.uint8, device=DEV)
        eidx = torch.empty(N, k, dtype=torch.int32, device=DEV)
        gate = torch.empty(N, k, device=DEV)
        cmp = tr.CompactionBuffers(c, B, t)
        tr.router(c, B, t, x, psi, D.rw, n1, mode, bit, eidx, gate, cmp.struct,
                  tr.workspace(c, tr.OP_ROUTER, B, t))
        tr.qkv_i8(c, B, t, n1, dw, q, kk, v, tr.workspace(c, tr.OP_QKV_I8, B, t),
                  pos0=two.seq_len().clone())
        tr.kv_append(c, two, B, t, kk, v, bit, tr.workspace(c, tr.OP_KV_APPEND, B, t))
        if t > 1:
            tr.attn_prefill(c, B, t, q, two, mode, cmp.struct, o)
        else:
            tr.attn_decode(c, B, q, two, mode, o, tr.workspace(c, tr.OP_ATTN_DECODE, B, 1))
        tr.linear_i8(o, mats["Wo"], xt, tr.linear_i8_workspace(N, H * dh), residual=x)
        tr.moe_i8(c, N, xt, dw, mw, eidx, gate, cmp.struct, x2, tr.workspace(c, tr.OP_MOE_I8, N, 1))
        torch.cuda.synchronize()
        assert one.status() == two.status() == 0
        # (a prefill layer may split its key ranges, which moves last bits of o)
        if t == 1 or cfg["act"] == "f32":
            assert torch.equal(xo, x2), step
        else:
            a, b = xo.double(), x2.double()
            assert float((a - b).norm() / b.norm()) < 0.02
        assert torch.equal(one.seq_len(), two.seq_len()) and torch.equal(one.pool_len(), two.pool_len())
