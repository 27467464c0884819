"""The 8-bit products' values: the same in any batch, and over the whole range of fp32."""
import numpy as np
import pytest
import torch

import gen
import paper_2607_06601_amd as tr
from oracle import i8
from paper_2607_06601_amd.device import to_dev

from _common import npy, torch_act
from _i8 import tokens, weight
from test_gpu_i8 import DEV, Experts, device_lists, dirty, matrix, run_linear, within

pytestmark = pytest.mark.gpu


def part(c, at):
    """x_out of the tokens `at` of c, in a call of their own."""
    n, eidx = len(at), c.eidx[at]
    t = [to_dev(eidx, torch.int32), to_dev(c.gate[at], torch.float32)] + device_lists(eidx, c.E)
    cmp = tr.Compaction(exp_cnt=t[2].data_ptr(), exp_off=t[3].data_ptr(), exp_rows=t[4].data_ptr())
    x = c.x[torch.from_numpy(np.asarray(at)).to(DEV)].contiguous()
    out = torch.full_like(x, float("nan"))
    tr.moe_i8(c.cfg, n, x, c.dw, c.mw, t[0], t[1], cmp, out,
              dirty(tr.workspace_bytes(c.cfg, tr.OP_MOE_I8, n, 1)))
    torch.cuda.synchronize()
    return out


def gains(c, g2):
    c.g2 = gen.to_act(np.asarray(g2, np.float32), c.act)
    c.t[0] = to_dev(c.g2, torch_act(c.act))
    c.dw = tr.DenseI8W(g2=c.t[0].data_ptr())


def weight_scale(c, which, at, factor):
    """Scales of rows `at` of each expert, multiplied."""
    q, s = c.W[which]
    s[:, at] *= np.float32(factor)
    c.mats[which].scale.copy_(to_dev(s.reshape(-1), torch.float32))


def some(n, most=60):
    return np.unique(np.linspace(0, n - 1, most).astype(int))


# ------------------------------------------------------------------ batches
@pytest.mark.parametrize("act,N,d,f,E,k", [
    ("bf16", 6000, 256, 512, 4, 2), ("bf16", 6000, 768, 192, 3, 1), ("bf16", 40, 64, 12352, 6, 4),
    ("f32", 2100, 256, 512, 4, 2)])
def test_a_token_alone_and_in_batches(act, N, d, f, E, k):
    """Each batch size takes other kernels: the bits of a token are the same in all."""
    c = Experts(61, act, N, d, f, E, k)
    whole = c.run()
    for n in (1, 2, 3, 5, 33, 333, 1500):
        for lo in range(0, N - n + 1, max(n, (N - n) // 3)):
            assert torch.equal(part(c, np.arange(lo, lo + n)), whole[lo:lo + n]), (n, lo)


@pytest.mark.parametrize("N", [1, 2, 40, 333, 1500, 6000])
def test_hidden_rows_are_fp32(N):
    """Tokens far smaller than the experts' outputs, which so show nothing but their one rounding."""
    c = Experts(62, "bf16", N, 256, 512, 4, 2)
    c.xt = gen.to_act(c.xt * np.float32(2.0 ** -60), "bf16")
    c.x = to_dev(c.xt, torch.bfloat16)
    gains(c, c.g2 * 2.0 ** 50)
    c.check(c.run(), some(N))


# ------------------------------------------------------------------ range
SIZES = [("bf16", 1), ("bf16", 2), ("bf16", 40), ("bf16", 333), ("bf16", 1500), ("bf16", 6000),
         ("f32", 2), ("f32", 40), ("f32", 333)]


@pytest.mark.parametrize("act,N", SIZES)
@pytest.mark.parametrize("gain,gate,up", [(2.0 ** 72, 2.0 ** -72, 2.0 ** -72), (2.0 ** -70, 2.0 ** 70, 2.0 ** 70),
                                          (1, 2.0 ** -90, 2.0 ** 90), (2.0 ** 90, 2.0 ** -85, 2.0 ** -95)])
def test_scales_far_from_one(act, N, gain, gate, up):
    """Gates and ups that are ordinary numbers while the scales' products are not."""
    c = Experts(63, act, N, 256, 512, 4, 2)
    gains(c, c.g2 * gain)
    weight_scale(c, 0, slice(None), gate)
    weight_scale(c, 1, slice(None), up)
    got = c.run()
    assert torch.isfinite(got).all()
    c.check(got, some(N))


@pytest.mark.parametrize("act,N", SIZES)
def test_saturated_and_zero_gates(act, N):
    """Gates far out on both sides of silu and of 0, unit by unit and 32 units together."""
    c = Experts(64, act, N, 256, 512, 2, 2)
    for at, factor in ((slice(0, 64, 3), 3000.0), (slice(64, 80), 0), (slice(96, 128), 0),
                       (slice(128, 192), 1e4), (slice(192, 224), 1e-30), (slice(256, 320), 300.0)):
        weight_scale(c, 0, at, factor)
    weight_scale(c, 1, slice(300, 352), 0)
    got = c.run()
    assert torch.isfinite(got).all()
    c.check(got, some(N))
    weight_scale(c, 0, slice(None), 0)             # no gate at all
    assert torch.equal(c.run(), c.x)


# ------------------------------------------------------------------ the norm
# Tokens (fp32) for which sums of the squares in another order give another n2, found by
# trying orders: block of rows, row, the first gain.
@pytest.mark.parametrize("d,seed,name,row,gain", [
    (1024, 81, "xt", 47, "0x1.04c166p+3"), (1024, 81, "xt", 182, "0x1.4e60cp+3"),
    (2560, 82, "xt6", 72, "0x1.aa11f8p+3"), (2560, 82, "xt2", 53, "0x1.83ccb4p+3"),
    (2560, 82, "xt9", 18, "0x1.d6e784p+3")])
def test_sum_of_squares_in_one_order(d, seed, name, row, gain):
    N = 2100
    c = Experts(65, "f32", N, d, 64, 2, 1, [0, 1050, 1050])
    x = gen.normal(seed, name, (400 if d == 1024 else 500, d))[row]
    x[0] = 4
    c.xt[:] = x
    c.x = to_dev(c.xt, torch.float32)
    g2 = np.ones(d, np.float32)
    g2[0] = float.fromhex(gain)
    gains(c, g2)
    whole = c.run()
    for n in (1, 4, 40, 333):
        assert torch.equal(part(c, np.arange(n)), whole[:n]), n


@pytest.mark.parametrize("act,N", SIZES + [("bf16", 4), ("bf16", 2600)])
@pytest.mark.parametrize("d", [256, 4224])
@pytest.mark.parametrize("size,gain,eps", [(2.0 ** 50, 2.0 ** 90, 1e-6), (2.0 ** -70, 2.0 ** -75, 1e-38),
                                           (2.0 ** 100, 2.0 ** 30, 1e-6), (1, 2.0 ** 100, 1e-6)])
def test_gains_far_from_one(act, N, d, size, gain, eps):
    """Products of tokens and gains that leave fp32 where the normalised token does not."""
    if d > 256 and N > 333 and N != 2600:
        N = 1500
    c = Experts(66, act, N, d, 128, 1, 1, [0, N])
    c.cfg.rms_eps = eps
    c.xt = gen.to_act(c.xt * np.float32(size), act)
    c.xt[N // 2] = 0
    c.x = to_dev(c.xt, torch_act(act))
    gains(c, c.g2 * gain)
    norm = gain * min(1.0, size / eps ** 0.5)
    for which in (0, 1):
        weight_scale(c, which, slice(None), 1 / norm)
    weight_scale(c, 2, slice(None), size)
    rows = some(N, 40)
    got = c.run()
    assert torch.isfinite(got).all()
    want, err = i8.moe(c.xt[rows], c.g2, *c.W, c.eidx[rows], c.gate[rows], act, eps=c.cfg.rms_eps)
    within(npy(got)[rows], want, err, "x_out")


# ------------------------------------------------------------------ linear
@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("N", [3, 40, 3000])
@pytest.mark.parametrize("size", [2.0 ** -119, 2.0 ** 104])
def test_linear_of_the_largest_and_smallest_tokens(size, N, act):
    k, m = 512, 264
    x, (w, t) = tokens(67, "x", N, k, act), weight(67, "W", m, k)
    x = gen.to_act(x / np.abs(x).max(axis=1, keepdims=True) * np.float32(size), act)
    t = (t / np.float32(size)).astype(np.float32)
    rows = some(N, 40)
    for guard in (3, 16):
        got = run_linear(to_dev(x, torch_act(act)), matrix(w, t), act, guard=guard)[rows]
        within(got, *i8.linear(x[rows], w, t, act), "y")


def test_linear_of_the_largest_tokens_and_longest_rows():
    """Every code +-127 along 2^17 channels of 2^104: sum times the token's scale is next to
    fp32's largest number."""
    k = 131072
    x = np.full((2, k), 2.0 ** 104, np.float32)
    x[1, ::2] *= -1
    w = np.full((3, k), 127, np.int8)
    w[1, ::2], w[2] = -127, -127
    t = np.full(3, 2.0 ** -110, np.float32)
    y, err = i8.linear(x, w, t, "f32")
    got = run_linear(to_dev(x, torch.float32), matrix(w, t), "f32")
    within(got, y, err, "y")
    assert np.abs(y).max() > 2.0 ** 17
