"""Gradient norm and clipping (triroute_grad_*) against numpy in fp64.

The norm's squares are summed in fp64: its error is that of n fp64 additions,
n 2^-53 relative at most.  A clipped value is off by the rounding of the
coefficient and of the product to fp32 (2^-24 each) and, in bf16, by one
rounding to bf16 (2^-8)."""
import math

import numpy as np
import pytest
import torch

import paper_2607_06601_amd as tr

from _common import npy

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    tr.lib()
    yield
    torch.cuda.synchronize()


def tensors(spec, seed=0, scale=1.0, shift=0):
    """[(elements, bf16?)] -> views of one buffer per type, `shift` elements off
    its start and packed without gaps, so that their alignments differ."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    out, at = [], {False: shift, True: shift}
    size = {h: shift + sum(n for n, x in spec if x == h) + 8 for h in (False, True)}
    buf = {h: (torch.randn(size[h], generator=g, device=DEV) * scale)
           .to(torch.bfloat16 if h else torch.float32) for h in (False, True)}
    for n, h in spec:
        out.append(buf[h][at[h]:at[h] + n])
        at[h] += n
    return out, buf


def f64(t):
    return npy(t).astype(np.float64)


def expect(ts, norm_type):
    v = [f64(t) for t in ts]
    if norm_type == 2:
        return math.sqrt(math.fsum(float((x * x).sum()) for x in v))
    return max((float(np.abs(x).max()) for x in v if x.size), default=0.0)


def check(src, dst, norm, max_norm, norm_type):
    want = expect(src, norm_type)
    n = sum(t.numel() for t in src)
    assert abs(norm.item() - want) <= (n + 2) * 2.0 ** -53 * want
    c = 1.0 if want <= max_norm else max_norm / want
    for s, d in zip(src, dst):
        x, y = f64(s) * c, f64(d)
        u = (2.0 ** -8 if s.dtype == torch.bfloat16 else 0.0) + 3 * 2.0 ** -24
        if c == 1.0:
            np.testing.assert_array_equal(y, x)
        else:
            assert (np.abs(y - x) <= u * np.abs(x) + 1e-40).all()


SPECS = {
    "one": [(1, False)],
    "one bf16": [(1, True)],
    "empty among": [(0, False), (5, True), (0, True), (3, False)],
    "piece edges": [(4095, False), (4096, False), (4097, False), (8191, True), (8192, True),
                    (8193, True), (16384 + 3, True)],
    "odd": [(n, i % 3 == 0) for i, n in enumerate((7, 1, 13, 1000, 33, 2, 65537, 12345, 15, 17))],
    "past one batch": [(1 + 37 * i % 301, i % 2 == 0) for i in range(150)],
    "large": [(3_000_001, True), (1_000_003, False)],
}


@pytest.mark.parametrize("norm_type", [2.0, math.inf])
@pytest.mark.parametrize("ratio", [0.3, 7.0])
@pytest.mark.parametrize("name", SPECS)
def test_clip(name, ratio, norm_type):
    for shift in (0, 1, 3):
        src, _ = tensors(SPECS[name], seed=shift, shift=shift)
        max_norm = expect(src, norm_type) / ratio
        dst, around = tensors(SPECS[name], seed=9, shift=shift)
        before = {h: b.clone() for h, b in around.items()}
        norm = torch.full((1,), float("nan"), dtype=torch.float64, device=DEV)
        ws = tr.grad_workspace()
        ws.fill_(0xFF)
        tr.grad_clip(tr.GradList(src, dst), max_norm, norm, ws, norm_type)
        torch.cuda.synchronize()
        check(src, dst, norm, max_norm, norm_type)
        for h, b in around.items():  # nothing beside the tensors is written
            used = shift + sum(n for n, x in SPECS[name] if x == h)
            assert torch.equal(b[:shift], before[h][:shift]) and torch.equal(b[used:], before[h][used:])
        # the two calls give the same norm and values; so does clipping in place
        two, _ = tensors(SPECS[name], seed=10, shift=shift)
        n2 = torch.zeros_like(norm)
        gl = tr.GradList(src, two)
        tr.grad_norm(gl, n2, ws, norm_type)
        tr.grad_scale(gl, n2, max_norm)
        assert n2.item() == norm.item()
        here = [t.clone() for t in src]
        tr.grad_clip(tr.GradList(here), max_norm, n2, ws, norm_type)
        torch.cuda.synchronize()
        for a, b, c in zip(dst, two, here):
            assert torch.equal(a, b) and torch.equal(a, c)


def test_source_and_destination_that_lie_differently():
    spec = [(1000, True), (777, False), (20000, True)]
    for a, b in ((0, 1), (1, 0), (3, 2), (0, 4)):
        src, _ = tensors(spec, seed=1, shift=a)
        dst, _ = tensors(spec, seed=2, shift=b)
        norm, ws = torch.zeros(1, dtype=torch.float64, device=DEV), tr.grad_workspace()
        tr.grad_clip(tr.GradList(src, dst), 1.0, norm, ws)
        torch.cuda.synchronize()
        check(src, dst, norm, 1.0, 2.0)


def test_range_of_squares():
    """Squares beyond fp32's range, and below it, count."""
    for scale in (1e30, 1e-30):
        src, _ = tensors([(5000, False), (3000, True)], seed=3, scale=scale)
        dst = [torch.empty_like(t) for t in src]
        norm, ws = torch.zeros(1, dtype=torch.float64, device=DEV), tr.grad_workspace()
        tr.grad_clip(tr.GradList(src, dst), scale, norm, ws)
        torch.cuda.synchronize()
        check(src, dst, norm, scale, 2.0)


@pytest.mark.parametrize("norm_type", [2.0, math.inf])
def test_values_that_are_no_numbers(norm_type):
    ws, norm = tr.grad_workspace(), torch.zeros(1, dtype=torch.float64, device=DEV)
    for bad, want in ((float("nan"), float("nan")), (float("-inf"), float("inf"))):
        for at in (0, 4099):
            src, _ = tensors([(6000, False), (6000, True)], seed=4)
            src[1][at] = bad
            tr.grad_norm(tr.GradList(src), norm, ws, norm_type)
            got = norm.item()
            assert got == want or (math.isnan(got) and math.isnan(want))
            tr.grad_clip(tr.GradList(src), 1.0, norm, ws, norm_type)
            torch.cuda.synchronize()
            # as the formula says: NaN everywhere, or 0 with a NaN for the infinity
            if math.isnan(want):
                assert torch.isnan(src[0]).all() and torch.isnan(src[1]).all()
            else:
                assert (src[0] == 0).all() and torch.isnan(src[1][at])
    # both at once: NaN wins
    src, _ = tensors([(6000, False)], seed=4)
    src[0][5], src[0][5000] = float("inf"), float("nan")
    tr.grad_norm(tr.GradList(src), norm, ws, norm_type)
    assert math.isnan(norm.item())


def test_zero_gradients_and_zero_threshold():
    ws, norm = tr.grad_workspace(), torch.ones(1, dtype=torch.float64, device=DEV)
    z = [torch.zeros(100, device=DEV), torch.zeros(33, device=DEV, dtype=torch.bfloat16)]
    tr.grad_clip(tr.GradList(z), 0.0, norm, ws)
    assert norm.item() == 0.0 and all((t == 0).all() for t in z)
    src, _ = tensors([(100, False)], seed=5)
    tr.grad_clip(tr.GradList(src), 0.0, norm, ws)
    assert (src[0] == 0).all()
    src, _ = tensors([(100, False)], seed=5)
    keep = src[0].clone()
    tr.grad_clip(tr.GradList(src), math.inf, norm, ws)
    assert torch.equal(src[0], keep) and norm.item() > 0
    tr.grad_norm(tr.GradList([torch.empty(0, device=DEV)]), norm, ws)
    assert norm.item() == 0.0


def test_stream_graph_and_same_bits():
    src, _ = tensors(SPECS["odd"] * 30, seed=6)
    dst = [torch.empty_like(t) for t in src]
    norm, ws = torch.zeros(1, dtype=torch.float64, device=DEV), tr.grad_workspace()
    gl = tr.GradList(src, dst)
    tr.grad_clip(gl, 1.0, norm, ws)
    torch.cuda.synchronize()
    want, wn = [t.clone() for t in dst], norm.item()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    tr.grad_clip(gl, 1.0, norm, ws, stream=s)
    s.synchronize()
    assert norm.item() == wn and all(torch.equal(a, b) for a, b in zip(dst, want))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        tr.grad_clip(gl, 1.0, norm, ws)
    for rep in range(3):
        norm.fill_(float("nan"))
        for t in dst:
            t.fill_(float("nan"))
        ws.fill_(0xFF)
        g.replay()
        torch.cuda.synchronize()
        assert norm.item() == wn and all(torch.equal(a, b) for a, b in zip(dst, want)), rep
    for t in src:
        t.mul_(2)
    g.replay()
    torch.cuda.synchronize()
    assert norm.item() == 2 * wn


def test_list_written_on_a_stream_of_its_own():
    """The list is written, and its memory taken, on the stream given: what the current
    stream still does with memory that it has freed does not reach it."""
    src = [torch.randn(5000 + i, device=DEV) for i in range(20)]
    want = math.sqrt(sum(float((t.double() ** 2).sum()) for t in src))
    ws, s = tr.grad_workspace(), torch.cuda.Stream()
    norm = torch.zeros(1, dtype=torch.float64, device=DEV)
    torch.cuda.synchronize()
    for _ in range(5):
        junk = [torch.empty(4096, dtype=torch.uint8, device=DEV) for _ in range(64)]
        big = torch.empty(1 << 28, device=DEV).fill_(1.0)  # (the current stream is busy)
        for t in junk:
            t.fill_(0xFF)
        del junk, big
        gl = tr.GradList(src, stream=s)
        tr.grad_norm(gl, norm, ws, stream=s)
        torch.cuda.synchronize()
        assert abs(norm.item() - want) <= 1e-12 * want


def test_list_dropped_while_a_call_on_another_stream_is_queued():
    """Its memory, and that of tensors which only the list held, goes to no other tensor
    before the call is done."""
    s = torch.cuda.Stream()
    for n in (1, 40):
        src = [torch.randn(3000 + i, device=DEV) for i in range(n)]
        want = math.sqrt(sum(float((t.double() ** 2).sum()) for t in src))
        norm, ws = torch.zeros(1, dtype=torch.float64, device=DEV), tr.grad_workspace()
        busy = torch.empty(1 << 29, device=DEV)
        torch.cuda.synchronize()
        gl = tr.GradList(src)
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            for i in range(50):
                busy.fill_(i)
        tr.grad_clip(gl, 1.0, norm, ws, stream=s)
        held = {gl.buf.data_ptr()} | {t.data_ptr() for t in src}
        sizes = [gl.buf.numel()] + [4 * t.numel() for t in src]
        del gl, src
        new = [torch.empty(b, dtype=torch.uint8, device=DEV) for b in sizes for _ in range(4)]
        if not s.query():  # the call is still queued
            assert not held & {t.data_ptr() for t in new}
        torch.cuda.synchronize()
        assert abs(norm.item() - want) <= 1e-12 * want
