"""Host-side refusals of the training operators (no GPU): the expert backward
pass and the gradient list, norm and clipping."""
import ctypes as C
import math

import pytest
import torch

import paper_2607_06601_amd as tr

FAKE = 1 << 40


def cfg160(**over):
    c = tr.make_cfg(768, 12, 3, 64, 128, 8, 2, 2048, 64, "bf16")
    for k, v in over.items():
        setattr(c, k, v)
    return c


def backward(c=None, n=16, ws_bytes=1 << 44, xt=FAKE, dx=FAKE, eidx=FAKE, ws=FAKE, cmp=None, mw=None,
             **out):
    c = cfg160() if c is None else c
    o = tr.MoeGradOut(**{**dict(dxt=FAKE, dWgate=FAKE, dWup=FAKE, dWdown=FAKE, dg2=FAKE, g_gate=FAKE),
                         **out})
    dw = tr.DenseW(g2=FAKE)
    mw = tr.MoeW(FAKE, FAKE, FAKE) if mw is None else mw
    cmp = tr.Compaction(exp_cnt=FAKE, exp_off=FAKE, exp_rows=FAKE) if cmp is None else cmp
    return tr.lib().triroute_moe_backward(C.byref(c), n, xt, C.byref(dw), C.byref(mw), eidx, FAKE,
                                          C.byref(cmp), dx, C.byref(o), ws, ws_bytes, None)


@pytest.mark.parametrize("over,code,word", [
    (dict(xt=None), -1, b"NULL"), (dict(dx=None), -1, b"NULL"), (dict(eidx=None), -1, b"NULL"),
    (dict(dxt=None), -1, b"NULL"), (dict(mw=tr.MoeW(FAKE, None, FAKE)), -1, b"NULL"),
    (dict(cmp=tr.Compaction(exp_cnt=FAKE, exp_rows=FAKE)), -1, b"NULL"),
    (dict(dWup=None), -1, b"all"), (dict(dWgate=None), -1, b"all"), (dict(dWdown=None), -1, b"all"),
    (dict(dxt=FAKE + 8), -1, b"aligned"), (dict(dWup=FAKE + 2), -1, b"aligned"),
    (dict(xt=FAKE + 4), -1, b"aligned"), (dict(dg2=FAKE + 2), -1, b"aligned"),
    (dict(n=0), -1, b">= 1"), (dict(n=(1 << 24) + 1), -2, b"tokens"),
    (dict(ws=None), -1, b"workspace"), (dict(ws=FAKE + 16), -1, b"aligned"),
    (dict(ws_bytes=1024), -3, b"workspace"), (dict(c=cfg160(d_ff=100)), -2, b"multiples")])
def test_moe_backward_refuses(over, code, word):
    assert backward(**over) == code
    assert word in tr.lib().triroute_last_error()


def test_moe_backward_workspace():
    c = cfg160()
    need = tr.workspace_bytes(c, tr.OP_MOE_BACKWARD, 16, 1)
    assert backward(ws_bytes=need - 1) == -3
    # the rows' four operands, and dn in fp32
    rows = 16 * 2
    assert need >= rows * (2 * 768 + 3 * 2048) * 2 + rows * 768 * 4
    assert tr.workspace_bytes(c, tr.OP_MOE_BACKWARD, 1000, 1) > need


def tensor(src=FAKE, dst=FAKE, numel=100, dtype=tr.F32):
    return tr.GradTensor(src, dst, numel, dtype)


def list_bytes(*ts, n=None):
    arr = (tr.GradTensor * max(1, len(ts)))(*ts)
    need = C.c_size_t()
    r = tr.lib().triroute_grad_list_bytes(arr, len(ts) if n is None else n, C.byref(need))
    return r, need.value


@pytest.mark.parametrize("bad,word", [
    (tensor(dtype=2), b"dtype"), (tensor(numel=-1), b"numel"), (tensor(src=None), b"NULL"),
    (tensor(src=FAKE + 2), b"aligned"), (tensor(dst=FAKE + 1), b"aligned"),
    (tensor(src=FAKE + 1, dtype=tr.BF16), b"aligned"), (tensor(numel=1 << 41), b"numel")])
def test_grad_list_refuses_tensors(bad, word):
    assert list_bytes(tensor(), bad)[0] == -1
    assert word in tr.lib().triroute_last_error()
    arr = (tr.GradTensor * 2)(tensor(), bad)
    d = tr.GradListDesc()
    assert tr.lib().triroute_grad_list_init(C.byref(d), arr, 2, FAKE, 1 << 30, None) == -1
    assert d.base is None


def test_grad_list_sizes():
    assert list_bytes(tensor(), n=0)[0] == -1
    # pieces of 16 KB, counted from the 16-byte address at or before src
    assert list_bytes(tensor(numel=0, src=None, dst=None)) == (0, 256)
    one = list_bytes(tensor(numel=4096))[1]
    assert one == list_bytes(tensor(numel=1))[1] == 256
    big = list_bytes(tensor(numel=1 << 30))[1]
    assert 24 * (1 << 18) <= big < 24 * (1 << 18) + 512
    d = tr.GradListDesc()
    arr = (tr.GradTensor * 1)(tensor(numel=1 << 30))
    f = tr.lib().triroute_grad_list_init
    assert f(C.byref(d), arr, 1, FAKE, big - 256, None) == -3
    assert f(C.byref(d), arr, 1, FAKE + 128, big, None) == -1
    assert f(C.byref(d), None, 1, FAKE, big, None) == -1


def test_grad_calls_refuse():
    lib = tr.lib()
    d = tr.GradListDesc(FAKE, 1, 1, 1)
    clip = lambda d=d, t=2.0, m=1.0, norm=FAKE, ws=FAKE, n=tr.GRAD_WS_BYTES: \
        lib.triroute_grad_clip(C.byref(d), t, m, norm, ws, n, None)  # noqa: E731
    assert clip(t=1.0) == -2 and b"norm_type" in lib.triroute_last_error()
    assert clip(t=-math.inf) == -2 and clip(t=math.nan) == -2
    assert clip(m=-1.0) == -1 and clip(m=math.nan) == -1
    assert clip(norm=None) == -1 and clip(norm=FAKE + 4) == -1
    assert clip(ws=None) == -1 and clip(ws=FAKE + 8) == -1 and clip(n=100) == -3
    assert clip(d=tr.GradListDesc()) == -1
    measured = tr.GradListDesc(FAKE, 1, 1, 0)
    assert clip(d=measured) == -1 and b"dst" in lib.triroute_last_error()
    assert lib.triroute_grad_scale(C.byref(measured), FAKE, 1.0, None) == -1
    assert lib.triroute_grad_scale(C.byref(d), FAKE, math.nan, None) == -1
    assert lib.triroute_grad_norm(C.byref(d), 3.0, FAKE, FAKE, tr.GRAD_WS_BYTES, None) == -2


def test_binding_refuses():
    f, h = torch.zeros(4, 4), torch.zeros(4, 4, dtype=torch.bfloat16)
    for bad in ([], [torch.zeros(3, dtype=torch.float16)], [f.t()[1:]]):
        with pytest.raises(ValueError):
            tr.GradList(bad)
    for dst in ([f], [f, f, f], [f, f]):
        with pytest.raises(ValueError):
            tr.GradList([f, h], dst)
    with pytest.raises(ValueError):
        tr.GradList([f], [torch.zeros(5)])


def test_binding_refuses_overlaps_and_host_tensors():
    """A destination that is another tensor, or another destination, in part or whole: its
    pieces would be scaled twice or under a reader.  Tensors in host memory: no kernel may
    be given their addresses."""
    flat, other = torch.zeros(100), torch.zeros(100)
    a, b, c = flat[:40], flat[40:80], flat[30:60]
    for src, dst in (([a, a], None), ([a, c], None), ([a, b], [other[:40], other[20:60]]),
                     ([a, b], [b, other[:40]]), ([a, b], [other[:40], a]), ([a], [flat[1:41]]),
                     ([flat, b], [other, b])):
        with pytest.raises(ValueError, match="overlap"):
            tr.GradList(src, dst)
    # none of these overlap; they are refused only for where they lie
    empty = flat[50:50]
    for src, dst in (([a, b], None), ([a, a], [other[:40], other[40:80]]), ([a, empty, b], None),
                     ([a, b], [other[40:80], other[:40]]), ([flat], [other])):
        with pytest.raises(ValueError, match="current GPU"):
            tr.GradList(src, dst)


def test_norm_must_lie_with_the_gradients():
    class L:
        ref = None
        device = torch.device("cuda", 0)
    norm, ws = torch.zeros(1, dtype=torch.float64), torch.zeros(tr.GRAD_WS_BYTES, dtype=torch.uint8)
    for call in (lambda: tr.grad_norm(L, norm, ws), lambda: tr.grad_scale(L, norm, 1.0),
                 lambda: tr.grad_clip(L, 1.0, norm, ws)):
        with pytest.raises(ValueError, match="device"):
            call()
    L.device = torch.device("cpu")
    with pytest.raises(ValueError, match="fp64"):
        tr.grad_norm(L, norm.float(), ws)


class FakeStream:
    device = torch.device("cuda", 0)

    def __init__(self, handle):
        self.cuda_stream = handle


class FakeTensor:
    """What the binding asks of a tensor on a GPU."""
    device, dtype = torch.device("cuda", 0), torch.float64

    def __init__(self, numel=1):
        self.n, self.streams = numel, []

    def numel(self):
        return self.n

    def data_ptr(self):
        return FAKE

    def record_stream(self, stream):
        self.streams.append(stream.cuda_stream)


class FakeLib:
    """Entry points that launch nothing."""

    def __init__(self):
        self.streams = []

    def __getattr__(self, name):
        return lambda *a: self.streams.append(a[-1]) or 0


@pytest.fixture
def fake_list(monkeypatch):
    """A list of two tensors as its constructor leaves it on stream 7, and the calls'
    arguments: no GPU is touched."""
    g = object.__new__(tr.GradList)
    a, b, c = FakeTensor(), FakeTensor(), FakeTensor()
    g.tensors, g.dst, g.buf, g.device, g.desc = [a, b], [a, c], FakeTensor(), a.device, tr.GradListDesc()
    g._known = {7}
    lib = FakeLib()
    monkeypatch.setattr(tr, "lib", lambda: lib)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: FakeStream(7))
    norm, ws = FakeTensor(), FakeTensor(tr.GRAD_WS_BYTES)
    calls = [lambda **k: tr.grad_norm(g, norm, ws, **k), lambda **k: tr.grad_scale(g, norm, 1.0, **k),
             lambda **k: tr.grad_clip(g, 1.0, norm, ws, **k)]
    return g, lib, calls


@pytest.mark.parametrize("which", range(3))
def test_calls_on_other_streams_hold_the_memory_of_list_and_tensors(fake_list, which):
    """The list's memory holds addresses that kernels read and write: given to another tensor
    while a call is queued, they would be any."""
    g, lib, calls = fake_list
    held = (g.buf, *g.tensors, *g.dst)
    calls[which]()
    assert lib.streams == [7] and not any(t.streams for t in held)
    calls[which](stream=FakeStream(9))
    assert lib.streams == [7, 9] and all(set(t.streams) == {9} for t in held)
    calls[which](stream=FakeStream(11))
    assert lib.streams == [7, 9, 11] and all(set(t.streams) == {9, 11} for t in held)


def test_list_takes_any_iterable():
    """Such as the gradients of a module's parameters; host tensors are refused only for
    where they lie."""
    t = [torch.zeros(4), torch.zeros(5, dtype=torch.bfloat16)]
    for args in ((iter(t),), (iter(t), iter([x.clone() for x in t])), (tuple(t), None)):
        with pytest.raises(ValueError, match="current GPU"):
            tr.GradList(*args)


@pytest.mark.parametrize("which", range(3))
def test_calls_refuse_another_current_device_and_its_streams(fake_list, which, monkeypatch):
    """A launch goes to the current device, whose streams do not order the list's memory."""
    g, lib, calls = fake_list
    other = FakeStream(9)
    other.device = torch.device("cuda", 1)
    with pytest.raises(ValueError, match="device"):
        calls[which](stream=other)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    for kw in ({}, dict(stream=FakeStream(9))):
        with pytest.raises(ValueError, match="current GPU"):
            calls[which](**kw)
    assert lib.streams == []


def test_list_refuses_a_stream_of_another_device(monkeypatch):
    """(host tensors, called the current GPU's)"""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)

    class OnGpu(torch.Tensor):
        device = torch.device("cuda", 0)
    other = FakeStream(9)
    other.device = torch.device("cuda", 1)
    with pytest.raises(ValueError, match="stream"):
        tr.GradList([torch.zeros(4).as_subclass(OnGpu)], stream=other)


def grad_list_init(*ts):
    """Into no memory at all: a list that is right is refused only for that, and nothing is
    launched."""
    d = tr.GradListDesc()
    r = tr.lib().triroute_grad_list_init(C.byref(d), (tr.GradTensor * len(ts))(*ts), len(ts), FAKE, 0, None)
    assert d.base is None
    return r, tr.lib().triroute_last_error()


A, B = FAKE, FAKE + (1 << 20)
HALF = tr.BF16


@pytest.mark.parametrize("ts", [
    [tensor(A, A), tensor(A, A)],                                   # one tensor twice, in place
    [tensor(A, A), tensor(A + 396, A + 396)],                       # .. the last element shared
    [tensor(A, A, dtype=HALF), tensor(A + 198, B, dtype=HALF)],
    [tensor(A, B), tensor(A + 400, B)],                             # one destination for two
    [tensor(A, B), tensor(A + 400, B + 4)],
    [tensor(A, A + 200)],                                           # over a part of its own source
    [tensor(A + 200, A)],
    [tensor(A, A + 400), tensor(A + 400, B)],                       # over another's source
    [tensor(A, B), tensor(B + 396, A + 800)],
    [tensor(A, B, numel=4000), tensor(B + 16, A + 40000, numel=1)],  # .. one far inside it
    [tensor(A, A), tensor(A, None, numel=1)],                       # measured while it is scaled
    [tensor(A, B), tensor(A + 8000, A + 400), tensor(A + 796, A + 4000)],
])
def test_grad_list_refuses_overlaps(ts):
    for order in (ts, ts[::-1]):
        r, why = grad_list_init(*order)
        assert r == -1 and b"overlap" in why, (r, why)


@pytest.mark.parametrize("ts", [
    [tensor(A, A)],
    [tensor(A, A), tensor(A + 400, A + 400)],                       # one behind the other
    [tensor(A, B), tensor(A, B + 400)],                             # one source for two
    [tensor(A, None), tensor(A, None), tensor(A + 4, None)],        # only measured
    [tensor(A, B), tensor(A + 400, A + 800), tensor(B + 400, B + 800)],
    [tensor(A, A), tensor(A, A, numel=0), tensor(A + 8, A + 12, numel=0)],
    [tensor(A, A, dtype=HALF), tensor(A + 200, A + 200, dtype=HALF), tensor(A + 400, A + 400)],
])
def test_grad_list_takes_neighbours(ts):
    for order in (ts, ts[::-1]):
        assert grad_list_init(*order)[0] == -3


def test_grad_list_of_many_tensors():
    ts = [tensor(A + 1000 * i, B * 2 + 1000 * i, numel=250) for i in range(5000)]
    assert grad_list_init(*ts)[0] == -3
    ts[4321] = tensor(A + 1000 * 4321, ts[17].dst + 996, numel=250)
    assert grad_list_init(*ts)[0] == -1
