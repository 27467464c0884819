"""Host-side refusals of the 8-bit operators (no GPU)."""
import ctypes as C

import pytest
import torch

import paper_2607_06601_amd as tr

FAKE = 1 << 40


def cfg160(**over):
    c = tr.make_cfg(768, 12, 3, 64, 128, 8, 2, 2048, 64, "bf16")
    for k, v in over.items():
        setattr(c, k, v)
    return c


def w(codes=FAKE, scale=FAKE):
    return tr.I8W(codes, scale)


def quantize(act=tr.BF16, rows=4, cols=100, x=FAKE, ldx=100, codes=FAKE, scale=FAKE):
    return tr.lib().triroute_i8_quantize(act, rows, cols, x, ldx, codes, scale, None)


@pytest.mark.parametrize("over,code,word", [
    (dict(act=2), -1, b"act"), (dict(x=None), -1, b"NULL"), (dict(codes=None), -1, b"NULL"),
    (dict(scale=None), -1, b"NULL"), (dict(rows=0), -1, b"rows"), (dict(rows=-3), -1, b"rows"),
    (dict(cols=0), -1, b"channels"), (dict(cols=131073, ldx=131073), -2, b"32-bit"),
    (dict(ldx=99), -1, b"stride"), (dict(x=FAKE + 1), -1, b"aligned"),
    (dict(act=tr.F32, x=FAKE + 2), -1, b"aligned"), (dict(codes=FAKE + 8), -1, b"aligned"),
    (dict(scale=FAKE + 2), -1, b"aligned")])
def test_quantize_refuses(over, code, word):
    assert quantize(**over) == code
    assert word in tr.lib().triroute_last_error()


def linear(act=tr.BF16, n=16, k=100, m=50, x=FAKE, ldx=100, wt=None, res=None, ldr=50, y=2 * FAKE, ldy=50,
           ws=FAKE, ws_bytes=1 << 40):
    wt = w() if wt is None else wt
    return tr.lib().triroute_linear_i8(act, n, k, m, x, ldx, C.byref(wt), res, ldr, y, ldy, ws,
                                       ws_bytes, None)


@pytest.mark.parametrize("over,code,word", [
    (dict(act=-1), -1, b"act"), (dict(n=0), -1, b">= 1"), (dict(n=(1 << 24) + 1), -2, b"tokens"),
    (dict(k=0), -1, b"channels"), (dict(k=131073, ldx=131073), -2, b"32-bit"),
    (dict(m=0), -1, b"out"), (dict(m=(1 << 24) + 1, ldy=1 << 25), -1, b"out"),
    (dict(x=None), -1, b"NULL"), (dict(y=None), -1, b"NULL"), (dict(ws=None), -1, b"NULL"),
    (dict(wt=w(codes=None)), -1, b"codes"), (dict(wt=w(scale=None)), -1, b"codes"),
    (dict(wt=w(codes=FAKE + 4)), -1, b"aligned"), (dict(ldx=99), -1, b"x: row stride"),
    (dict(ldy=49), -1, b"y: row stride"), (dict(res=FAKE, ldr=49), -1, b"residual: row stride"),
    (dict(res=FAKE + 1), -1, b"aligned"), (dict(y=2 * FAKE, res=2 * FAKE, ldr=60), -1, b"y's row stride"),
    (dict(y=FAKE), -1, b"x's place"),
    (dict(ws=FAKE + 16), -1, b"aligned"), (dict(ws_bytes=2047), -3, b"workspace")])
def test_linear_refuses(over, code, word):
    assert linear(**over) == code
    assert word in tr.lib().triroute_last_error()


def test_linear_workspace():
    n = C.c_size_t()
    assert tr.lib().triroute_linear_i8_workspace_bytes(16, 100, C.byref(n)) == 0
    assert n.value == 16 * 128 + 256      # codes, scales (rounded to 256 B)
    assert tr.lib().triroute_linear_i8_workspace_bytes(16, 100, None) == -1
    assert tr.lib().triroute_linear_i8_workspace_bytes(0, 100, C.byref(n)) == -1


def qkv(c=None, B=2, T=8, n1=FAKE, q=FAKE, ws=FAKE, ws_bytes=1 << 44, **over):
    c = cfg160() if c is None else c
    dw = tr.DenseI8W(**{**dict(Wq=w(), Wk=w(), Wv=w()), **over})
    return tr.lib().triroute_qkv_i8(C.byref(c), B, T, n1, C.byref(dw), None, q, FAKE, FAKE, ws,
                                    ws_bytes, None)


@pytest.mark.parametrize("over,code,word", [
    (dict(n1=None), -1, b"NULL"), (dict(q=None), -1, b"NULL"), (dict(Wk=w(codes=None)), -1, b"codes"),
    (dict(Wv=w(scale=None)), -1, b"codes"), (dict(Wq=w(codes=FAKE + 8)), -1, b"aligned"),
    (dict(n1=FAKE + 8), -1, b"aligned"), (dict(B=0), -1, b">= 1"), (dict(ws=None), -1, b"workspace"),
    (dict(ws_bytes=64), -3, b"workspace"), (dict(c=cfg160(head_dim=96)), -2, b"head_dim"),
    (dict(c=cfg160(d_model=131136)), -2, b"32-bit")])
def test_qkv_refuses(over, code, word):
    assert qkv(**over) == code
    assert word in tr.lib().triroute_last_error()


def moe(c=None, n=16, xt=FAKE, xo=FAKE, g2=FAKE, eidx=FAKE, cmp=None, ws=FAKE, ws_bytes=1 << 44, **over):
    c = cfg160() if c is None else c
    dw = tr.DenseI8W(g2=g2)
    mw = tr.MoeI8W(**{**dict(Wgate=w(), Wup=w(), Wdown=w()), **over})
    cmp = tr.Compaction(exp_cnt=FAKE, exp_off=FAKE, exp_rows=FAKE) if cmp is None else cmp
    return tr.lib().triroute_moe_i8(C.byref(c), n, xt, C.byref(dw), C.byref(mw), eidx, FAKE,
                                    C.byref(cmp), xo, ws, ws_bytes, None)


@pytest.mark.parametrize("over,code,word", [
    (dict(xt=None), -1, b"NULL"), (dict(xo=None), -1, b"NULL"), (dict(g2=None), -1, b"g2"),
    (dict(eidx=None), -1, b"NULL"), (dict(Wgate=w(codes=None)), -1, b"codes"),
    (dict(Wdown=w(scale=None)), -1, b"codes"), (dict(Wup=w(codes=FAKE + 1)), -1, b"aligned"),
    (dict(cmp=tr.Compaction(exp_cnt=FAKE, exp_rows=FAKE)), -1, b"NULL"),
    (dict(g2=FAKE + 2), -1, b"aligned"), (dict(xo=FAKE + 4), -1, b"aligned"),
    (dict(n=0), -1, b">= 1"), (dict(ws=FAKE + 16), -1, b"aligned"), (dict(ws_bytes=64), -3, b"workspace"),
    (dict(c=cfg160(d_ff=131136)), -2, b"32-bit"), (dict(c=cfg160(d_ff=100)), -2, b"multiples")])
def test_moe_refuses(over, code, word):
    assert moe(**over) == code
    assert word in tr.lib().triroute_last_error()


def test_layer_refuses_missing_weights():
    c, lib = cfg160(), tr.lib()
    cache = tr.KVCacheDesc(base=FAKE, n_seq=4, capacity=64, tile_slots=64, n_tiles=1)
    rw = tr.RouterW(*[FAKE] * 12)
    mw = tr.MoeI8W(w(), w(), w())

    def call(decode, **over):
        dw = tr.DenseI8W(**{**dict(Wq=w(), Wk=w(), Wv=w(), Wo=w(), g2=FAKE), **over})
        a = (C.byref(c), 2) + (() if decode else (8,)) + (None, FAKE, FAKE, C.byref(rw), C.byref(dw),
                                                         C.byref(mw), C.byref(cache), FAKE, None, FAKE, 64, None)
        return (lib.triroute_layer_decode_i8 if decode else lib.triroute_layer_prefill_i8)(*a)

    for decode in (False, True):
        assert call(decode, Wo=w(codes=None)) == -1 and b"codes" in lib.triroute_last_error()
        assert call(decode, Wq=w(scale=None)) == -1
        assert call(decode, g2=None) == -1 and b"g2" in lib.triroute_last_error()
        assert call(decode) == -3
        op = tr.OP_LAYER_DECODE_I8 if decode else tr.OP_LAYER_PREFILL_I8
        assert tr.workspace_bytes(c, op, 2, 1) > tr.workspace_bytes(c, tr.OP_MOE_I8, 2, 1)


def test_matrix_takes_whole_rows_of_codes():
    codes, scale = torch.zeros(5, 128, dtype=torch.int8), torch.zeros(5)
    m = tr.I8Matrix(codes, scale, 100)
    assert m.rows == 5 and m.w.codes == codes.data_ptr() and m.w.scale == scale.data_ptr()
    for bad in ((codes, scale, 129), (codes[:, :100], scale, 100), (codes.float(), scale, 100),
                (codes, scale[:4], 100), (codes, scale.double(), 100)):
        with pytest.raises(ValueError):
            tr.I8Matrix(*bad)


def test_tensors_of_other_shapes_are_refused(monkeypatch):
    class Stream:  # (no GPU here: tensors of the CPU have the index -1)
        device_index, cuda_stream = -1, 0

    monkeypatch.setattr(tr, "_i8_stream", lambda s: Stream if s is None else s)
    m = tr.I8Matrix(torch.zeros(5, 128, dtype=torch.int8), torch.zeros(5), 100)
    x, y, ws = torch.zeros(3, 100), torch.zeros(3, 5), torch.zeros(4096, dtype=torch.uint8)
    for bad, word in ((dict(x=x[:, :99]), "x"), (dict(y=y[:2]), "y"), (dict(y=y.bfloat16()), "y"),
                      (dict(residual=y[:, :4]), "residual"), (dict(x=x.double()), "x"),
                      (dict(x=torch.zeros(100, 3).T), "contiguous"), (dict(residual=y.bfloat16()), "residual"),
                      (dict(y=torch.zeros(5, 3).T), "contiguous")):
        a = {**dict(x=x, y=y, residual=None), **bad}
        with pytest.raises(ValueError, match=word):
            tr.linear_i8(a["x"], m, a["y"], ws, residual=a["residual"])
    Stream.device_index = 0                        # ... and are refused by a stream of a GPU
    with pytest.raises(ValueError, match="current GPU"):
        tr.linear_i8(x, m, y, ws)
    with pytest.raises(ValueError, match="current GPU"):
        tr.i8_quantize(x, torch.zeros(3, 128, dtype=torch.int8), torch.zeros(3))
    Stream.device_index = -1
    for codes, scale in ((torch.zeros(3, 100, dtype=torch.int8), torch.zeros(3)),
                         (torch.zeros(3, 128, dtype=torch.int8), torch.zeros(2)),
                         (torch.zeros(3, 128), torch.zeros(3))):
        with pytest.raises(ValueError):
            tr.i8_quantize(x, codes, scale)


@pytest.mark.parametrize("act,N", [("bf16", 3), ("bf16", 700), ("f32", 700)])
def test_experts_workspace_holds_what_is_used(act, N):
    """Codes and scales of the normalised and the hidden rows, both rows' fp32 values, the
    lists' entries: nothing else."""
    d, f, k = 768, 2112, 2
    c, rows = tr.make_cfg(d, 12, 3, 64, 128, 8, k, f, 64, act), N * k
    used = rows * (768 + 2176 + 4 + 4 + 4 * f + 4 * d + 4)
    assert used <= tr.workspace_bytes(c, tr.OP_MOE_I8, N, 1) <= used + 7 * 255


class CpuStream:  # (no GPU here: tensors of the CPU have the index -1)
    device_index, cuda_stream = -1, 0


def zeros_i8(rows, cols):
    return tr.I8Matrix(torch.zeros(rows, tr.i8_pitch(cols), dtype=torch.int8), torch.zeros(rows), cols)


def layer_calls(cfg, dw, mw, t, cache):
    """Each call over a layer's weights, its tensors being t (too small for a call: refused before it)."""
    return dict(
        qkv=lambda: tr.qkv_i8(cfg, 1, 1, t, dw, t, t, t, t),
        moe=lambda: tr.moe_i8(cfg, 1, t, dw, mw, t, t, tr.Compaction(), t, t),
        prefill=lambda: tr.layer_prefill_i8(cfg, 1, 1, t, t, tr.RouterW(), dw, mw, cache, t, t),
        decode=lambda: tr.layer_decode_i8(cfg, 1, t, t, tr.RouterW(), dw, mw, cache, t, t))


def test_matrices_of_other_shapes_are_refused(monkeypatch):
    monkeypatch.setattr(tr, "_i8_stream", lambda s: CpuStream if s is None else s)
    c = cfg160(n_experts=3, d_ff=128)
    d, hd, kd, f, E = 768, 768, 192, 128, 3
    dense = dict(Wq=(hd, d), Wk=(kd, d), Wv=(kd, d), Wo=(d, hd))
    experts = dict(Wgate=(E * f, d), Wup=(E * f, d), Wdown=(E * d, f))
    t = torch.zeros(16)

    class Cache:
        buf, ref = t, None

    def weights(kind, shapes, **over):
        return kind(**{n: zeros_i8(*s).w for n, s in {**shapes, **over}.items()})

    good_d, good_m = weights(tr.DenseI8W, dense), weights(tr.MoeI8W, experts)
    for name in ("qkv", "moe", "prefill", "decode"):          # these reach the library, which wants more
        with pytest.raises(RuntimeError):
            layer_calls(c, good_d, good_m, t, Cache)[name]()
    for over, names in ((dict(Wq=(hd, d - 64)), ("qkv", "prefill", "decode")), (dict(Wk=(hd, d)), ("qkv", "prefill")),
                        (dict(Wv=(kd - 64, d)), ("qkv", "decode")), (dict(Wo=(d - 1, hd)), ("prefill", "decode"))):
        dw = weights(tr.DenseI8W, dense, **over)
        for name in names:
            with pytest.raises(ValueError, match=next(iter(over))):
                layer_calls(c, dw, good_m, t, Cache)[name]()
    for over in (dict(Wgate=(2 * f, d)), dict(Wup=(E * f, d + 64)), dict(Wdown=(E * d, f + 1)), dict(Wdown=(E * f, d))):
        mw = weights(tr.MoeI8W, experts, **over)
        for name in ("moe", "prefill", "decode"):
            with pytest.raises(ValueError, match=next(iter(over))):
                layer_calls(c, good_d, mw, t, Cache)[name]()
    # a matrix set later counts, one set back too, and another layer's call does not remember this one's
    good_m.Wup = zeros_i8(E * f, 64).w
    with pytest.raises(ValueError, match="Wup"):
        layer_calls(c, good_d, good_m, t, Cache)["moe"]()
    good_m.Wup = zeros_i8(E * f, d).w
    with pytest.raises(RuntimeError):
        layer_calls(c, good_d, good_m, t, Cache)["moe"]()
    with pytest.raises(ValueError, match="Wgate"):
        layer_calls(cfg160(n_experts=4, d_ff=128), good_d, good_m, t, Cache)["moe"]()


def test_weights_keep_their_matrices():
    m = zeros_i8(5, 100)
    at = m.codes.data_ptr()
    held = m.codes
    mw = tr.MoeI8W(Wgate=m.w)
    del m
    assert mw.Wgate.codes == at and mw.held["Wgate"].held[0] is held


def test_tensors_and_matrices_of_another_gpu_are_refused(monkeypatch):
    class Gpu:
        device_index, cuda_stream = 0, 0

    c, t = cfg160(n_experts=3, d_ff=128), torch.zeros(16)

    class Cache:
        buf, ref = t, None

    monkeypatch.setattr(tr, "_i8_stream", lambda s: Gpu)
    for call in layer_calls(c, tr.DenseI8W(), tr.MoeI8W(), t, Cache).values():
        with pytest.raises(ValueError, match="current GPU"):
            call()
    # tensors given as addresses, matrices of the CPU
    Cache.buf = 0
    dw = tr.DenseI8W(Wk=zeros_i8(192, 768).w)
    mw = tr.MoeI8W(Wdown=zeros_i8(3 * 768, 128).w)

    for name, word in (("qkv", "Wk"), ("moe", "Wdown"), ("prefill", "Wk"), ("decode", "Wk")):
        with pytest.raises(ValueError, match=word + ".*current GPU"):
            layer_calls(c, dw, mw, FAKE, Cache)[name]()
