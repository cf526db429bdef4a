"""What the e4m3 linear layers and the clipping refuse: the C entry points by their
status, the torch wrappers by an exception, in each case before any device
work; and the experts' rows that offsets stand for.  CPU only; the addresses
below are never read."""
import contextlib
import copy
import ctypes
import os
import pickle
import types

import numpy as np
import pytest

import f8_reference as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2609_26077_amd", "libfmm8.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libfmm8.so not built")

P = 1 << 20        # an aligned address


@pytest.fixture(scope="module")
def fm():
    import paper_2609_26077_amd as fm
    return fm


def status(fm, name, *args):
    return getattr(fm._lib, name)(*args)


def test_reference_codes_are_torchs():
    """The oracle's codes against a conversion by other code, its scales by direct search."""
    import torch
    u = np.concatenate([np.linspace(-448, 448, 40001), 2.0 ** np.arange(-12, 8.5, 1 / 64), [0.0, -0.0, 17.0, 19.0]])
    u = u.astype(np.float32)
    want = torch.from_numpy(u).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(ref.nearest(u.astype(np.float64)), want)
    for a in (1e-45, 2.0 ** -118, 0.4375, np.nextafter(0.4375, 1), 1.0, 447.99, 448.0, 448.001, 3.4e38):
        e = -126
        while a > 448 * 2.0 ** e:
            e += 1
        assert ref.exponent(a) == e
    assert ref.exponent(0.0) == 0


def test_reference_spans():
    assert ref.spans([0, 3, 3, 10], 10) == [(0, 3), (3, 3), (3, 10)]
    assert ref.spans([-5, 6, 4, 99, 7], 10) == [(0, 6), (6, 6), (6, 10), (10, 10)]


def test_pitches(fm):
    from paper_2609_26077_amd import f8
    for cols in (0, 1, 127, 128, 129, 2048, 2049, 4096, 131071):
        assert fm.fmm_f8_scale_pitch(cols) == f8.scale_pitch(cols) == ref.scale_pitch(cols)
        assert f8.pitch(cols) == ref.pitch(cols)
    assert fm.fmm_f8_scale_pitch(-1) == -1


@pytest.mark.parametrize("weight", [False, True])
def test_quantize_refuses(fm, weight):
    def call(type=0, count=1, rows=4, cols=8, x=P, codes=P, scales=P):
        if weight:
            return status(fm, "fmm_f8_quantize_weight", type, count, rows, cols, x, codes, scales, None)
        return status(fm, "fmm_f8_quantize", type, rows, cols, x, codes, scales, None)

    for bad in (dict(type=3), dict(type=-1), dict(rows=-1), dict(cols=-1), dict(x=None), dict(codes=None), dict(scales=None),
                dict(x=P + 2), dict(type=1, x=P + 1), dict(codes=P + 8), dict(scales=P + 8)):
        assert call(**bad) == fm.FMM_ERR_ARG, bad
    for bad in (dict(rows=(1 << 30) + 1), dict(cols=(1 << 22) + 1), dict(rows=1 << 20, cols=(1 << 14) + 1)):
        assert call(**bad) == fm.FMM_ERR_UNSUPPORTED, bad
    assert call(rows=0, x=None, codes=None) == call(cols=0, x=None, scales=None) == fm.FMM_OK
    if weight:
        assert call(count=-1) == fm.FMM_ERR_ARG and call(count=0, x=None) == fm.FMM_OK
        assert call(count=(1 << 22) + 1) == call(count=1 << 22, rows=1, cols=129) == fm.FMM_ERR_UNSUPPORTED


def test_dequantize_refuses(fm):
    def call(type=0, count=1, rows=4, cols=8, block=1, codes=P, scales=P, out=P):
        return status(fm, "fmm_f8_dequantize", type, count, rows, cols, block, codes, scales, out, None)

    for bad in (dict(type=7), dict(rows=-1), dict(cols=-2), dict(count=-1), dict(block=0), dict(block=64), dict(codes=None),
                dict(scales=None), dict(out=None), dict(codes=P + 4), dict(scales=P + 4), dict(out=P + 2)):
        assert call(**bad) == fm.FMM_ERR_ARG, bad
    assert call(rows=0) == call(cols=0) == call(count=0) == fm.FMM_OK


def test_matmul_refuses(fm):
    def call(rows=4, experts=2, N=5, K=6, type=0, a=P, sa=P, w=P, sw=P, off=P, bias=P, c=P, desc=True):
        d = fm.fmm_f8_desc(rows, experts, N, K, type)
        return status(fm, "fmm_f8_matmul", d if desc else None, a, sa, w, sw, off, bias, c, None)

    for bad in (dict(desc=False), dict(rows=-1), dict(N=-1), dict(K=-1), dict(experts=0), dict(experts=-1), dict(type=9),
                dict(a=None), dict(w=None), dict(a=P + 8), dict(w=P + 4), dict(sa=None), dict(sw=None), dict(sa=P + 8),
                dict(sw=P + 4), dict(off=None), dict(off=P + 2), dict(bias=P + 1), dict(c=None), dict(c=P + 2)):
        assert call(**bad) == fm.FMM_ERR_ARG, bad
    for bad in (dict(rows=(1 << 22) + 1), dict(N=(1 << 22) + 1), dict(K=(1 << 22) + 1), dict(experts=4097),
                dict(rows=1 << 20, N=1 << 14), dict(rows=1 << 20, K=1 << 14), dict(experts=128, N=1 << 14, K=(1 << 13) + 1)):
        assert call(**bad) == fm.FMM_ERR_UNSUPPORTED, bad
    assert call(rows=0, a=None, c=None) == call(N=0, w=None) == fm.FMM_OK


def test_backward_refuses(fm):
    need = fm.fmm_f8_linear_backward_scratch_size(fm.fmm_f8_desc(4, 2, 5, 6, 1))
    assert need > 0
    assert status(fm, "fmm_f8_linear_backward_scratch_size", fm.fmm_f8_desc(4, 2, 5, 6, 1), None) == fm.FMM_ERR_ARG
    n = ctypes.c_size_t()
    assert status(fm, "fmm_f8_linear_backward_scratch_size", fm.fmm_f8_desc(1 << 23, 2, 5, 6, 1), n) == fm.FMM_ERR_UNSUPPORTED

    def call(rows=4, experts=2, N=5, K=6, type=1, dy=P, a=P, sa=P, w=P, sw=P, off=P, dx=P, dw=P, db=P, scratch=P, nbytes=need,
             desc=True):
        d = fm.fmm_f8_desc(rows, experts, N, K, type)
        return status(fm, "fmm_f8_linear_backward", d if desc else None, dy, a, sa, w, sw, off, dx, dw, db, scratch, nbytes, None)

    for bad in (dict(desc=False), dict(rows=-1), dict(experts=0), dict(type=5), dict(dy=None), dict(dy=P + 1), dict(a=None),
                dict(a=P + 4), dict(sa=None), dict(w=None), dict(w=P + 1), dict(sw=None), dict(dx=P + 1), dict(dw=P + 1),
                dict(db=P + 2), dict(off=None)):
        assert call(**bad) == fm.FMM_ERR_ARG, bad
    for bad in (dict(scratch=None), dict(nbytes=need - 1), dict(scratch=P + 128)):
        assert call(**bad) == fm.FMM_ERR_WORKSPACE, bad
    for bad in (dict(rows=(1 << 22) + 1), dict(N=(1 << 22) + 1), dict(K=1 << 23), dict(experts=4097)):
        assert call(**bad) == fm.FMM_ERR_UNSUPPORTED, bad
    assert call(dx=None, dw=None, db=None, dy=None) == fm.FMM_OK


def test_clip_refuses(fm):
    need = fm.fmm_clip_scratch_size()

    def call(types=(0, 1), sizes=(5, 6), ins=(P, 2 * P), outs=(P, 2 * P), count=2, most=1.0, norm=P, scratch=P, nbytes=need,
             arrays=True):
        n = max(count, 0)
        t, s = (ctypes.c_int32 * n)(*types[:n]), (ctypes.c_int64 * n)(*sizes[:n])
        i, o = (ctypes.c_void_p * n)(*ins[:n]), (ctypes.c_void_p * n)(*outs[:n])
        return status(fm, "fmm_clip", t if arrays else None, s, i, o, count, most, norm, scratch, nbytes, None)

    for bad in (dict(count=-1), dict(most=-1.0), dict(most=float("nan")), dict(norm=None), dict(norm=P + 2), dict(arrays=False),
                dict(types=(0, 3)), dict(sizes=(-1, 6)), dict(ins=(None, P)), dict(outs=(P, None)), dict(ins=(P + 2, P)),
                dict(outs=(P, P + 1))):
        assert call(**bad) == fm.FMM_ERR_ARG, bad
    for bad in (dict(scratch=None), dict(scratch=P + 4), dict(nbytes=need - 1)):
        assert call(**bad) == fm.FMM_ERR_WORKSPACE, bad
    assert call(sizes=(1 << 42, 1)) == fm.FMM_ERR_UNSUPPORTED
    assert status(fm, "fmm_clip", None, None, None, None, 122881, 1.0, P, P, need, None) == fm.FMM_ERR_UNSUPPORTED


def test_kernels_are_named_and_each_is_tested(fm):
    """The kernels that sizes take, over a range of sizes, against the GPU tests' lists."""
    import test_gpu_f8_kernels as gpu
    products, gradients = set(), set()
    for rows in (1, 40, 300, 1300, 5000, 9000):
        for experts in (1, 3, 8, 50):
            for N in (8, 70, 400, 1500, 2600, 6000):
                for K in (9, 140, 1200, 2500, 5100):
                    for t in range(3):
                        d = fm.fmm_f8_desc(rows, experts, N, K, t)
                        products.add((fm.fmm_f8_matmul_kernel(d), t == 0))
                        gradients.update((fm.fmm_f8_linear_backward_kernel(d, *w), t == 0) for w in ((1, 1), (1, 0), (0, 1)))
    assert products == {(c[0], c[1] == "fp32") for c in gpu.PRODUCTS}
    assert gradients == {(c[0], c[1] == "fp32") for c in gpu.GRADIENTS}
    for kernel, t, rows, experts, N, K in gpu.PRODUCTS:
        assert fm.fmm_f8_matmul_kernel(fm.fmm_f8_desc(rows, max(1, experts), N, K, gpu.TYPE[t])) == kernel
    for kernel, t, rows, experts, N, K, want in gpu.GRADIENTS:
        assert fm.fmm_f8_linear_backward_kernel(fm.fmm_f8_desc(rows, max(1, experts), N, K, gpu.TYPE[t]), *want) == kernel
    for bad in ((-1, 1, 4, 4, 0), (4, 0, 4, 4, 0), (4, 1, 4, 1 << 23, 0), (4, 1, 4, 4, 3)):
        assert fm.fmm_f8_matmul_kernel(fm.fmm_f8_desc(*bad)) is None
        assert fm.fmm_f8_linear_backward_kernel(fm.fmm_f8_desc(*bad)) is None
    assert fm.fmm_f8_matmul_kernel(None) is None and fm.fmm_f8_linear_backward_kernel(None) is None


# ---- the torch wrappers -----------------------------------------------------------------
def _operands(device="cpu"):
    import torch
    from paper_2609_26077_amd import f8
    codes = lambda *s: torch.zeros(s, dtype=torch.uint8).view(f8.CODES)      # noqa: E731
    scales = lambda *s: torch.full(s, 127, dtype=torch.uint8).view(f8.SCALES)  # noqa: E731
    o = types.SimpleNamespace(a=codes(4, 256), sa=scales(4, 16), w=codes(6, 256), sw=scales(1, 16), gw=codes(3, 6, 256),
                              gsw=scales(3, 1, 16), off=torch.zeros(4, dtype=torch.int32),
                              dy=torch.zeros(4, 6, dtype=torch.bfloat16), x=torch.zeros(4, 200, dtype=torch.bfloat16))
    lin = f8.LinearF8(4, 6, 200, torch.bfloat16, device)
    return torch, f8, o, lin, f8.GroupedLinearF8(4, 3, 6, 200, torch.bfloat16, device)


def test_wrappers_refuse_types_and_shapes():
    torch, f8, o, lin, group = _operands()
    flat = torch.zeros(4 * 256 + 64, dtype=torch.uint8)
    at = -flat.data_ptr() % 16 + 8
    off16 = flat[at:at + 4 * 256].view(4, 256).view(f8.CODES)
    for call, what in ((lambda: f8.quantize(o.x.double()), "dtype"), (lambda: f8.quantize(o.x[0]), "matrix"),
                       (lambda: f8.quantize(o.x.t()), "contiguous"), (lambda: f8.quantize([1.0]), "torch.Tensor"),
                       (lambda: f8.quantize(o.x, codes=o.a.view(torch.uint8)), "dtype"),
                       (lambda: f8.quantize(o.x, scales=o.sa[:3]), "shape"),
                       (lambda: f8.quantize(o.x, codes=off16), "aligned"),
                       (lambda: f8.quantize_weight(o.x[0]), "matrix"), (lambda: f8.quantize_weight(None), "torch.Tensor"),
                       (lambda: f8.quantize_weight(o.x.t()), "contiguous"),
                       (lambda: f8.quantize_weight(o.x[None, None]), "matrix"),
                       (lambda: f8.dequantize(o.a, o.sa, 300), "shape"), (lambda: f8.dequantize(o.a, o.sa[:2], 200), "shape"),
                       (lambda: f8.dequantize(o.a, o.sa, 200, torch.int8), "dtype"),
                       (lambda: f8.dequantize(o.a, None, 200), "torch.Tensors"),
                       (lambda: f8.dequantize(o.a.view(torch.uint8), o.sa, 200), "dtype"),
                       (lambda: f8.dequantize(o.a, o.sa, 200, out=o.x), "dtype"),
                       (lambda: f8.LinearF8(4, 6, 200, torch.float64), "dtype"),
                       (lambda: lin.matmul(o.a[:, :200], o.sa, o.w, o.sw), "shape"),
                       (lambda: lin.matmul(o.a, o.sa, o.w[:5], o.sw), "shape"),
                       (lambda: lin.matmul(o.a, o.sa.view(torch.uint8), o.w, o.sw), "dtype"),
                       (lambda: lin.matmul(off16, o.sa, o.w, o.sw), "aligned"),
                       (lambda: lin.matmul(o.a, o.sa, o.w, o.sw, bias=o.dy[0]), "dtype"),
                       (lambda: lin.matmul(o.a, o.sa, o.w, o.sw, C=o.dy.float()), "dtype"),
                       (lambda: lin.matmul(o.a, o.sa, o.gw, o.gsw), "shape"),
                       (lambda: lin.backward(o.dy.t(), o.a, o.sa, o.w, o.sw), "shape"),
                       (lambda: lin.backward(o.dy, o.a, o.sa, o.w, o.sw[:, :1]), "shape"),
                       (lambda: group.matmul(o.a, o.sa, o.gw, o.gsw, None), "offsets"),
                       (lambda: group.matmul(o.a, o.sa, o.gw, o.gsw, o.off.long()), "dtype"),
                       (lambda: group.matmul(o.a, o.sa, o.gw, o.gsw, o.off[:3]), "shape"),
                       (lambda: group.matmul(o.a, o.sa, o.w, o.sw, o.off), "shape"),
                       (lambda: group.backward(o.dy, o.a, o.sa, o.gw, o.gsw, None), "offsets")):
        with pytest.raises(ValueError, match=what):
            call()


def test_clip_wrapper_refuses():
    import torch
    from paper_2609_26077_amd import grads
    a, b = torch.zeros(8), torch.zeros(4, 4)
    for call, what in ((lambda: grads.clip([], 1.0), "no tensors"), (lambda: grads.clip([a], -1.0), "max_norm"),
                       (lambda: grads.clip([a], float("nan")), "max_norm"), (lambda: grads.clip([a, 1.0], 1.0), "torch.Tensor"),
                       (lambda: grads.clip([b.t()[1:]], 1.0), "contiguous"), (lambda: grads.clip([a.double()], 1.0), "dtype"),
                       (lambda: grads.clip([a, a], 1.0), "overlap"), (lambda: grads.clip([a, a[3:5]], 1.0), "overlap"),
                       (lambda: grads.clip([a], 1.0, out=[]), "out"), (lambda: grads.clip([a], 1.0, out=[b]), "out"),
                       (lambda: grads.clip([a], 1.0, out=[a.half()]), "out"),
                       (lambda: grads.clip([a[:4], a[4:]], 1.0, out=[a[4:], a[:4]]), "overlap"),
                       (lambda: grads.clip([a[:4], a[4:]], 1.0, out=[b[0], b[0]]), "overlap"),
                       (lambda: grads.clip([a[:4]], 1.0, out=[a[1:5]]), "overlap"),
                       (lambda: grads.clip([a, b], 1.0), "device cpu"),
                       (lambda: grads.clip([a[:4], a[:4]], 1.0, out=[b[0], b[1]]), "device cpu"),
                       (lambda: grads.clip([a, b], 1.0, out=[a, b]), "device cpu")):
        with pytest.raises(ValueError, match=what):
            call()


def test_wrappers_refuse_other_devices():
    torch, f8, o, lin, group = _operands("cuda:0")
    with pytest.raises(ValueError, match="expected cuda:0"):
        lin.matmul(o.a, o.sa, o.w, o.sw)
    with pytest.raises(ValueError, match="expected cuda:0"):
        group.backward(o.dy, o.a, o.sa, o.gw, o.gsw, o.off)


@pytest.mark.parametrize("stream", [None, 0, 0x1230])
def test_wrappers_refuse_host_memory(monkeypatch, stream):
    """Tensors and objects that are all on the CPU: nothing reaches the library, whatever stream is named."""
    torch, f8, o, lin, group = _operands("cpu")
    from paper_2609_26077_amd import grads

    class NoLibrary:
        def __getattr__(self, name):
            raise AssertionError(f"{name} called")

    monkeypatch.setattr(f8, "_lib", NoLibrary())
    monkeypatch.setattr(grads, "_lib", NoLibrary())
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "device", lambda index: contextlib.nullcontext())
    monkeypatch.setattr(torch.cuda, "stream", lambda s: contextlib.nullcontext())
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle: types.SimpleNamespace(cuda_stream=handle))
    monkeypatch.setattr(torch.cuda, "default_stream", lambda index: types.SimpleNamespace(cuda_stream=0))
    for call in (lambda: f8.quantize(o.x, stream=stream), lambda: f8.quantize_weight(o.x, stream=stream),
                 lambda: f8.dequantize(o.a, o.sa, 200, stream=stream), lambda: lin.matmul(o.a, o.sa, o.w, o.sw, stream=stream),
                 lambda: lin.backward(o.dy, o.a, o.sa, o.w, o.sw, stream=stream),
                 lambda: group.matmul(o.a, o.sa, o.gw, o.gsw, o.off, stream=stream),
                 lambda: group.backward(o.dy, o.a, o.sa, o.gw, o.gsw, o.off, bias=True, stream=stream),
                 lambda: grads.clip([o.x], 1.0, stream=stream)):
        with pytest.raises(ValueError, match="device cpu"):
            call()


def test_objects_can_be_copied_and_pickled():
    _, f8, _, lin, group = _operands()
    for x in (lin, group):
        for y in (copy.deepcopy(x), pickle.loads(pickle.dumps(x))):
            assert type(y) is type(x) and y.dtype is x.dtype and y.device == x.device and bytes(y.desc) == bytes(x.desc)
            assert y.grad_scratch is not x.grad_scratch and not y.grad_scratch.blocks
