"""What the 8-bit linear layer refuses: the C entry points by their status, the
torch wrappers by an exception, in each case before any device work.  CPU
only; the addresses below are never read."""
import ctypes
import os

import numpy as np
import pytest

import q8_reference as ref

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


def test_pitch(fm):
    from paper_2609_26077_amd import q8
    for cols in (0, 1, 127, 128, 129, 4096, 131071):
        assert fm.fmm_q8_pitch(cols) == q8.pitch(cols) == ref.pitch(cols)
    assert fm.fmm_q8_pitch(-1) == -1


def test_quantize_refuses(fm):
    def call(type=0, rows=4, cols=8, x=P, codes=P, scales=P):
        return status(fm, "fmm_q8_quantize", type, rows, cols, x, codes, scales, None)

    for bad in (dict(type=3), dict(type=-1), dict(rows=-1), dict(cols=-1), dict(x=None), dict(codes=None),
                dict(scales=None), dict(x=P + 2), dict(type=1, x=P + 1), dict(codes=P + 8), dict(scales=P + 2)):
        assert call(**bad) == fm.FMM_ERR_ARG, bad
    assert call(rows=(1 << 30) + 1) == call(cols=(1 << 24) + 1) == fm.FMM_ERR_UNSUPPORTED
    assert call(rows=0, x=None, codes=None, scales=None) == fm.FMM_OK


def test_dequantize_refuses(fm):
    def call(type=0, rows=4, cols=8, group=0, codes=P, scales=P, out=P):
        return status(fm, "fmm_q8_dequantize", type, rows, cols, group, codes, scales, out, None)

    for bad in (dict(type=7), dict(rows=-1), dict(cols=-2), dict(group=64), dict(group=1), dict(codes=None),
                dict(scales=None), dict(out=None), dict(codes=P + 4), dict(out=P + 2)):
        assert call(**bad) == fm.FMM_ERR_ARG, bad
    assert call(rows=0) == call(cols=0) == fm.FMM_OK


def test_norm_refuses(fm):
    def call(rows=4, cols=8, type=0, eps=1e-6, x=P, res=P, gain=P, h=P, codes=P, scales=P, saved=P, saved_scales=P, rstd=P,
             desc=True):
        d = fm.fmm_norm_desc(rows, cols, type, eps)
        return status(fm, "fmm_rmsnorm_q8", d if desc else None, x, res, gain, h, codes, scales, saved, saved_scales, rstd,
                      None)

    for bad in (dict(desc=False), dict(rows=-1), dict(cols=-1), dict(type=4), dict(eps=-1.0), dict(eps=float("nan")),
                dict(eps=float("inf")), dict(x=None), dict(x=P + 1), dict(res=P + 2), dict(gain=P + 1), dict(h=P + 3),
                dict(codes=None), dict(codes=P + 4), dict(scales=None), dict(rstd=None), dict(rstd=P + 1), dict(saved=None),
                dict(saved_scales=None), dict(saved=P + 8)):
        assert call(**bad) == fm.FMM_ERR_ARG, bad
    assert call(cols=0) == fm.FMM_ERR_SHAPE
    assert call(rows=1 << 31) == fm.FMM_ERR_UNSUPPORTED
    assert call(cols=32769, h=P, res=P) == fm.FMM_ERR_UNSUPPORTED       # read twice: not in place
    assert call(rows=0, x=None, codes=None) == fm.FMM_OK


def test_norm_backward_refuses(fm):
    n = ctypes.c_size_t()
    d = fm.fmm_norm_desc(4000, 8, 0, 1e-6)
    assert status(fm, "fmm_rmsnorm_q8_backward_scratch_size", d, None) == fm.FMM_ERR_ARG
    assert status(fm, "fmm_rmsnorm_q8_backward_scratch_size", fm.fmm_norm_desc(4, 0, 0, 0.0), n) == fm.FMM_ERR_SHAPE
    need = fm.fmm_rmsnorm_q8_backward_scratch_size(d)
    assert need > 0

    def call(dy=P, dh=P, h=P, saved=None, saved_scales=None, rstd=P, gain=P, dx=2 * P, dgain=P, scratch=P, nbytes=need):
        return status(fm, "fmm_rmsnorm_q8_backward", d, dy, dh, h, saved, saved_scales, rstd, gain, dx, dgain, scratch,
                      nbytes, None)

    for bad in (dict(dy=None), dict(dy=P + 2), dict(dh=P + 1), dict(h=None), dict(h=None, saved=P),
                dict(h=None, saved=P + 8, saved_scales=P), dict(rstd=None), dict(gain=P + 2), dict(dx=None), dict(dx=P),
                dict(dgain=P + 2)):
        assert call(**bad) == fm.FMM_ERR_ARG, bad
    for bad in (dict(scratch=None), dict(nbytes=need - 1), dict(scratch=P + 8)):
        assert call(**bad) == fm.FMM_ERR_WORKSPACE, bad


def test_matmul_refuses(fm):
    def call(M=4, N=5, K=6, type=0, a=P, sa=P, w=P, sw=P, bias=P, c=P, desc=True):
        d = fm.fmm_q8_desc(M, N, K, type)
        return status(fm, "fmm_q8_matmul", d if desc else None, a, sa, w, sw, bias, c, None)

    for bad in (dict(desc=False), dict(M=-1), dict(N=-1), dict(K=-1), dict(type=9), dict(a=None), dict(w=None), dict(a=P + 8),
                dict(w=P + 4), dict(sa=None), dict(sw=None), dict(sa=P + 2), dict(bias=P + 1), dict(c=None), dict(c=P + 2)):
        assert call(**bad) == fm.FMM_ERR_ARG, bad
    for bad in (dict(K=131072), dict(M=(1 << 30) + 1), dict(N=1 << 31), dict(M=1 << 20, N=(1 << 17) + 1)):
        assert call(**bad) == fm.FMM_ERR_UNSUPPORTED, bad
    assert call(M=0, a=None, c=None) == call(N=0, w=None) == fm.FMM_OK


def test_linear_backward_refuses(fm):
    need = fm.fmm_q8_linear_backward_scratch_size(fm.fmm_q8_desc(4, 5, 6, 1))
    assert need > 0

    def call(M=4, N=5, K=6, type=1, dy=P, a=P, sa=P, w=P, sw=P, dx=P, dw=P, db=P, scratch=P, nbytes=need, desc=True):
        d = fm.fmm_q8_desc(M, N, K, type)
        return status(fm, "fmm_q8_linear_backward", d if desc else None, dy, a, sa, w, sw, dx, dw, db, scratch, nbytes, None)

    for bad in (dict(desc=False), dict(M=-1), dict(type=5), dict(dy=None), dict(dy=P + 8), dict(a=None), dict(a=P + 4),
                dict(sa=None), dict(w=None), dict(w=P + 1), dict(sw=None), dict(dx=P + 1), dict(dw=P + 1), dict(db=P + 2)):
        assert call(**bad) == fm.FMM_ERR_ARG, bad
    for bad in (dict(scratch=None), dict(nbytes=need - 1), dict(scratch=P + 128)):
        assert call(**bad) == fm.FMM_ERR_WORKSPACE, bad
    for bad in (dict(M=(1 << 22) + 1), dict(N=(1 << 22) + 1), dict(K=131072), dict(M=1 << 22, K=(1 << 12) + 1),
                dict(N=1 << 22, K=(1 << 12) + 1), dict(M=1 << 20, N=(1 << 14) + 1)):
        assert call(**bad) == fm.FMM_ERR_UNSUPPORTED, bad
    assert call(dx=None, dw=None, db=None, dy=None) == fm.FMM_OK


def test_kernels_are_named_and_each_is_tested(fm):
    """The kernels that sizes take, over a range of sizes, against the GPU tests' lists."""
    import test_gpu_q8 as gpu
    sizes = (1, 10, 40, 130, 520, 1030, 2100, 5000, 9000, 20001)
    types = {"fp32": 0, "bf16": 1, "fp16": 2}
    products, gradients = set(), set()
    for M in sizes:
        for N in sizes:
            for K in (1, 200, 560, 2100, 8200):
                products.add(fm.fmm_q8_matmul_kernel(fm.fmm_q8_desc(M, N, K, 1)))
                for t in range(3):
                    for want in ((1, 1), (1, 0), (0, 1)):
                        kernel, runs = fm.fmm_q8_linear_backward_kernel(fm.fmm_q8_desc(M, N, K, t), *want)
                        gradients.add(kernel)
                        assert all(1 <= r <= 16 for r in runs)
    assert products == {c[0] for c in gpu.PRODUCTS} and gradients == {c[1] for c in gpu.GRADIENTS}
    for kernel, M, N, K in gpu.PRODUCTS:
        assert fm.fmm_q8_matmul_kernel(fm.fmm_q8_desc(M, N, K, 1)) == kernel, (M, N, K)
    for t, kernel, runs, s, want in gpu.GRADIENTS:
        assert fm.fmm_q8_linear_backward_kernel(fm.fmm_q8_desc(*s, types[t]), *want) == (kernel, runs), (t, s)
    for bad in ((-1, 4, 4, 0), (4, 4, 131072, 0), (4, 4, 4, 3)):
        assert fm.fmm_q8_matmul_kernel(fm.fmm_q8_desc(*bad)) is None
        assert fm.fmm_q8_linear_backward_kernel(fm.fmm_q8_desc(*bad)) is None
    assert fm.fmm_q8_matmul_kernel(None) is None and fm.fmm_q8_linear_backward_kernel(None) is None


# ---- the torch wrappers -----------------------------------------------------------------
def _objects(device="cpu"):
    import torch
    from paper_2609_26077_amd import q8
    n = q8.RMSNormQ8(4, 200, torch.bfloat16, device=device)
    return torch, q8, n, q8.LinearQ8(4, 6, 200, torch.bfloat16, device=device)


def test_wrappers_refuse_types_and_shapes():
    torch, q8, n, lin = _objects()
    x = torch.zeros((4, 200), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="dtype"):
        q8.RMSNormQ8(4, 200, torch.float64)
    for call, what in ((lambda: q8.quantize(x.double()), "dtype"), (lambda: q8.quantize(x[0]), "matrix"),
                       (lambda: q8.quantize(x.t()), "contiguous"), (lambda: q8.quantize([1.0]), "torch.Tensor"),
                       (lambda: n.forward(x.float()), "dtype"), (lambda: n.forward(x[:3]), "shape"),
                       (lambda: n.forward(torch.zeros((200, 4), dtype=torch.bfloat16).t()), "contiguous"),
                       (lambda: n.forward(x, x[:, :8]), "shape"), (lambda: n.forward(x, gain=x[0].float()), "dtype"),
                       (lambda: n.forward(x, gain=x), "shape"), (lambda: n.forward(x, inplace=True), "inplace")):
        with pytest.raises(ValueError, match=what):
            call()
    r = torch.zeros(4)
    q, s = torch.zeros((4, 256), dtype=torch.int8), torch.zeros((4, 2))
    for call, what in ((lambda: n.backward(x, r), "exactly one"), (lambda: n.backward(x, r, h=x, saved=(q, s)), "exactly one"),
                       (lambda: n.backward(x, r[:3], h=x), "shape"), (lambda: n.backward(x.float(), r, h=x), "dtype"),
                       (lambda: n.backward(x, r, saved=(q[:, :200], s)), "shape"),
                       (lambda: n.backward(x, r, saved=(q, s[:, :1])), "shape"),
                       (lambda: n.backward(x, r, saved=(q.to(torch.uint8), s)), "dtype"),
                       (lambda: n.backward(x, r, h=x, dh=x.float()), "dtype")):
        with pytest.raises(ValueError, match=what):
            call()
    w, sw = torch.zeros((6, 256), dtype=torch.int8), torch.zeros(6)
    dy = torch.zeros((4, 6), dtype=torch.bfloat16)
    flat = torch.zeros(4 * 256 + 64, dtype=torch.int8)
    at = -flat.data_ptr() % 16 + 8
    off = flat[at:at + 4 * 256].view(4, 256)
    for call, what in ((lambda: lin.matmul(q[:, :200], r, w, sw), "shape"), (lambda: lin.matmul(q, r, w[:5], sw), "shape"),
                       (lambda: lin.matmul(q, r.double(), w, sw), "dtype"), (lambda: lin.matmul(off, r, w, sw), "aligned"),
                       (lambda: lin.matmul(q, r, w, sw, bias=dy[0]), "dtype"),
                       (lambda: lin.matmul(q, r, w, sw, C=dy.float()), "dtype"),
                       (lambda: lin.backward(dy.t(), q, r, w, sw), "shape"),
                       (lambda: lin.backward(dy, q, r, w, sw[:2]), "shape"),
                       (lambda: q8.dequantize(q, s, 300), "shape"), (lambda: q8.dequantize(q, r[:2], 200), "shape"),
                       (lambda: q8.dequantize(q, s, 200, torch.int8), "dtype")):
        with pytest.raises(ValueError, match=what):
            call()


def test_wrappers_refuse_other_devices():
    torch, q8, n, lin = _objects("cuda:0")
    x = torch.zeros((4, 200), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="expected cuda:0"):
        n.forward(x)
    with pytest.raises(ValueError, match="expected cuda:0"):
        lin.matmul(torch.zeros((4, 256), dtype=torch.int8), torch.zeros(4), torch.zeros((6, 256), dtype=torch.int8),
                   torch.zeros(6))


@pytest.mark.parametrize("stream", [None, 0, 0x1230])
def test_wrappers_refuse_host_memory(monkeypatch, stream):
    """Tensors and objects that are all on the CPU: nothing reaches the library, whatever stream is named."""
    import contextlib
    import types
    torch, q8, n, lin = _objects("cpu")

    class NoLibrary:
        def __getattr__(self, name):
            raise AssertionError(f"{name} called")

    monkeypatch.setattr(q8, "_lib", NoLibrary())
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "device", lambda index: contextlib.nullcontext())
    monkeypatch.setattr(torch.cuda, "stream", lambda s: contextlib.nullcontext())
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle: types.SimpleNamespace(cuda_stream=handle))
    monkeypatch.setattr(torch.cuda, "default_stream", lambda index: types.SimpleNamespace(cuda_stream=0))
    x, r = torch.zeros((4, 200), dtype=torch.bfloat16), torch.zeros(4)
    q, s = torch.zeros((4, 256), dtype=torch.int8), torch.zeros((4, 2))
    w, sw, dy = torch.zeros((6, 256), dtype=torch.int8), torch.zeros(6), torch.zeros((4, 6), dtype=torch.bfloat16)
    for call in (lambda: q8.quantize(x, stream=stream), lambda: q8.quantize(x, codes=q, scales=r, stream=stream),
                 lambda: q8.dequantize(q, r, 200, stream=stream),
                 lambda: q8.dequantize(q, s, 200, torch.bfloat16, out=x, stream=stream),
                 lambda: n.forward(x, x, checkpoint=True, stream=stream), lambda: n.backward(x, r, h=x, stream=stream),
                 lambda: n.backward(x, r, saved=(q, s), stream=stream), lambda: lin.matmul(q, r, w, sw, stream=stream),
                 lambda: lin.backward(dy, q, r, w, sw, bias=True, stream=stream)):
        with pytest.raises(ValueError, match="device cpu"):
            call()


def test_objects_can_be_copied_and_pickled():
    """As part of a model that is: the copy has the sizes, and a workspace of its own."""
    import copy
    import pickle
    _, q8, n, lin = _objects("cpu")
    for x in (n, lin):
        for y in (copy.deepcopy(x), pickle.loads(pickle.dumps(x))):
            assert type(y) is type(x) and y.dtype is x.dtype and y.device == x.device
            assert bytes(y.desc) == bytes(x.desc)
            held = [v for v in vars(y).values() if isinstance(v, q8._Workspace)]
            assert len(held) == 1 and held[0] not in vars(x).values() and not held[0].blocks


def test_handle_zero_is_the_default_stream(monkeypatch):
    """torch's own default stream has the handle 0, which a caller may pass on; torch
    makes of ExternalStream(0) a stream of its pool."""
    import contextlib
    import types

    import torch
    from paper_2609_26077_amd import q8
    made = []

    def stream(handle):
        return types.SimpleNamespace(cuda_stream=handle, device_index=0, device=torch.device("cuda:0"))

    monkeypatch.setattr(torch.cuda, "device", lambda index: contextlib.nullcontext())
    monkeypatch.setattr(torch.cuda, "stream", lambda s: (made.append(s), contextlib.nullcontext())[1])
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, *a, **k: stream(handle or 0x7700))
    monkeypatch.setattr(torch.cuda, "default_stream", lambda index: stream(0))
    for handle in (0, 0x1230):
        with q8._switched(0, handle) as used:
            assert used == handle and made[-1].cuda_stream == handle


def test_stream_of_another_device_is_refused(monkeypatch):
    """Its handle would be used with this device current, and its order is not that of the tensors."""
    import contextlib
    import types

    import torch
    from paper_2609_26077_amd import q8
    monkeypatch.setattr(torch.cuda, "device", lambda index: contextlib.nullcontext())
    monkeypatch.setattr(torch.cuda, "stream", lambda s: contextlib.nullcontext())
    other = types.SimpleNamespace(cuda_stream=0x1230, device_index=1, device=torch.device("cuda:1"))
    with pytest.raises(ValueError, match="stream: of device 1, expected 0"):
        with q8._switched(0, other):
            pass
    with q8._switched(1, other) as used:
        assert used == 0x1230


def test_backward_calls_that_may_overlap_share_no_workspace(monkeypatch):
    """Calls of one object on two streams may run at once, and a captured call beside
    later ones on its stream: what one adds up must not pass through the other's
    memory.  (What is allocated is held here, so that memory that is the same was handed
    out once.)"""
    import torch
    from paper_2609_26077_amd import q8
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    seen, held = [], []
    fresh = torch.empty

    class Library:
        def fmm_rmsnorm_q8_backward(self, *a):
            seen.append((a[-3], a[-2]))
            return 0
        fmm_q8_linear_backward = fmm_rmsnorm_q8_backward

    def empty(*shape, **kw):
        held.append(fresh(*shape, **kw))
        return held[-1]

    monkeypatch.setattr(q8, "_lib", Library())
    monkeypatch.setattr(q8, "_run", lambda device, stream, call, *tensors: call(stream))
    monkeypatch.setattr(torch, "empty", empty)
    n, lin = (q8.RMSNormQ8(2000, 300, torch.float32, device="cpu"), q8.LinearQ8(2000, 6, 300, torch.float32, device="cpu"))
    x, r = torch.zeros((2000, 300)), torch.zeros(2000)
    q, w, sw, dy = (torch.zeros((2000, 384), dtype=torch.int8), torch.zeros((6, 384), dtype=torch.int8), torch.zeros(6),
                    torch.zeros((2000, 6)))
    for call in (lambda s: n.backward(x, r, h=x, stream=s), lambda s: lin.backward(dy, q, r, w, sw, stream=s)):
        del seen[:]
        for stream, capturing in ((1, False), (2, False), (1, True), (2, True), (1, False)):
            monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing)
            call(stream)
        blocks, sizes = zip(*seen)
        assert all(blocks) and len(set(blocks[:4])) == 4 and len(set(sizes)) == 1 and sizes[0] > 0
        assert blocks[4] == blocks[0]                   # (a stream's calls are in its order: they may share)


def test_example_keeps_few_plans():
    """A prompt may have any number of tokens; what is kept for each must not pile up."""
    import torch
    from examples import q8_feedforward as example
    layer = example.FeedForward.__new__(example.FeedForward)
    layer.width, layer.hidden, layer.dtype, layer.device, layer.plans = 256, 512, torch.bfloat16, "cpu", {}
    one = layer._plan(1)
    for tokens in range(2, 100):
        assert layer._plan(tokens) is layer._plan(tokens) and layer._plan(1) is one
        assert len(layer.plans) <= example.KEPT_PLANS
    assert layer._plan(2)[0].rows == 2


# ---- the reference itself ------------------------------------------------------------------
def test_reference_gradient_is_the_losses_derivative():
    """The norm's gradient formula against central differences, binary64."""
    rng = np.random.default_rng(1)
    R, K, e = 5, 37, 1e-6
    h, gain, dy, dh = (rng.standard_normal(s) for s in ((R, K), (K,), (R, K), (R, K)))

    def loss(h, gain):
        return (dy * h * ((h ** 2).mean(axis=1, keepdims=True) + 1e-3) ** -0.5 * gain).sum() + (dh * h).sum()

    rstd = ((h ** 2).mean(axis=1) + 1e-3) ** -0.5
    dx, dg, terms, terms_g = ref.norm_gradient(h, rstd, dy, gain, dh)
    for i, j in ((0, 0), (4, 36), (2, 17)):
        d = np.zeros((R, K))
        d[i, j] = e
        assert abs((loss(h + d, gain) - loss(h - d, gain)) / (2 * e) - dx[i, j]) <= 1e-6 * (1 + terms[i, j])
        d = np.zeros(K)
        d[j] = e
        assert abs((loss(h, gain + d) - loss(h, gain - d)) / (2 * e) - dg[j]) <= 1e-6 * (1 + terms_g[j])


def test_reference_codes_are_nearest():
    rng = np.random.default_rng(2)
    x = (rng.standard_normal((20, 300)) * 10.0 ** rng.uniform(-6, 6, (20, 1))).astype(np.float32)
    q, s = ref.padded_codes(x)
    assert q.shape == (20, 384) and (q[:, 300:] == 0).all() and np.abs(q.astype(int)).max() == 127
    v = ref.values(q, s, 300)
    assert (np.abs(v - x) <= (0.5 + 2.0 ** -15) * s[:, None].astype(np.float64)).all()
    q, s = ref.checkpoint(x)
    v = ref.values(q, s, 300)
    assert (np.abs(v - x) <= (0.5 + 2.0 ** -15) * np.repeat(s, 128, axis=1)[:, :300]).all()
