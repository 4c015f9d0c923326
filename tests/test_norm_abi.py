"""The C ABI of the norms and of the clipped step without a GPU: bad arguments
are refused before anything asks for a device."""
import contextlib
import ctypes

import pytest

import paper_2609_18178_gb300 as apc
from paper_2609_18178_gb300 import operators
from paper_2609_18178_gb300.operators import _Fp8Matrix



class _Norm(ctypes.Structure):
    """apc_norm, field by field."""
    _fields_ = [(n, ctypes.c_void_p) for n in ("x", "residual", "weight", "sum")] + \
               [(n, ctypes.c_int64) for n in ("rows", "cols", "pitch", "residual_pitch", "sum_pitch")] + \
               [("dtype", ctypes.c_uint32), ("weight_dtype", ctypes.c_uint32), ("eps", ctypes.c_double)]


class _NormGrad(ctypes.Structure):
    """apc_norm_grad, field by field."""
    _fields_ = [(n, ctypes.c_void_p) for n in ("dout", "x", "weight", "dresidual", "rstd")] + \
               [(n, ctypes.c_int64) for n in ("rows", "cols", "dout_pitch", "pitch", "dresidual_pitch")] + \
               [("dtype", ctypes.c_uint32), ("weight_dtype", ctypes.c_uint32)]


EINVAL, EALIGN, ERANGE, ECUDA = 1, 2, 3, 4
AT = 1 << 40  # an address that nothing dereferences
GB = 1 << 32


def fp8(data=AT + 8 * GB, scale=AT + 9 * GB, pitch=256, scale_pitch=64, fmt=0, block=1):
    return _Fp8Matrix(data, scale, pitch, scale_pitch, fmt, block)


def ref(x):
    return None if x is None else ctypes.addressof(x)


def norm(what="same", out=AT + 5 * GB, opitch=256, rstd=AT + 6 * GB, q=None, qt=None, **kw):
    f = dict(x=AT, residual=AT + GB, weight=AT + 2 * GB, sum=AT + 3 * GB, rows=64, cols=256, pitch=256, residual_pitch=256,
             sum_pitch=256, dtype=1, weight_dtype=0, eps=1e-6)
    f.update(kw)
    d = _Norm(**f)
    if what == "same":
        return apc.library().apc_rms_norm(ref(d), out, opitch, rstd, None)
    q = q or fp8()
    return apc.library().apc_rms_norm_fp8(ref(d), ref(q), ref(qt), rstd, None)


def grad(dx=AT + 5 * GB, xpitch=256, dw=AT + 6 * GB, dwtype=0, work=AT + 7 * GB, **kw):
    f = dict(dout=AT, x=AT + GB, weight=AT + 2 * GB, dresidual=AT + 3 * GB, rstd=AT + 4 * GB, rows=9000, cols=256, dout_pitch=256,
             pitch=256, dresidual_pitch=256, dtype=1, weight_dtype=0)
    f.update(kw)
    d = _NormGrad(**f)
    return apc.library().apc_rms_norm_grad(ref(d), dx, xpitch, dw, dwtype, work, None)


@pytest.mark.parametrize("want,kw", [
    (EINVAL, dict(x=None)),
    (EINVAL, dict(weight=None)),
    (EINVAL, dict(sum=None)),                     # a residual without a place for the sum
    (EINVAL, dict(residual=None)),                # a place for the sum without a residual
    (EINVAL, dict(out=None)),
    (EINVAL, dict(rstd=None)),
    (EINVAL, dict(rows=-1)),
    (ERANGE, dict(cols=1 << 31)),
    (EINVAL, dict(dtype=3)),
    (EINVAL, dict(weight_dtype=3)),
    (EINVAL, dict(eps=0.0)),
    (EINVAL, dict(eps=-1e-6)),
    (EINVAL, dict(eps=1e-21)),
    (EINVAL, dict(eps=float("nan"))),
    (EINVAL, dict(eps=float("inf"))),
    (EINVAL, dict(eps=1e39)),
    (EINVAL, dict(pitch=255)),
    (EINVAL, dict(residual_pitch=255)),
    (EINVAL, dict(sum_pitch=255)),
    (EINVAL, dict(opitch=255)),
    (EALIGN, dict(x=AT + 1)),
    (EALIGN, dict(weight=AT + 2 * GB + 2)),       # fp32
    (EALIGN, dict(rstd=AT + 6 * GB + 2)),
    (ERANGE, dict(rows=1 << 30, pitch=1 << 40)),
    (EINVAL, dict(out=AT)),                       # the output over the input
    (EINVAL, dict(out=AT + 3 * GB)),              # and over the sum
    (EINVAL, dict(sum=AT + 2)),                   # the sum over x, but not in its place
    (EINVAL, dict(sum=AT, sum_pitch=264)),
    (EINVAL, dict(rstd=AT + 2 * GB)),             # over the weight
    (EINVAL, dict(what="fp8", q=fp8(data=None))),
    (EINVAL, dict(what="fp8", q=fp8(block=128))),
    (EINVAL, dict(what="fp8", q=fp8(fmt=2))),
    (EALIGN, dict(what="fp8", q=fp8(data=AT + 8 * GB + 8))),
    (EINVAL, dict(what="fp8", q=fp8(scale_pitch=63))),
    (EINVAL, dict(what="fp8", qt=fp8(AT + 10 * GB, AT + 11 * GB, scale_pitch=256, fmt=1))),
    (EINVAL, dict(what="fp8", qt=fp8(AT + 10 * GB, AT + 11 * GB, scale_pitch=256, block=128))),
    (EINVAL, dict(what="fp8", qt=fp8(AT + 8 * GB + 4096, AT + 11 * GB, scale_pitch=256))),  # the two outputs overlap
])
def test_norm_refuses(want, kw):
    assert norm(**kw) == want
    assert apc.library().apc_last_error()


@pytest.mark.parametrize("kw", [dict(), dict(sum=AT), dict(sum=AT + GB), dict(residual=None, sum=None), dict(x=AT + GB),
                                dict(what="fp8", qt=fp8(AT + 10 * GB, AT + 11 * GB, scale_pitch=256))])
def test_norm_takes(kw):
    """Good arguments get as far as the question whose memory this is, which no device answers here."""
    assert norm(**kw) in (EINVAL, ECUDA)
    assert not any(w in apc.library().apc_last_error() for w in (b"overlaps", b"null", b"pitch"))


@pytest.mark.parametrize("want,kw", [
    (EINVAL, dict(dout=None)),
    (EINVAL, dict(x=None)),
    (EINVAL, dict(weight=None)),
    (EINVAL, dict(rstd=None)),
    (EINVAL, dict(dx=None)),
    (EINVAL, dict(work=None)),
    (EINVAL, dict(rows=-1)),
    (ERANGE, dict(rows=1 << 31)),
    (EINVAL, dict(dtype=3)),
    (EINVAL, dict(weight_dtype=9)),
    (EINVAL, dict(dwtype=3)),
    (EINVAL, dict(dout_pitch=255)),
    (EINVAL, dict(dresidual_pitch=255)),
    (EINVAL, dict(xpitch=255)),
    (EALIGN, dict(dout=AT + 1)),
    (EALIGN, dict(dw=AT + 6 * GB + 2)),
    (EALIGN, dict(work=AT + 7 * GB + 2)),
    (EINVAL, dict(dx=AT + GB)),                   # the gradient over x
    (EINVAL, dict(dx=AT + 2)),                    # over dout, but not in its place
    (EINVAL, dict(dx=AT, xpitch=264)),
    (EINVAL, dict(dw=AT + 7 * GB + 1024)),        # inside the workspace
    (EINVAL, dict(work=AT + 3 * GB)),
])
def test_grad_refuses(want, kw):
    assert grad(**kw) == want
    assert apc.library().apc_last_error()


@pytest.mark.parametrize("kw", [dict(), dict(dx=AT), dict(dx=AT + 3 * GB), dict(dresidual=None), dict(dw=None, work=None),
                                dict(rows=4, work=None)])
def test_grad_takes(kw):
    assert grad(**kw) in (EINVAL, ECUDA)
    assert not any(w in apc.library().apc_last_error() for w in (b"overlaps", b"null", b"pitch"))


def test_empty_calls_need_no_device():
    none = dict(x=None, residual=None, weight=None, sum=None)
    assert norm(rows=0, out=None, rstd=None, **none) == 0
    assert norm(what="fp8", rows=0, rstd=None, q=fp8(None, None), qt=fp8(None, None), **none) == 0
    assert norm(cols=0, out=None, rstd=None, **none) == 0
    assert grad(dout=None, x=None, weight=None, dresidual=None, rstd=None, rows=0, dx=None, dw=None, work=None) == 0
    assert grad(dout=None, x=None, weight=None, dresidual=None, rstd=None, cols=0, dx=None, dw=None, work=None) == 0


def test_grad_workspace():
    f = apc.library().apc_rms_norm_grad_workspace
    assert f(0, 4096) == f(4, 4096) == f(64, 4096) == f(-1, 5) == f(5, 1 << 31) == 0
    assert f(65, 4096) == 65 * 4096 * 4 and f(8192, 4096) == 304 * 4096 * 4
    assert f(9000, 256) == 8 * 304 * 256 * 4


# ---- the gradients' norm and the clipped step

def buffers(n=1000, count=3, dtype=1, slot=0, at=AT, step=GB):
    arr = (apc._Buffer * max(count, 1))()
    for k in range(count):
        arr[k] = apc._Buffer(None if at is None else at + k * step, n, 0, dtype, slot)
    return arr, count


def grad_norm(slots=1, work=AT + 20 * GB, out=AT + 21 * GB, **kw):
    arr, count = buffers(**kw)
    return apc.library().apc_grad_norm(arr, count, slots, work, None, out)


@pytest.mark.parametrize("want,kw", [
    (EINVAL, dict(at=None)),
    (EINVAL, dict(out=None)),
    (EINVAL, dict(slots=0)),
    (EINVAL, dict(slots=9)),
    (EINVAL, dict(slot=1)),
    (EINVAL, dict(dtype=3)),
    (EALIGN, dict(at=AT + 1)),
    (EALIGN, dict(dtype=0, at=AT + 2)),
    (EALIGN, dict(out=AT + 21 * GB + 2)),
    (EALIGN, dict(work=AT + 20 * GB + 4)),
    (EINVAL, dict(out=AT + 64)),                  # inside a buffer
    (EINVAL, dict(work=AT + 64)),
    (EINVAL, dict(work=AT + 21 * GB - 8)),        # the workspace over the output
    (ERANGE, dict(n=1 << 62)),
])
def test_grad_norm_refuses(want, kw):
    assert grad_norm(**kw) == want
    assert apc.library().apc_last_error()


def test_other_buffer_lists_take_no_fp16():
    arr, n = buffers(dtype=apc.F16)
    lib = apc.library()
    assert lib.apc_digest(arr, n, 1, None, AT + 21 * GB) == EINVAL and lib.apc_count_nonzero(arr, n, 1, None, AT + 21 * GB) == EINVAL


def test_grad_norm_workspace():
    f = apc.library().apc_grad_norm_workspace
    for n, count, want in ((1000, 3, 0), (2048 * 4096, 1, 0), (2048 * 4096 + 1, 1, apc.GRAD_NORM_WORKSPACE), (1, 1600, 0),
                           (1, 1601, apc.GRAD_NORM_WORKSPACE), (0, 5000, 0), (1 << 41, 1, apc.GRAD_NORM_WORKSPACE)):
        arr, k = buffers(n=n, count=count)
        assert f(arr, k) == want
    assert f(None, 0) == 0


def commit(norm=AT + 30 * GB, max_norm=1.0, flags=0, bf16=False, step=1, out=AT + 31 * GB):
    hp = apc._hp(None)
    at = [AT + k * GB for k in range(5)]
    lib = apc.library()
    if bf16:
        arr = (apc._TensorBF16 * 1)(apc._TensorBF16(*at[:4], 1000, 0))
        return lib.apc_commit_step_bf16_clipped(arr, 1, ctypes.byref(hp), step, flags, norm, max_norm, None, out)
    arr = (apc._Tensor * 1)(apc._Tensor(*at, 1000, 0))
    return lib.apc_commit_step_clipped(arr, 1, ctypes.byref(hp), step, flags, norm, max_norm, None, out)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("want,kw", [
    (EINVAL, dict(norm=None)),
    (EALIGN, dict(norm=AT + 30 * GB + 2)),
    (EINVAL, dict(max_norm=0.0)),
    (EINVAL, dict(max_norm=-1.0)),
    (EINVAL, dict(max_norm=1e-60)),
    (EINVAL, dict(max_norm=1e39)),
    (EINVAL, dict(max_norm=float("nan"))),
    (EINVAL, dict(max_norm=float("inf"))),
    (EINVAL, dict(norm=AT + 64)),                 # inside the parameters, which are written
    (EINVAL, dict(norm=AT + 31 * GB + 8)),        # inside the digests
    (EINVAL, dict(norm=AT + 3 * GB, flags=1)),    # inside gradients that are zeroed
    (EINVAL, dict(flags=2)),
    (EINVAL, dict(step=0)),
])
def test_clipped_commit_refuses(bf16, want, kw):
    assert commit(bf16=bf16, **kw) == want
    assert apc.library().apc_last_error()


def test_packed_structures_are_the_header_s():
    """What the binding packs has the fields' places of the structures."""
    for pack, like, values in ((operators._pack_norm, _Norm, list(range(1, 12)) + [0.5]),
                               (operators._pack_norm_grad, _NormGrad, list(range(1, 13))),
                               (operators._pack_fp8, _Fp8Matrix, list(range(1, 7)))):
        assert pack(*values) == bytes(like(*values)) and len(pack(*values)) == ctypes.sizeof(like)


# ---- the binding

@pytest.fixture
def on_cpu(monkeypatch):
    """The binding with the CPU for the current device and a library that takes everything."""
    real = apc.library()

    class Library:
        def __getattr__(self, name):
            if "workspace" in name:
                return getattr(real, name)
            return lambda *a: self.calls.append((name, a)) or 0

    lib = Library()
    lib.calls = []
    monkeypatch.setattr(operators, "_current_device", lambda: -1)
    monkeypatch.setattr(operators, "_raw_stream", lambda device: 0)
    monkeypatch.setattr(operators, "_lib", lib)
    monkeypatch.setattr(apc, "_lib", lib)
    monkeypatch.setattr(apc, "_ptr", lambda x, size=None: 0 if x is None else x if isinstance(x, int) else x.data_ptr())
    monkeypatch.setattr(apc, "_stream", lambda s: 0 if s is None else s if isinstance(s, int) else s.cuda_stream)
    return lib


def test_binding_checks_its_tensors(on_cpu):
    import torch
    x, w = torch.zeros(4, 32), torch.ones(32)
    bad = [lambda: apc.rms_norm(x, w[:31]), lambda: apc.rms_norm(x[0], w), lambda: apc.rms_norm(x.double(), w),
           lambda: apc.rms_norm(x, w.double()), lambda: apc.rms_norm(x.t(), torch.ones(4)), lambda: apc.rms_norm(x, w, residual=x[:3]),
           lambda: apc.rms_norm(x, w, residual=x.bfloat16()), lambda: apc.rms_norm(x, w, sum=x), lambda: apc.rms_norm(x, w, out=x.half()),
           lambda: apc.rms_norm(x, w, rstd=torch.ones(5)), lambda: apc.rms_norm_fp8(x, w, dtype=torch.int8),
           lambda: apc.rms_norm_fp8(x, w, out=(x, x)), lambda: apc.rms_norm_fp8(x, w, out=(x,)),
           lambda: apc.rms_norm_grad(x, x, w, torch.ones(3)), lambda: apc.rms_norm_grad(x.half(), x, w, torch.ones(4)),
           lambda: apc.rms_norm_grad(x, x, w, torch.ones(4), dweight=w, weight_grad=False),
           lambda: apc.rms_norm_grad(x, x, w, torch.ones(4), dweight=w[:3]),
           lambda: apc.grad_norm([x.double()]), lambda: apc.grad_norm([5]), lambda: apc.grad_norm([x], out=torch.ones(1).half()),
           lambda: apc.grad_norm([apc.BufferEntry(x, 0, n=129)]), lambda: apc.grad_norm([apc.BufferEntry(x, 0, dtype=apc.BF16)]),
           lambda: apc.grad_norm(apc.PreparedTable("buffers", None, 0, None, [])),
           lambda: apc.grad_norm([x], workspace=torch.zeros(3)),
           lambda: apc._clip(None, 1.0), lambda: apc._clip(w[:1], None), lambda: apc._clip(w[:2], 1.0), lambda: apc._clip(w[:1].half(), 1.0)]
    for k, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            print("call", k)
    assert not on_cpu.calls


def test_workspaces_that_are_refused_and_taken(on_cpu):
    import torch
    x, w = torch.zeros(3000, 400), torch.ones(400)
    n = operators.rms_norm_grad_workspace(3000, 400)
    for workspace in (torch.zeros(2, n + 8)[:, :n], torch.zeros(2 * n, 2)[:, 0], torch.zeros(n, 2)[:, 0], torch.zeros(n - 1),
                      torch.zeros(n).int(), torch.zeros(n).double()):
        with pytest.raises(ValueError):
            apc.rms_norm_grad(x, x, w, torch.ones(3000), workspace=workspace)
    assert not on_cpu.calls
    for workspace in (torch.zeros(n), torch.zeros(n + 5), torch.zeros(2, n)):
        apc.rms_norm_grad(x, x, w, torch.ones(3000), workspace=workspace)
        assert on_cpu.calls[-1][1][5] == workspace.data_ptr()


def test_every_operator_is_the_package_s_too():
    assert all(getattr(apc, n) is getattr(operators, n) for n in operators.__all__)
    assert apc.rms_norm_grad_workspace(3000, 400) == 8 * 304 * 400  # as rms_norm_grad's documentation names it


def test_allocated_outputs_are_memory_of_the_stream_given(on_cpu, monkeypatch):
    import torch

    class Stream:
        cuda_stream = 0x1230

        def __init__(self, handle=0x1230, device=None):
            assert handle == 0x1230

    current, asked = [], []

    @contextlib.contextmanager
    def use(stream):
        current.append(stream.cuda_stream)
        yield
        current.pop()

    empty = torch.empty
    held = []
    monkeypatch.setattr(operators, "_raw_alloc", lambda size, stream: asked.append([stream]) or held.append(size) or 1 << 40)
    monkeypatch.setattr(operators, "_raw_free", lambda at: held.pop())
    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    monkeypatch.setattr(torch.cuda, "ExternalStream", Stream)
    monkeypatch.setattr(torch.cuda, "stream", use)
    x, w = torch.zeros(400, 32), torch.ones(32)
    big = torch.zeros(3_000, 400)
    monkeypatch.setattr(torch, "empty", lambda *a, **kw: asked.append(list(current)) or empty(*a, **kw))
    for s in (0x1230, Stream()):
        for call, outputs in ((lambda: apc.rms_norm(x, w, residual=x, stream=s), 3),
                              (lambda: apc.rms_norm_fp8(x, w, residual=x, transposed=True, stream=s), 6),
                              (lambda: apc.rms_norm_grad(x, x, w, torch.ones(400), stream=s), 2),
                              (lambda: apc.rms_norm_grad(big, big, torch.ones(400), torch.ones(3000), stream=s), 3),
                              (lambda: apc.grad_norm([x], stream=s), 1),
                              (lambda: apc.grad_norm([x] * 1700, stream=s), 2)):
            del asked[:]
            call()
            assert asked == [[0x1230]] * outputs and not held
    # a call that is refused gives its workspace back
    monkeypatch.setattr(operators, "_check", lambda status: 1 / 0)
    with pytest.raises(ZeroDivisionError):
        apc.rms_norm_grad(big, big, torch.ones(400), torch.ones(3000), stream=0x1230)
    assert not held


def test_a_commit_table_gives_its_gradients(on_cpu):
    import torch
    t = [apc.TensorEntry(*(torch.zeros(n) for _ in range(3)), *(torch.zeros(n, dtype=torch.bfloat16) for _ in range(2)), 0) for n in (5, 70)]
    for grads in (t, apc.prepare_table(t), [e.g for e in t], apc.prepare_grads(t), [apc.BufferEntry(e.g, 0) for e in t]):
        arr, n, _ = apc._grads(grads)
        assert n == 2 and [(arr[k].data, arr[k].n, arr[k].dtype, arr[k].slot) for k in range(2)] == [(e.g.data_ptr(), e.count(), apc.BF16, 0) for e in t]
    p = apc.prepare_table(t)
    assert apc._grads(p)[0] is apc._grads(p)[0] and p.work == 0
