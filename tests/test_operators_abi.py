"""The operators' C ABI without a GPU: bad arguments are refused before
anything asks for a device."""
import ctypes

import pytest

import paper_2609_18178_gb300 as apc
from paper_2609_18178_gb300.operators import _Distill, _Fp8Matrix

EINVAL, EALIGN, ERANGE = 1, 2, 3
AT = 1 << 40  # an address that nothing dereferences


def fp8(data=AT, scale=AT + (1 << 30), pitch=256, scale_pitch=64, fmt=0, block=1):
    return _Fp8Matrix(data, scale, pitch, scale_pitch, fmt, block)


def ref(x):
    return None if x is None else ctypes.addressof(x)


def quantize(x=AT + (1 << 32), rows=64, cols=256, pitch=256, dtype=1, q=None, qt=None):
    q = q or fp8()
    return apc.library().apc_quantize_fp8(x, rows, cols, pitch, dtype, ref(q), ref(qt), None)


def matmul(a=None, b=None, m=64, n=64, k=256, out=AT + (1 << 32), pitch=64, dtype=1):
    a, b = a or fp8(), b or fp8(AT + (1 << 33), AT + (1 << 34))
    return apc.library().apc_matmul_fp8(ref(a), ref(b), m, n, k, out, pitch, dtype, None)


def distill(what="loss_grad", loss=AT + (5 << 32), lse=AT + (6 << 32), g=AT + (7 << 32), d=AT + (8 << 32), dpitch=1000, **kw):
    f = dict(logits=AT, ids=AT + (1 << 32), teacher=AT + (2 << 32), teacher_lse=None, labels=None, rows=16, vocab=1000, k=8,
             pitch=1000, ids_pitch=8, teacher_pitch=8, dtype=1, ids_dtype=1, teacher_dtype=0, labels_dtype=0,
             temperature=1.0, kd_weight=1.0, label_weight=0.0)
    f.update(kw)
    s = _Distill(**f)
    lib = apc.library()
    if what == "loss":
        return lib.apc_distill_loss(ref(s), loss, lse, None)
    if what == "grad":
        return lib.apc_distill_grad(ref(s), lse, g, d, dpitch, None)
    return lib.apc_distill_loss_grad(ref(s), g, loss, lse, d, dpitch, None)


@pytest.mark.parametrize("want,kw", [
    (EINVAL, dict(x=None)),
    (EINVAL, dict(rows=-1)),
    (ERANGE, dict(cols=1 << 31)),
    (EINVAL, dict(dtype=3)),
    (EINVAL, dict(pitch=255)),
    (EALIGN, dict(x=AT + 1)),
    (ERANGE, dict(rows=1 << 30, pitch=1 << 40)),
    (EINVAL, dict(q=fp8(data=None))),
    (EINVAL, dict(q=fp8(scale=None))),
    (EALIGN, dict(q=fp8(data=AT + 8))),
    (EALIGN, dict(q=fp8(pitch=260))),
    (EALIGN, dict(q=fp8(scale=AT + 2))),
    (EINVAL, dict(q=fp8(scale_pitch=63))),
    (EINVAL, dict(q=fp8(fmt=2))),
    (EINVAL, dict(q=fp8(block=64))),
    (EINVAL, dict(q=fp8(), qt=fp8(AT + (1 << 33), AT + (1 << 34), block=128))),
    (EINVAL, dict(q=fp8(), qt=fp8(AT + (1 << 33), AT + (1 << 34), fmt=1))),
    (EINVAL, dict(q=fp8(), qt=fp8(AT + 4096, AT + (1 << 34)))),       # the two outputs overlap
    (EINVAL, dict(x=AT)),                                               # an output over the input
])
def test_quantize_refuses(want, kw):
    assert quantize(**kw) == want
    assert apc.library().apc_last_error()


@pytest.mark.parametrize("want,kw", [
    (EINVAL, dict(out=None)),
    (EINVAL, dict(m=-1)),
    (ERANGE, dict(n=1 << 31)),
    (EINVAL, dict(dtype=7)),
    (EINVAL, dict(pitch=63)),
    (EALIGN, dict(out=AT + (1 << 32) + 1)),
    (EALIGN, dict(dtype=0, out=AT + (1 << 32) + 2)),
    (EINVAL, dict(a=fp8(data=None))),
    (EALIGN, dict(b=fp8(AT + (1 << 33) + 4, AT + (1 << 34)))),
    (EALIGN, dict(b=fp8(AT + (1 << 33), AT + (1 << 34), pitch=264))),
    (EINVAL, dict(a=fp8(scale_pitch=10))),
    (EINVAL, dict(out=AT)),
])
def test_matmul_refuses(want, kw):
    assert matmul(**kw) == want


@pytest.mark.parametrize("want,kw", [
    (EINVAL, dict(logits=None)),
    (EINVAL, dict(ids=None)),
    (EINVAL, dict(loss=None)),
    (EINVAL, dict(lse=None)),
    (EINVAL, dict(g=None)),
    (EINVAL, dict(d=None)),
    (EINVAL, dict(vocab=0)),
    (EINVAL, dict(k=1025, ids_pitch=2000, teacher_pitch=2000)),
    (EINVAL, dict(k=-1)),
    (EINVAL, dict(dtype=3)),
    (EINVAL, dict(ids_dtype=2)),
    (EINVAL, dict(teacher_dtype=3)),
    (EINVAL, dict(labels=AT + (9 << 32), labels_dtype=2)),
    (EINVAL, dict(temperature=0.0)),
    (EINVAL, dict(temperature=-1.0)),
    (EINVAL, dict(temperature=float("nan"))),
    (EINVAL, dict(temperature=1e-39)),
    (EINVAL, dict(kd_weight=-1.0)),
    (EINVAL, dict(label_weight=float("inf"))),
    (EINVAL, dict(pitch=999)),
    (EINVAL, dict(dpitch=999)),
    (EALIGN, dict(ids=AT + (1 << 32) + 4)),
    (EALIGN, dict(lse=AT + (6 << 32) + 2)),
    (EINVAL, dict(d=AT + 64)),                    # the gradient over the logits, but not in their place
    (EINVAL, dict(d=AT, dpitch=1008)),
    (EINVAL, dict(loss=AT + (6 << 32) + 32)),     # over the statistics
    (EINVAL, dict(what="loss", loss=None)),
    (EINVAL, dict(what="grad", d=None)),
    (EINVAL, dict(what="grad", lse=None)),
])
def test_distill_refuses(want, kw):
    assert distill(**kw) == want


def test_empty_calls_need_no_device():
    none = fp8(data=None, scale=None)
    assert quantize(x=None, rows=0, q=none) == 0
    assert quantize(x=None, cols=0, q=none, qt=none) == 0
    assert matmul(a=none, m=0, out=None) == 0
    assert distill(logits=None, ids=None, teacher=None, loss=None, lse=None, g=None, d=None, rows=0) == 0


def test_struct_layout():
    assert ctypes.sizeof(_Fp8Matrix) == 40
    assert ctypes.sizeof(_Distill) == 5 * 8 + 6 * 8 + 4 * 4 + 3 * 8


@pytest.mark.parametrize("handle", [False, True])
def test_allocated_outputs_are_memory_of_the_stream_given(handle, monkeypatch):
    """Every output that a call allocates, on the CPU: the allocator is asked
    while the stream given is the current one."""
    import contextlib

    import torch

    from paper_2609_18178_gb300 import operators

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

    empty, lib = torch.empty, type("Library", (), {"__getattr__": lambda self, name: lambda *a: 0})()

    def recorded(*a, **kw):
        asked.append(list(current))
        return empty(*a, **kw)

    # what the checks take for the current device is the CPU's
    monkeypatch.setattr(operators, "_current_device", lambda: -1)
    monkeypatch.setattr(operators, "_lib", lib)
    monkeypatch.setattr(apc, "_lib", lib)
    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    monkeypatch.setattr(torch.cuda, "ExternalStream", Stream)
    monkeypatch.setattr(torch.cuda, "stream", use)
    x, f8 = torch.zeros(4, 32), torch.zeros(4, 32).to(torch.float8_e4m3fn)
    scale, ids, g = torch.ones(1, 4), torch.zeros(4, 2, dtype=torch.int64), torch.ones(4)
    monkeypatch.setattr(torch, "empty", recorded)
    s = 0x1230 if handle else Stream()
    for call, outputs in ((lambda: apc.quantize_fp8(x, transposed=True, stream=s), 4),
                          (lambda: apc.matmul_fp8(f8, scale, f8, scale, stream=s), 1),
                          (lambda: apc.distill_loss(x, ids, x[:, :2], stream=s), 2),
                          (lambda: apc.distill_grad(x, ids, x[:, :2], g[None], g, stream=s), 1),
                          (lambda: apc.distill_loss_grad(x, ids, x[:, :2], g, stream=s), 3),
                          (lambda: apc._out(None, 4, x, s), 1)):  # digests and counts
        del asked[:]
        call()
        assert asked == [[0x1230]] * outputs


def test_star_import_needs_no_torch():
    """The package without the operators works where torch cannot be imported."""
    import os
    import subprocess
    import sys

    root = os.path.dirname(os.path.dirname(os.path.abspath(apc.__file__)))
    code = "import sys; sys.modules['torch'] = None\nfrom paper_2609_18178_gb300 import *\nprint(DEFAULT_HPARAMS['lr'], commit_step)"
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    assert "3e-04" in r.stdout or "0.0003" in r.stdout
    assert apc.quantize_fp8.__module__.endswith("operators")


@pytest.mark.parametrize("kw,fine", [
    (dict(kd_weight=0.0, label_weight=1.0, temperature=1e20), True),    # the square scales the teacher's part alone
    (dict(kd_weight=0.0, label_weight=3e38, temperature=2.0), True),
    (dict(kd_weight=1.0, label_weight=0.0, temperature=1e20), False),
    (dict(kd_weight=3e38, label_weight=0.0, temperature=2.0), False),
    (dict(kd_weight=float("nan"), label_weight=0.0), False),
    (dict(kd_weight=0.0, label_weight=-1.0), False),
])
def test_distill_weights(kw, fine):
    """Refused for a weight or not: without a device a call ends later all the same."""
    distill(labels=AT + (9 << 32), **kw)
    assert (b"weight" in apc.library().apc_last_error()) == (not fine)


@pytest.mark.parametrize("d,dpitch,pitch,apart", [
    (AT + 2000, 2000, 2000, True),          # two halves of one buffer
    (AT + 2000 + 4000 * 3, 2000, 2000, True),   # the second half, some rows further on
    (AT - 4000 * 2 + 2000, 2000, 2000, True),   # and some rows before
    (AT + 1998, 2000, 2000, False),         # one element into the logits
    (AT + 2002, 2000, 2000, False),         # and into their next row
    (AT + 2000, 2008, 2000, False),         # rows that do not keep step
    (AT - 4000 * 2 + 2002, 2000, 2000, False),
])
def test_columns_of_one_buffer_do_not_overlap(d, dpitch, pitch, apart):
    """Logits and gradient side by side in a buffer: 16 rows of 1000 16-bit elements."""
    distill(d=d, dpitch=dpitch, pitch=pitch)
    assert (b"overlaps" in apc.library().apc_last_error()) == (not apart)
