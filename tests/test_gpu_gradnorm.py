"""The gradients' norm against 64-bit sums, and the clipped step against the
step's fixed order of binary32 operations, on the GPU.

Bounds: a tile's sum of squares passes at most 16 multiply-adds, 2 additions and
5 more between lanes, each off by 2^-24 of a partial sum of non-negative terms,
and tiles add exactly: 23 * 2^-24, of which a square root leaves half, and one
rounding: below 2^-20 in all."""
import math
import os

import numpy as np
import pytest
import torch

import oracle
import paper_2609_18178_gb300 as apc

pytestmark = pytest.mark.gpu
REL = 2.0 ** -20
TYPES = [torch.bfloat16, torch.float16, torch.float32]


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def exact(tensors):
    """Squares of fp32 values are exact in 64 bits; fsum rounds their sum once."""
    return math.sqrt(math.fsum(math.fsum((t.double().cpu().numpy().ravel() ** 2).tolist()) for t in tensors))


def placed(x, off):
    """x, `off` elements behind an allocation's start, between NaNs."""
    room = torch.full((x.numel() + 64,), math.nan, device="cuda").to(x.dtype)
    v = room[off:off + x.numel()]
    v.copy_(x)
    return v


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 2, 7, 8, 9, 255, 1023, 1024, 1025, 2047, 2048, 2049, 4097, 100_003, 9_000_001])
def test_norm_at_every_alignment(dtype, n):
    x = torch.randn(n, generator=gen(n), device="cuda").to(dtype)
    want = exact([x])
    bits = set()
    for off in range(0, 16 // x.element_size()):
        got = apc.grad_norm([placed(x, off)])
        assert got.dtype == torch.float32 and got.shape == (1,)
        bits.add(got.item())
    assert len(bits) == 1  # the address does not count
    assert abs(bits.pop() - want) <= REL * want


@pytest.mark.parametrize("count", [1, 24, 25, 240, 241, 1100, 1600, 1601, 3333])
@pytest.mark.parametrize("size", [300, 6000, 60_000])
def test_norm_of_many_buffers(count, size):
    sizes = torch.randint(1, size, (count,), generator=torch.Generator().manual_seed(count)).tolist()
    whole = torch.randn(sum(sizes), generator=gen(3), device="cuda").mul_(1e-3).bfloat16()
    parts = list(whole.split(sizes))
    a = apc.grad_norm(parts)
    want = exact([whole])
    assert abs(a.item() - want) <= REL * want
    assert torch.equal(a, apc.grad_norm(parts[::-1]))  # nor does their order
    assert torch.equal(a, apc.grad_norm(apc.prepare_grads(parts)))


def test_norm_does_not_depend_on_the_grid(monkeypatch):
    x = [torch.randn(n, generator=gen(n), device="cuda").to(t) for n, t in
         ((3_000_001, torch.bfloat16), (70_001, torch.float32), (1_234_567, torch.float16), (5, torch.float32))] * 400
    a = apc.grad_norm(x)
    for limit in ("1", "7", "151"):
        monkeypatch.setenv("APC_GRID_LIMIT", limit)
        assert torch.equal(a, apc.grad_norm(x))
    monkeypatch.delenv("APC_GRID_LIMIT")
    apc.set_reserved_sms(40)
    try:
        assert torch.equal(a, apc.grad_norm(x))
    finally:
        apc.set_reserved_sms(0)
    assert abs(a.item() - 20 * exact(x[:4])) <= 2 * REL * a.item()


def test_norm_by_slots_and_types():
    a = torch.randn(10_007, generator=gen(1), device="cuda")
    b, c = (a * 3).bfloat16(), (a * 0.5).half()
    e = apc.BufferEntry
    got = apc.grad_norm([e(a, 2), e(b, 0), e(c, 2), e(b, 7), e(a, 0, n=5000), e(a, 3, n=0)], num_slots=8)
    want = [exact([b, a[:5000]]), 0.0, exact([a, c]), 0.0, 0.0, 0.0, 0.0, exact([b])]
    for g, w in zip(got.tolist(), want):
        assert abs(g - w) <= REL * w


@pytest.mark.parametrize("value", [2.0 ** -149, 2.0 ** -133, 1e-38, 1e-30, 1e-23, 2.0 ** -50, 2.0 ** 60, 1e20, 1e30, 3.3e38])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_norm_of_tiny_and_huge_values(value, dtype):
    for n in (1, 1537, 9001):
        x = torch.full((n,), value, dtype=torch.float64).to(dtype)
        x[::3] *= -0.5
        want = exact([x])
        got = apc.grad_norm([x.cuda()]).item()
        if want > 3.4028235e38:
            assert got == math.inf
        else:
            assert abs(got - want) <= REL * want + 2.0 ** -149
    # beside ordinary values, in the same tile and in another
    y = torch.randn(4000, generator=gen(9), device="cuda").to(dtype)
    y[17] = value
    want = exact([y, y[:100]])
    assert abs(apc.grad_norm([y, y[:100].clone()]).item() - want) <= REL * want or want > 3.4e38


def test_norm_of_half_at_its_ends():
    for v in (2.0 ** -24, 65504.0):
        x = torch.full((5001,), v, dtype=torch.float16, device="cuda")
        want = exact([x])
        assert abs(apc.grad_norm([x]).item() - want) <= REL * want


@pytest.mark.parametrize("dtype", TYPES)
def test_norm_of_values_that_are_not_finite(dtype):
    x = torch.randn(9001, generator=gen(4), device="cuda").to(dtype)
    for at in (0, 2047, 9000):
        y = x.clone()
        y[at] = -math.inf
        assert apc.grad_norm([x, y]).item() == math.inf
        y[77] = math.nan
        assert math.isnan(apc.grad_norm([x, y]).item())
        e = apc.BufferEntry
        two = apc.grad_norm([e(x, 0), e(y, 1)], num_slots=2).tolist()
        assert math.isfinite(two[0]) and math.isnan(two[1])


def test_norm_of_nothing():
    out = torch.full((3,), 7.0, device="cuda")
    assert apc.grad_norm([], num_slots=3, out=out).tolist() == [0.0, 0.0, 0.0]
    z = torch.zeros(5000, device="cuda")
    z[::2] = -0.0
    assert apc.grad_norm([z, z[:0]]).item() == 0.0


def test_norm_on_another_stream_and_in_a_graph():
    x = [torch.randn(n, generator=gen(n), device="cuda").bfloat16() for n in (500_000, 33, 70_001)]
    want = apc.grad_norm(x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = apc.grad_norm(x, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got, want)
    table, out = apc.prepare_grads(x), torch.empty(1, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        apc.grad_norm(table, out=out)
    for k in range(3):
        for t in x:
            t.mul_(2)
        g.replay()
        assert out.item() == want.item() * 2 ** (k + 1)


# ---- the clipped step

def clipped(p, m, v, g16, c, h):
    """The step's fixed order in binary32 on the gradient times c."""
    f = np.float32
    g = (g16.astype(np.uint32) << 16).view(f) * f(c)
    m2 = h[0] * m + h[1] * g
    v2 = h[2] * v + h[3] * (g * g)
    den = np.sqrt(v2) * h[7] + h[4]
    return p * h[5] - h[6] * (m2 / den), m2, v2


def widen(x16):
    return (x16.astype(np.uint32) << 16).view(np.float32)


def inputs(sizes, seed, odd, bf16):
    """Host arrays and device tensors of a table, its buffers `odd` elements behind each other."""
    rng = np.random.default_rng(seed)
    host, rows, goff = [], [], (1 << 32) - 1000
    for n in sizes:
        p, m = (rng.standard_normal(n) * 0.02).astype(np.float32), (rng.standard_normal(n) * 1e-4).astype(np.float32)
        v = ((rng.standard_normal(n) * 1e-3) ** 2).astype(np.float32)
        g = oracle.bf16_rne((rng.standard_normal(n) * 1e-2).astype(np.float32))
        g[rng.random(n) < 0.05] = 0
        if bf16:
            p, m, v = (oracle.bf16_rne(x) for x in (p, m, v))
        host.append((p, m, v, g, goff))

        def put(x, off):
            t = torch.from_numpy(x.view(np.int16) if x.dtype == np.uint16 else x).cuda()
            room = torch.zeros(n + 32, dtype=t.dtype, device="cuda")
            room[off:off + n] = t
            return room[off:off + n]

        o = [odd * k % 7 for k in (1, 2, 3, 4, 5)]
        bufs = [put(x, k) for x, k in zip((p, m, v, g), o)]
        if bf16:
            rows.append(apc.TensorEntryBF16(*bufs, goff))
        else:
            rows.append(apc.TensorEntry(*bufs, put(np.zeros(n, np.uint16), o[4]), goff))
        goff += n
    return host, rows


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("odd", [0, 1, 3])
@pytest.mark.parametrize("zero", [False, True])
@pytest.mark.parametrize("norm,max_norm", [(2.7, 1.0), (0.5, 1.0), (1.0, 1.0), (123.456, 0.3), (1e-3, 1e-4)])
def test_clipped_step_bit_for_bit(bf16, odd, zero, norm, max_norm):
    sizes = [1, 31, 5000, 20_557, 100_003] + [257] * (20 if odd else 100)
    host, rows = inputs(sizes, 11, odd, bf16)
    h = oracle.resolve_hparams(oracle.DEFAULT_HP, 7)
    f = np.float32
    c = f(max_norm) / f(norm) if f(norm) > f(max_norm) else f(1)
    out = (apc.commit_step_bf16 if bf16 else apc.commit_step)(
        rows, 7, grad_norm=torch.tensor([norm], device="cuda"), max_norm=max_norm, zero_grad=zero)
    total = [0] * (3 if bf16 else 4)
    for (p, m, v, g, goff), r in zip(host, rows):
        if bf16:
            want = [oracle.bf16_rne(x) for x in clipped(widen(p), widen(m), widen(v), g, c, h)]
            digests = [oracle.digest_u16(x, goff) for x in want]
        else:
            want = list(clipped(p, m, v, g, c, h))
            digests = [oracle.digest_f32(x, goff) for x in want]
            want.append(oracle.bf16_rne(want[0]))
            digests.append(oracle.digest_u16(want[3], goff))
        for x, name in zip(want, "pmvw"):
            got = getattr(r, name).cpu().numpy()
            assert np.array_equal(got.view(x.dtype) if x.dtype == np.uint16 else got, x), name
        assert np.array_equal(r.g.cpu().numpy().view(np.uint16), np.zeros_like(g) if zero else g)
        total = [(a + b) & apc.MASK64 for a, b in zip(total, digests)]
    assert apc.digests_to_host(out) == total


@pytest.mark.parametrize("bf16", [False, True])
def test_clipping_that_does_not_apply_is_the_plain_step(bf16):
    step = apc.commit_step_bf16 if bf16 else apc.commit_step
    _, a = inputs([70_001, 33], 5, 1, bf16)
    _, b = inputs([70_001, 33], 5, 1, bf16)
    x = step(a, 3, grad_norm=torch.tensor([0.9], device="cuda"), max_norm=0.95)
    assert torch.equal(x, step(b, 3))


@pytest.mark.parametrize("bf16", [False, True])
def test_clipping_by_a_norm_that_is_not_finite(bf16):
    step = apc.commit_step_bf16 if bf16 else apc.commit_step
    _, a = inputs([9001], 5, 0, bf16)
    _, b = inputs([9001], 5, 0, bf16)
    b[0].g.zero_()
    x = step(a, 3, grad_norm=torch.tensor([math.inf], device="cuda"), max_norm=1.0)
    assert torch.equal(x, step(b, 3))  # every gradient times 0 (a -0 enters no moment)
    step(a, 4, grad_norm=torch.tensor([math.nan], device="cuda"), max_norm=1.0)
    m = a[0].m.view(torch.bfloat16) if bf16 else a[0].m
    assert m.isnan().all()


def test_norm_and_step_together_on_one_stream(monkeypatch):
    """As a job runs them: the norm of the table's gradients, then the step, without a wait between; replicas agree."""
    results = []
    for odd, limit in ((0, None), (3, None), (1, "5")):
        if limit:
            monkeypatch.setenv("APC_GRID_LIMIT", limit)
        host, rows = inputs([40_001, 7, 3000] + [129] * 500, 21, odd, False)
        table = apc.prepare_table(rows)
        norm = apc.grad_norm(table)
        results.append((norm.item(), apc.digests_to_host(apc.commit_step(table, 2, grad_norm=norm, max_norm=0.25))))
        assert torch.equal(norm, apc.grad_norm(rows))
    assert results[0] == results[1] == results[2]
    want = exact([torch.from_numpy(widen(g)) for *_, g, _ in host])
    assert abs(results[0][0] - want) <= REL * want and want > 0.25


def test_norm_and_step_in_a_graph():
    host, rows = inputs([40_001, 129], 22, 0, False)
    _, ref = inputs([40_001, 129], 22, 0, False)
    table, norm, out = apc.prepare_table(rows), torch.empty(1, device="cuda"), torch.empty(4, dtype=torch.int64, device="cuda")
    work = torch.empty(apc.GRAD_NORM_WORKSPACE, dtype=torch.uint8, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        apc.grad_norm(table, out=norm, workspace=work)
        apc.commit_step(table, 2, out=out, grad_norm=norm, max_norm=0.25)
    g.replay()
    n = apc.grad_norm(ref)
    assert torch.equal(out, apc.commit_step(ref, 2, grad_norm=n, max_norm=0.25)) and torch.equal(n, norm)
    g.replay()
    assert torch.equal(out, apc.commit_step(ref, 2, grad_norm=n, max_norm=0.25))
