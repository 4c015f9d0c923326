"""The operators around the output head against plain implementations in 64
bits, on the GPU, at the sizes, types, strides and masks where they can go
wrong.  Bounds are forward rounding bounds of the operators' definitions."""
import math

import numpy as np
import pytest
import torch

import paper_2609_18178_gb300 as apc

pytestmark = pytest.mark.gpu

E4M3, E5M2 = torch.float8_e4m3fn, torch.float8_e5m2
LARGEST = {E4M3: 448.0, E5M2: 57344.0}
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}  # half an ulp of 1
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def strided(x, extra=0, offset=0):
    """x in memory with rows `extra` elements further apart, `offset` elements
    behind an allocation's start; what surrounds it is NaN."""
    r, c = x.shape
    room = torch.full((offset + r * (c + extra) + 64,), math.nan, device="cuda").to(x.dtype)
    v = room[offset:offset + r * (c + extra)].view(r, c + extra)[:, :c]
    v.copy_(x)
    return v


# ---- quantization

def ref_scales(x, block, fmt):
    """The definition, in exact arithmetic on the host (float64 holds every product)."""
    x = x.double().cpu().numpy()
    r, c = x.shape
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    out = np.ones((-(-c // 128), -(-r // block)), np.float64)
    for i in range(out.shape[0]):
        for j in range(out.shape[1]):
            m = a[j * block:(j + 1) * block, i * 128:(i + 1) * 128].max()
            if m > 0:
                e = -126
                while LARGEST[fmt] * 2.0 ** e < m:
                    e += 1
                out[i, j] = 2.0 ** e
    return torch.from_numpy(out)


def spread(s, r, c, block):
    return s.t().repeat_interleave(block, 0)[:r].repeat_interleave(128, 1)[:, :c]


def check_quantized(x, q, s, block, fmt):
    want = ref_scales(x, block, fmt)
    assert torch.equal(s.double().cpu(), want)
    y = (x.double().cpu() / spread(want, *x.shape, block)).float()  # exact but where it rounds to zero
    y = y.to(fmt)
    got, want = q.cpu().float(), y.float()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(got.nan_to_num(nan=7.0), want.nan_to_num(nan=7.0))


def awkward(r, c, dtype, seed):
    """Magnitudes over the type's range, block by block, with zeros, zero
    blocks and signs of both kinds."""
    g = gen(seed)
    top = {torch.float32: 126, torch.bfloat16: 126, torch.float16: 15}[dtype]
    x = torch.randn(r, c, generator=g, device="cuda")
    e = torch.randint(-top, top - 4, (-(-r // 5), -(-c // 96)), generator=g, device="cuda").float()
    x = x * torch.exp2(e).repeat_interleave(5, 0)[:r].repeat_interleave(96, 1)[:, :c]
    x[torch.rand(r, c, generator=g, device="cuda") < 0.05] = 0
    x[r // 2:r // 2 + 2] = 0
    return x.to(dtype)


@pytest.mark.parametrize("r,c", [(1, 1), (1, 128), (1, 4096), (3, 127), (5, 129), (127, 640), (128, 128), (129, 257),
                                 (300, 1000), (1, 5000), (2500, 3), (257, 384)])
@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_quantize(r, c, block, dtype):
    x = awkward(r, c, dtype, r * 7 + c)
    for fmt in (E4M3, E5M2):
        q, s = apc.quantize_fp8(x, block_rows=block, dtype=fmt)
        check_quantized(x, q, s, block, fmt)
        q2, s2, qt, st = apc.quantize_fp8(x, block_rows=block, dtype=fmt, transposed=True)
        assert torch.equal(q2.view(torch.uint8), q.view(torch.uint8)) and torch.equal(s2, s)
        check_quantized(x.t(), qt, st, block, fmt)


@pytest.mark.parametrize("extra,offset", [(0, 1), (1, 0), (3, 5), (8, 0), (8, 8), (64, 3)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_quantize_strides_and_surroundings(extra, offset, dtype):
    r, c = 150, 333
    x = awkward(r, c, dtype, 5)
    v = strided(x, extra, offset)
    for block in (1, 128):
        room = [torch.full((r, 352), 0x55, dtype=torch.uint8, device="cuda").view(E4M3),
                torch.full((3, 160), -5.0, device="cuda"),
                torch.full((c, 176), 0x55, dtype=torch.uint8, device="cuda").view(E4M3),
                torch.full((2, 400), -5.0, device="cuda")]
        n, nt = -(-r // block), -(-c // block)
        out = (room[0][:, :c], room[1][:, :n], room[2][:, :r], room[3][:, :nt])
        got = apc.quantize_fp8(v, block_rows=block, transposed=True, out=out)
        check_quantized(x, got[0], got[1], block, E4M3)
        check_quantized(x.t(), got[2], got[3], block, E4M3)
        assert (room[0].view(torch.uint8)[:, c:] == 0x55).all() and (room[2].view(torch.uint8)[:, r:] == 0x55).all()
        assert (room[1][:, n:] == -5).all() and (room[3][:, nt:] == -5).all()


@pytest.mark.parametrize("fmt", [E4M3, E5M2])
@pytest.mark.parametrize("block", [1, 128])
def test_quantize_non_finite(fmt, block):
    """Infinities and NaNs stay out of the scale and do not become numbers."""
    x = torch.randn(130, 260, generator=gen(3), device="cuda")
    x[0, 5], x[0, 200], x[7, 130] = math.inf, -math.inf, math.nan
    x[9] = math.inf       # nothing finite in the row
    x[10] = 0.0
    x[10, 3] = math.nan   # nothing but zeros beside it
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        y = x.to(dtype)
        q, s, qt, st = apc.quantize_fp8(y, block_rows=block, dtype=fmt, transposed=True)
        for data, scale, src in ((q, s, y), (qt, st, y.t())):
            assert torch.equal(scale.double().cpu(), ref_scales(src, block, fmt))
            v, w = data.float(), src.float()
            assert torch.equal(torch.isfinite(v), torch.isfinite(w))
            if fmt == E5M2:
                assert torch.equal(v[torch.isinf(w)], w[torch.isinf(w)])
            fine = torch.isfinite(w)
            n = (w / spread(scale, *w.shape, block)).to(fmt).float()
            assert torch.equal(v[fine], n[fine])


@pytest.mark.parametrize("fmt", [E4M3, E5M2])
def test_quantize_every_16_bit_value(fmt):
    """Every finite bf16 and fp16 value, each in a block with the value that sets the scale."""
    for dtype in (torch.bfloat16, torch.float16):
        v = torch.arange(1 << 16, device="cuda").to(torch.int32).to(torch.int16).view(dtype)
        v = v[torch.isfinite(v.float())]
        for lead in (1.0, 447.0, 449.0, 60000.0):
            n = -(-v.numel() // 127)
            x = torch.zeros(n, 128, device="cuda", dtype=dtype)
            x[:, 0] = lead
            flat = torch.nn.functional.pad(v, (0, n * 127 - v.numel()))
            x[:, 1:] = flat.view(n, 127)
            q, s = apc.quantize_fp8(x, dtype=fmt)
            a = x.float().abs().amax(1)
            assert ((s[0] * LARGEST[fmt] >= a) & (s[0] * (LARGEST[fmt] / 2) < a)).all()
            assert torch.equal(q.float(), (x.double() / s[0].double()[:, None]).float().to(fmt).float())


def test_quantize_empty_and_refusals():
    for r, c in ((0, 5), (5, 0), (0, 0)):
        x = torch.empty(r, c, device="cuda")
        q, s = apc.quantize_fp8(x)
        assert q.shape == (r, c) and s.shape == (-(-c // 128), r)
    x = torch.randn(8, 64, device="cuda")
    with pytest.raises(ValueError):
        apc.quantize_fp8(x.double())
    with pytest.raises(ValueError):
        apc.quantize_fp8(x.cpu())
    with pytest.raises(ValueError):
        apc.quantize_fp8(x.t())  # not row-major
    with pytest.raises(ValueError):
        apc.quantize_fp8(x, block_rows=64)
    with pytest.raises(ValueError):
        apc.quantize_fp8(x, dtype=torch.float16)
    with pytest.raises(ValueError):
        apc.quantize_fp8(x, out=(torch.empty(8, 63, dtype=E4M3, device="cuda"), torch.empty(1, 8, device="cuda")))
    with pytest.raises(apc.ApcError) as e:  # rows not 16 bytes apart
        apc.quantize_fp8(x, out=(torch.empty(8, 72, dtype=E4M3, device="cuda")[:, :64], torch.empty(1, 8, device="cuda")))
    assert e.value.status == 2


# ---- product

def operand(r, k, block, fmt, seed, scale_extra=0):
    """Random 8-bit values with scales that are no powers of two."""
    g = gen(seed)
    q = torch.randn(r, k, generator=g, device="cuda").mul_(40).to(fmt)
    room = torch.empty(r, -(-k // 16) * 16 + 32, dtype=fmt, device="cuda")
    room.view(torch.uint8).fill_(0x7f)  # NaN behind the last column
    room[:, :k] = q
    n = -(-r // block)
    s = torch.rand(-(-k // 128), n + scale_extra, generator=g, device="cuda").add_(0.5).mul_(0.01)
    return room[:, :k], s[:, :n]


def ref_matmul(a, sa, ba, b, sb, bb):
    x = a.double() * spread(sa.double(), *a.shape, ba)
    y = b.double() * spread(sb.double(), *b.shape, bb)
    return x @ y.t(), x.abs() @ y.abs().t()


def check_matmul(out, ref, size, k):
    """|error| <= half an ulp of the result in out's type + the rounding of a
    sum of k products in 32 bits whose terms need not be rounded to nearest."""
    blocks = -(-k // 128)
    bound = UNIT[out.dtype] * ref.abs() + size * (2.0 ** -23 * (128 + blocks + 4)) * (1 + UNIT[out.dtype]) + TINY[out.dtype]
    assert out.shape == ref.shape
    worst = ((out.double() - ref).abs() / bound).max().item() if out.numel() else 0.0
    assert worst <= 1.0, worst


@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 16, 128), (1, 4096, 4096), (2, 129, 100), (7, 1000, 300), (16, 256, 2048),
                                   (17, 130, 129), (31, 65, 127), (33, 257, 640), (64, 4097, 256), (65, 500, 1111),
                                   (100, 128, 5000), (128, 128, 128), (129, 255, 384), (200, 700, 90), (256, 256, 1024),
                                   (300, 513, 777), (513, 300, 257), (1000, 1, 1000), (1025, 513, 130), (2100, 2050, 16),
                                   (2100, 2050, 1111), (5000, 600, 640)])
@pytest.mark.parametrize("ba,bb", [(1, 128), (1, 1), (128, 128)])
def test_matmul(m, n, k, ba, bb):
    a, sa = operand(m, k, ba, E4M3, m + k)
    b, sb = operand(n, k, bb, E4M3, n + 3 * k, 3)
    ref, size = ref_matmul(a, sa, ba, b, sb, bb)
    for dtype in (torch.bfloat16, torch.float32):
        out = apc.matmul_fp8(a, sa, b, sb, out_dtype=dtype)
        check_matmul(out, ref, size, k)
    assert apc.device_status() == 0


@pytest.mark.parametrize("m,n,k", [(2100, 2050, 1111), (1500, 5000, 512), (5000, 600, 640), (600, 3001, 9000), (4100, 4100, 130)])
@pytest.mark.parametrize("bb", [1, 128])
@pytest.mark.parametrize("fa,fb", [(E4M3, E4M3), (E5M2, E4M3)])
def test_matmul_power_of_two_scales(m, n, k, bb, fa, fb):
    """Large products of what quantization makes, whose scales may be the tensor
    cores' own; and with single scales that are not powers of two, 0, or beyond
    their range, from the first tile on or from a later one."""
    x = torch.randn(m, k, generator=gen(1), device="cuda") * torch.exp2(torch.randint(-9, 9, (m, 1), generator=gen(2), device="cuda").float())
    y = torch.randn(n, k, generator=gen(3), device="cuda") * torch.exp2(torch.randint(-9, 9, (n, 1), generator=gen(4), device="cuda").float())
    a, sa = apc.quantize_fp8(x, dtype=fa)
    b, sb = apc.quantize_fp8(y, block_rows=bb, dtype=fb)
    ref, size = ref_matmul(a, sa, 1, b, sb, bb)
    for dtype in (torch.bfloat16, torch.float32):
        check_matmul(apc.matmul_fp8(a, sa, b, sb, out_dtype=dtype), ref, size, k)
    blocks = sa.shape[0]
    for at, value in ((0, 3.0), (m - 1, 0.75), (m // 2, 0.0), (m - 1, 2.0 ** -130)):
        odd = sa.clone()
        odd[blocks - 1, at] = value
        ref, size = ref_matmul(a, odd, 1, b, sb, bb)
        check_matmul(apc.matmul_fp8(a, odd, b, sb), ref, size, k)
    odd = sb.clone()
    odd[0, odd.shape[1] - 1] = 1.5
    ref, size = ref_matmul(a, sa, 1, b, odd, bb)
    check_matmul(apc.matmul_fp8(a, sa, b, odd, out_dtype=torch.float32), ref, size, k)
    assert apc.device_status() == 0


@pytest.mark.parametrize("m,n,k", [(1, 300, 500), (40, 200, 1000), (300, 400, 500), (700, 600, 1300)])
@pytest.mark.parametrize("fa,fb", [(E4M3, E5M2), (E5M2, E4M3), (E5M2, E5M2)])
def test_matmul_formats(m, n, k, fa, fb):
    a, sa = operand(m, k, 1, fa, 1)
    b, sb = operand(n, k, 128, fb, 2)
    ref, size = ref_matmul(a, sa, 1, b, sb, 128)
    check_matmul(apc.matmul_fp8(a, sa, b, sb, out_dtype=torch.float16), ref, size, k)
    assert apc.device_status() == 0


@pytest.mark.parametrize("m,n,k", [(3, 77, 200), (50, 333, 128), (333, 129, 260), (520, 777, 130)])
@pytest.mark.parametrize("extra,offset", [(0, 1), (1, 0), (3, 5), (8, 8), (16, 0)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_matmul_out_strides(m, n, k, extra, offset, dtype):
    """Any row pitch and start of out; what surrounds it stays."""
    a, sa = operand(m, k, 1, E4M3, 1)
    b, sb = operand(n, k, 128, E4M3, 2)
    room = torch.full((offset + m * (n + extra) + 64,), 3.0, dtype=dtype, device="cuda")
    out = room[offset:offset + m * (n + extra)].view(m, n + extra)
    apc.matmul_fp8(a, sa, b, sb, out=out[:, :n])
    ref, size = ref_matmul(a, sa, 1, b, sb, 128)
    check_matmul(out[:, :n], ref, size, k)
    assert (out[:, n:] == 3).all() and (room[:offset] == 3).all() and (room[offset + m * (n + extra):] == 3).all()
    assert apc.device_status() == 0


def test_matmul_equals_quantized_product_with_infinities_kept_apart():
    """A NaN in one row of a stays in that row of out; one of b in its column."""
    a, sa = operand(40, 300, 1, E4M3, 1)
    b, sb = operand(70, 300, 1, E4M3, 2)
    a.view(torch.uint8)[5, 100] = 0x7f
    b.view(torch.uint8)[9, 299] = 0xff
    out = apc.matmul_fp8(a, sa, b, sb)
    bad = torch.isnan(out)
    want = torch.zeros_like(bad)
    want[5], want[:, 9] = True, True
    assert torch.equal(bad, want)


def test_matmul_repeats_and_does_not_depend_on_the_grid(monkeypatch):
    for m, n, k in ((1, 1000, 4096), (48, 640, 5000), (700, 900, 1500)):
        a, sa = operand(m, k, 1, E4M3, 1)
        b, sb = operand(n, k, 128, E4M3, 2)
        first = apc.matmul_fp8(a, sa, b, sb, out_dtype=torch.float32)
        assert torch.equal(first, apc.matmul_fp8(a, sa, b, sb, out_dtype=torch.float32))
        monkeypatch.setenv("APC_GRID_LIMIT", "7")
        assert torch.equal(first, apc.matmul_fp8(a, sa, b, sb, out_dtype=torch.float32))
        monkeypatch.delenv("APC_GRID_LIMIT")
    assert apc.device_status() == 0


def test_matmul_empty_and_refusals():
    a, sa = operand(5, 200, 1, E4M3, 1)
    b, sb = operand(9, 200, 128, E4M3, 2)
    assert apc.matmul_fp8(a[:0], sa[:, :0], b, sb).shape == (0, 9)
    zero = apc.matmul_fp8(a[:, :0], sa[:0], b[:, :0], sb[:0])
    assert zero.shape == (5, 9) and not zero.any()
    with pytest.raises(ValueError):
        apc.matmul_fp8(a, sa, b[:, :100], sb[:1])
    with pytest.raises(ValueError):
        apc.matmul_fp8(a, sa[:1], b, sb)
    with pytest.raises(ValueError):
        apc.matmul_fp8(a, sa, b, sb, out=torch.empty(5, 8, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(ValueError):
        apc.matmul_fp8(a.float(), sa, b, sb)
    with pytest.raises(apc.ApcError) as e:
        apc.matmul_fp8(a[:, 1:].view(torch.uint8).view(E4M3), sa, b[:, 1:], sb)  # starts off a 16-byte boundary
    assert e.value.status == 2


# ---- distillation

def teacher_of(rows, vocab, k, seed, dtype=torch.float32, wide=True, ragged=True):
    g = gen(seed)
    ids = torch.rand(rows, vocab, generator=g, device="cuda").topk(min(k, vocab), 1).indices
    if k > vocab:
        ids = torch.randint(0, vocab, (rows, k), generator=g, device="cuda")
    u = torch.randn(rows, k, generator=g, device="cuda").mul_(2).to(dtype)
    if ragged:
        ids[torch.rand(rows, k, generator=g, device="cuda") < 0.1] = -1
        ids[torch.rand(rows, k, generator=g, device="cuda") < 0.05] = vocab
        u[torch.rand(rows, k, generator=g, device="cuda") < 0.1] = -math.inf
        u[(ids < 0) | (ids >= vocab)] = math.nan
    return ids.to(torch.int64 if wide else torch.int32), u


def ref_distill(z, ids, u, g, tau, wk, wl, lse_t=None, labels=None):
    """The definition row by row in float64; also what bounds need: the sums
    of magnitudes that the gradient adds up."""
    z, u = z.double().cpu(), u.double().cpu() / tau
    ids = ids.cpu().long()
    rows, v = z.shape
    loss, lse = torch.zeros(rows).double(), torch.zeros(2, rows).double()
    d, size, p_sum = torch.zeros_like(z), torch.zeros_like(z), torch.zeros(rows).double()
    for t in range(rows):
        lse[0, t], lse[1, t] = torch.logsumexp(z[t] / tau, 0), torch.logsumexp(z[t], 0)
        ok = (ids[t] >= 0) & (ids[t] < v) & (u[t] != -math.inf)
        i, x = ids[t][ok], u[t][ok]
        if z[t].max() <= -1e30:  # masked whole
            lse[:, t] = -math.inf
            continue
        if len(i):
            lp = x - (lse_t[t].double().cpu() if lse_t is not None else torch.logsumexp(x, 0))
            p, lq = lp.exp(), z[t, i] / tau - lse[0, t]
            loss[t] = wk * tau ** 2 * torch.where(p == 0, 0.0, p * (lp - lq)).sum()
            p_sum[t] = p.sum()
            e = torch.softmax(z[t] / tau, 0) * p.sum()
            d[t] += wk * tau * e
            size[t] += wk * tau * e
            d[t].index_add_(0, i, -wk * tau * p)
            size[t].index_add_(0, i, wk * tau * p)
        if labels is not None and 0 <= labels[t] < v:
            y = int(labels[t])
            if wl:
                loss[t] += wl * (lse[1, t] - z[t, y])
            e = wl * torch.softmax(z[t], 0)
            d[t] += e
            size[t] += e
            d[t, y] -= wl
            size[t, y] += wl
        if g is not None:
            d[t] *= float(g[t])
            size[t] *= abs(float(g[t]))
            if float(g[t]) == 0:
                d[t], size[t] = 0, 0
    return loss, lse, d, size, p_sum


def close(got, want, bound):
    """Infinities and NaNs where the result, in got's type, has them; |error| <= bound elsewhere (where the bound
    reaches beyond the type's range, the result may have left it)."""
    want = want.double()
    fine = torch.isfinite(want.to(got.dtype))
    edge = fine & ~torch.isfinite((want.abs() + bound.nan_to_num(nan=0.0)).to(got.dtype))
    got = torch.where(edge.to(got.device), want.to(got.dtype).to(got.device), got)
    got, want = got.double().cpu(), torch.where(fine, want, want.to(got.dtype).double())
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    there = ~fine & ~torch.isnan(want)
    assert torch.equal(got[there], want[there])
    assert torch.isfinite(got[fine]).all()
    worst = ((got - want).abs()[fine] / bound[fine]).max().item() if fine.any() else 0.0
    assert worst <= 1.0, worst


def relative(z, u, tau):
    """The relative error of an exponential of a difference of logits and
    normaliser in 32 bits: both are rounded at magnitudes up to M, in base 2, and
    the function itself is good to 2^-22; the sums add less than 2^-20."""
    m = max((x[torch.isfinite(x) & (x.abs() < 1e30)].abs().max().item() if x.numel() and (torch.isfinite(x) & (x.abs() < 1e30)).any() else 0.0)
            for x in (z.float(), u.float()))
    return 2.0 ** -22 * (8 + 4 * (m * 1.45 * max(1.0, 1 / tau) + 20))


def check_distill(z, ids, u, g, tau=1.0, wk=1.0, wl=0.0, lse_t=None, labels=None, dlogits=None):
    kw = dict(temperature=tau, kd_weight=wk, teacher_lse=lse_t, labels=labels, label_weight=wl)
    keep = z.clone()
    loss, lse, d, size, p_sum = ref_distill(z, ids, u, g, tau, wk, wl, lse_t, labels)
    n = 1 if labels is None else 2
    rel = relative(z, u, tau)
    spread_ = lse[0].abs().nan_to_num(posinf=0, neginf=0) + lse[1].abs().nan_to_num(posinf=0, neginf=0) + 8
    bound_lse = rel * torch.ones_like(lse) * 2
    # an entry on a masked logit (its type's lowest value) makes terms as large as the loss itself
    bound_loss = (wk * tau ** 2 * p_sum + wl + 1e-30) * rel * (2 + spread_) * 4 + rel * loss.abs().nan_to_num(nan=0, posinf=0)
    bound_d = size * (UNIT[z.dtype] + 2 * rel) + TINY[z.dtype] + UNIT[z.dtype] * d.abs()
    got, stats = apc.distill_loss(z, ids, u, **kw)
    close(stats, lse[:n], bound_lse[:n])
    close(got, loss, bound_loss)
    grad = apc.distill_grad(z, ids, u, stats, g, **kw)
    close(grad, d, bound_d)
    got2, stats2, grad2 = apc.distill_loss_grad(z, ids, u, g, out=dlogits, **kw)
    close(stats2, lse[:n], bound_lse[:n])
    close(got2, loss, bound_loss)
    close(grad2, d, bound_d)
    if dlogits is None:
        assert torch.equal(z.nan_to_num(nan=9.0), keep.nan_to_num(nan=9.0))
    # in the logits' place
    for form in ("both", "grad"):
        y = keep.clone()
        r = apc.distill_loss_grad(y, ids, u, g, out=y, **kw)[2] if form == "both" else \
            apc.distill_grad(y, ids, u, stats, g, out=y, **kw)
        assert r.data_ptr() == y.data_ptr()
        close(y, d, bound_d)
    return got, stats, grad


def weights(rows, seed=11):
    g = torch.rand(rows, generator=gen(seed), device="cuda") + 0.5
    g[rows // 3:rows // 3 + 1] = 0.0
    g[rows // 2:rows // 2 + 1] = -2.0
    return g


@pytest.mark.parametrize("rows,vocab,k", [(1, 1, 1), (1, 7, 3), (2, 31, 40), (3, 100, 0), (5, 129, 1), (4, 1000, 33),
                                          (7, 4097, 64), (2, 32768, 128), (3, 50001, 200), (1, 150001, 1024), (33, 515, 31),
                                          (400, 70, 5), (2, 300007, 16), (1, 1200003, 8)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_distill(rows, vocab, k, dtype):
    z = torch.randn(rows, vocab, generator=gen(1), device="cuda").mul_(4).to(dtype)
    ids, u = teacher_of(rows, vocab, k, 2, wide=rows % 2 == 0)
    check_distill(z, ids, u, weights(rows))


@pytest.mark.parametrize("vocab,k", [(777, 20), (32769, 100)])
@pytest.mark.parametrize("tau", [0.5, 1.0, 3.0])
@pytest.mark.parametrize("mode", ["labels", "lse", "labels lse", "label only"])
@pytest.mark.parametrize("teacher_dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_distill_options(vocab, k, tau, mode, teacher_dtype):
    rows = 6
    z = torch.randn(rows, vocab, generator=gen(1), device="cuda").mul_(3).bfloat16()
    ids, u = teacher_of(rows, vocab, k, 2, teacher_dtype)
    lse_t = labels = None
    if "lse" in mode:
        lse_t = torch.logsumexp(torch.where(torch.isfinite(u.float()), u.float(), -30.0) / tau, 1) + 0.3
    if "label" in mode:
        labels = torch.randint(0, vocab, (rows,), generator=gen(4), device="cuda").to(torch.int32 if tau == 1 else torch.int64)
        labels[2], labels[3] = -100, vocab
        if k and 0 <= ids[0, 0] < vocab:
            labels[0] = ids[0, 0]
    wk = 0.0 if mode == "label only" else 0.7
    check_distill(z, ids, u, weights(rows), tau, wk, 0.3 if labels is not None else 0.0, lse_t, labels)


@pytest.mark.parametrize("extra,offset,dextra,doffset", [(0, 1, 0, 1), (0, 1, 0, 0), (1, 0, 1, 0), (3, 2, 3, 2), (8, 0, 8, 8),
                                                         (5, 0, 0, 3), (16, 7, 0, 0)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_distill_strides(extra, offset, dextra, doffset, dtype):
    """Any row pitch and start of the logits and their gradient; what surrounds the gradient stays."""
    rows, vocab, k = 5, 1003, 17
    z = strided(torch.randn(rows, vocab, generator=gen(1), device="cuda").to(dtype), extra, offset)
    ids, u = teacher_of(rows, vocab, k, 2)
    room = torch.full((doffset + rows * (vocab + dextra) + 64,), 3.0, dtype=dtype, device="cuda")
    out = room[doffset:doffset + rows * (vocab + dextra)].view(rows, vocab + dextra)
    labels = torch.arange(rows, device="cuda") * 200
    check_distill(z, ids, u, weights(rows), 2.0, 1.0, 0.5, None, labels, dlogits=out[:, :vocab])
    assert (out[:, vocab:] == 3).all() and (room[:doffset] == 3).all()
    assert (room[doffset + rows * (vocab + dextra):] == 3).all()


@pytest.mark.parametrize("vocab", [300, 40000])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_distill_masks(vocab, dtype):
    """Masked logits of both kinds, rows without a student, rows without a
    teacher, entries and labels on masked places, probabilities of zero."""
    rows, k = 9, 12
    low = torch.finfo(dtype).min
    z = torch.randn(rows, vocab, generator=gen(1), device="cuda").mul_(3).to(dtype)
    ids, u = teacher_of(rows, vocab, k, 2, ragged=False)
    z[0, 100:] = -math.inf
    z[1, 100:] = low
    z[2] = -math.inf
    z[3] = low                      # masked whole too
    ids[4] = -1
    u[5] = -math.inf
    ids[0] = torch.arange(k, device="cuda")
    ids[1] = torch.arange(k, device="cuda")
    u[6, 1:] = -300.0               # probabilities that are zero in 32 bits
    z[7, 0] = 1000.0                # all of the student on one place
    ids[8, 3:] = -5
    u[8, 3:] = math.inf             # beside a padded id nothing counts
    labels = torch.randint(0, 50, (rows,), generator=gen(4), device="cuda")
    check_distill(z, ids, u, weights(rows), 1.0, 1.0, 0.0)
    check_distill(z, ids, u, weights(rows), 2.0, 1.0, 0.25, None, labels)
    # an entry or a label on a masked place: an infinite loss, a finite gradient
    z[0, 5] = -math.inf
    loss, _, d = apc.distill_loss_grad(z, ids, u, weights(rows), temperature=1.0)
    assert loss[0] == math.inf and torch.isfinite(d[0].float()).all()
    assert torch.isfinite(loss[1:]).all()


def test_distill_nan_stays_in_its_row():
    rows, vocab, k = 6, 5000, 9
    z = torch.randn(rows, vocab, generator=gen(1), device="cuda")
    ids, u = teacher_of(rows, vocab, k, 2, ragged=False)
    z[1, 4000] = math.nan
    u[2, 3] = math.nan
    z[4, 10] = math.inf
    g = torch.ones(rows, device="cuda")
    g[5] = 0.0
    z[5, 7] = math.nan              # a row that does not count
    loss, lse, d = apc.distill_loss_grad(z, ids, u, g)
    grad = apc.distill_grad(z, ids, u, lse, g)
    for x in (d, grad):
        assert torch.isnan(x[1]).any() and torch.isnan(x[2]).any() and torch.isnan(x[4]).any()
        assert torch.isfinite(x[[0, 3]]).all() and not x[5].any()
    assert torch.isnan(loss[[1, 2]]).all() and torch.isfinite(loss[[0, 3]]).all()


def test_distill_same_id_twice():
    """Entries of one place add up, in the loss and in the gradient, with the label on it too."""
    rows, vocab, k = 4, 600, 64
    z = torch.randn(rows, vocab, generator=gen(1), device="cuda")
    ids = torch.randint(0, 9, (rows, k), generator=gen(2), device="cuda")
    u = torch.randn(rows, k, generator=gen(3), device="cuda")
    labels = torch.full((rows,), 4, device="cuda")
    check_distill(z, ids, u, weights(rows), 1.5, 1.0, 0.5, None, labels)


@pytest.mark.parametrize("tau,wl", [(1.0, 0.0), (2.0, 0.5)])
def test_distill_gradient_against_differences(tau, wl):
    """Central differences of the loss: their error is the loss's own over h
    plus h^2/6 times the third derivative, at most kd_weight/tau + label_weight."""
    vocab, k, h = 40, 6, 2.0 ** -5
    z = torch.randn(1, vocab, generator=gen(1), device="cuda")
    ids, u = teacher_of(1, vocab, k, 2, ragged=False)
    labels = torch.full((2 * vocab,), 3, device="cuda")
    step = torch.cat([torch.eye(vocab, device="cuda"), -torch.eye(vocab, device="cuda")]) * h
    kw = dict(temperature=tau, label_weight=wl)
    loss, _ = apc.distill_loss(z + step, ids.expand(2 * vocab, k).contiguous(), u.expand(2 * vocab, k).contiguous(),
                               labels=labels, **kw)
    slope = (loss[:vocab].double() - loss[vocab:].double()) / (2 * h)
    _, _, d = apc.distill_loss_grad(z, ids, u, torch.ones(1, device="cuda"), labels=labels[:1], **kw)
    err_loss = (tau ** 2 + wl) * relative(z, u, tau) * 40
    bound = err_loss / h + h * h / 6 * (1 / tau + wl)
    assert (slope - d[0].double()).abs().max().item() <= bound


def test_distill_repeats_and_does_not_depend_on_the_grid(monkeypatch):
    for rows, vocab in ((3, 32768), (2, 200001), (500, 1000)):
        z = torch.randn(rows, vocab, generator=gen(1), device="cuda").bfloat16()
        ids, u = teacher_of(rows, vocab, 50, 2)
        g = weights(rows)
        first = apc.distill_loss_grad(z, ids, u, g, temperature=2.0)
        again = apc.distill_loss_grad(z, ids, u, g, temperature=2.0)
        monkeypatch.setenv("APC_GRID_LIMIT", "5")
        other = apc.distill_loss_grad(z, ids, u, g, temperature=2.0)
        monkeypatch.delenv("APC_GRID_LIMIT")
        for x, y, w in zip(first, again, other):
            assert torch.equal(x, y) and torch.equal(x, w)


@pytest.mark.parametrize("vocab,k", [(1, 1), (5, 7), (100, 10), (513, 40), (2049, 256), (4095, 33), (4097, 300)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_distill_many_short_rows(vocab, k, dtype):
    """More rows than SMs: masks of both kinds, rows without a student or a
    teacher, equal ids, labels on them, odd starts of the rows."""
    rows = 170
    z = torch.randn(rows, vocab, generator=gen(1), device="cuda").mul_(3)
    z[::7, vocab // 2:] = -math.inf
    z[1::7, vocab // 2:] = torch.finfo(dtype).min
    z[2::31] = -math.inf
    z[3::37] = torch.finfo(dtype).min
    z = strided(z.to(dtype), 1, 3)
    ids, u = teacher_of(rows, vocab, k, 2, wide=False)
    ids[::7] = ids[::7].clamp(max=max(0, vocab // 2 - 1)) if vocab > 1 else -1  # not on the masked half
    ids[4::41] = -1
    ids[5::43, k // 2:] = ids[5::43, :1]
    u[5::43] = 1.0
    labels = torch.randint(0, max(1, vocab // 2), (rows,), generator=gen(4), device="cuda")
    if vocab == 1:
        labels[::7] = -1
    labels[::5] = -100
    g = torch.rand(rows, generator=gen(5), device="cuda") - 0.3
    g[::11] = 0.0
    check_distill(z, ids, u, g)
    check_distill(z, ids, u, g, 2.5, 0.7, 0.3, None, labels)
    check_distill(z, ids, u, g, 1.0, 0.7, 0.3, torch.full((rows,), 4.0, device="cuda"), labels)


@pytest.mark.parametrize("vocab", [30000, 250000])
def test_distill_rows_beyond_shared_memory(vocab):
    """Rows that are read a second time for the gradient, many and few."""
    for rows, dtype in ((160, torch.float32), (3, torch.float32), (2, torch.bfloat16)):
        z = torch.randn(rows, vocab, generator=gen(1), device="cuda").mul_(3).to(dtype)
        ids, u = teacher_of(rows, vocab, 600, 2)
        check_distill(z, ids, u, weights(rows), 1.5, 1.0, 0.5, None, torch.arange(rows, device="cuda"))


def test_operators_on_a_stream_of_their_own():
    """Work is enqueued on the stream given, behind what it already holds."""
    s = torch.cuda.Stream()
    x = torch.zeros(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        for _ in range(20):
            x.add_(1.0)
        q, sc = apc.quantize_fp8(x)
        out = apc.matmul_fp8(q[:256], sc[:, :256], q[:512], sc[:, :512], out_dtype=torch.float32)
        ids = torch.zeros(256, 1, dtype=torch.int64, device="cuda")
        loss, _ = apc.distill_loss(out, ids, torch.zeros(256, 1, device="cuda"))
    s.synchronize()
    assert (out == 400.0 * 4096).all()
    assert torch.allclose(loss, torch.full_like(loss, math.log(512.0)), rtol=0, atol=0.25)  # ulp of 2.4e6 in base 2
    r = apc.quantize_fp8(x, stream=s.cuda_stream)
    s.synchronize()
    assert torch.equal(r[1], sc)


def test_distill_refusals():
    z = torch.randn(4, 50, device="cuda")
    ids, u = teacher_of(4, 50, 5, 2)
    g = torch.ones(4, device="cuda")
    for bad in (lambda: apc.distill_loss(z.t(), ids, u), lambda: apc.distill_loss(z, ids[:3], u),
                lambda: apc.distill_loss(z, ids.float(), u), lambda: apc.distill_loss(z, ids, u[:, :4]),
                lambda: apc.distill_loss(z, ids, u, labels=torch.zeros(3, dtype=torch.int64, device="cuda")),
                lambda: apc.distill_loss_grad(z, ids, u, g[:2]), lambda: apc.distill_loss(z.cpu(), ids, u),
                lambda: apc.distill_loss_grad(z, ids, u, g, out=torch.empty(4, 50, device="cuda").bfloat16())):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: apc.distill_loss(z, ids, u, temperature=0.0), lambda: apc.distill_loss(z, ids, u, kd_weight=-1.0),
                lambda: apc.distill_loss_grad(z, ids, u, g, out=z.view(-1).as_strided((4, 50), (49, 1)))):
        with pytest.raises((apc.ApcError, ValueError)):
            bad()
    with pytest.raises(apc.ApcError) as e:
        apc.distill_loss_grad(z, ids, u, g, loss=g)  # the loss over its own weights
    assert e.value.status == 1


def test_example_learns_and_its_replicas_agree():
    """The operators as they are used together: a distilled head's steps."""
    import importlib.util
    import os

    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "distill_head.py")
    spec = importlib.util.spec_from_file_location("distill_head", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses = example.main(["--tokens", "300", "--vocab", "2003", "--hidden", "520", "--k", "20", "--steps", "6"])
    assert all(b < a for a, b in zip(losses, losses[1:]))


def test_head_gradients_against_64_bits():
    """The chain's gradients, from the quantized operands that it used, as the
    formula gives them in 64 bits."""
    tokens, vocab, hidden, k = 200, 1003, 272, 12
    x = torch.randn(tokens, hidden, generator=gen(1), device="cuda").bfloat16()
    w = torch.randn(vocab, hidden, generator=gen(2), device="cuda").mul_(0.1).bfloat16()
    x8, xs, x8t, xst = apc.quantize_fp8(x, transposed=True)
    w8, ws, w8t, wst = apc.quantize_fp8(w, block_rows=128, transposed=True)
    logits = apc.matmul_fp8(x8, xs, w8, ws, out_dtype=torch.float32)
    ids, u = teacher_of(tokens, vocab, k, 3)
    g = torch.full((tokens,), 1.0 / tokens, device="cuda")
    _, _, d = apc.distill_loss_grad(logits, ids, u, g, temperature=2.0)
    _, _, want, size, _ = ref_distill(logits, ids, u, g, 2.0, 1.0, 0.0)
    close(d, want, size * (UNIT[torch.float32] + 2 * relative(logits, u, 2.0)) + TINY[torch.float32])
    d8, ds, d8t, dst = apc.quantize_fp8(d, transposed=True)
    for a, sa, ba, b, sb, bb in ((d8, ds, 1, w8t, wst, 128), (d8t, dst, 1, x8t, xst, 1)):
        ref, size = ref_matmul(a, sa, ba, b, sb, bb)
        check_matmul(apc.matmul_fp8(a, sa, b, sb, out_dtype=torch.float32), ref, size, a.shape[1])
    # and the gradient of the head within what 8 bits keep: half an ulp of E4M3, 2^-4, of each factor
    dw = apc.matmul_fp8(d8t, dst, x8t, xst, out_dtype=torch.float32).double()
    full = d.double().t() @ x.double()
    size = d.double().abs().t() @ x.double().abs()
    floor = (d8t.shape[1] * 2.0 ** -10) * dst.max().double() * x.double().abs().max()  # values below the least normal one
    assert ((dw - full).abs() <= size * (2 * 2.0 ** -4 + 2.0 ** -8) + floor * 2).all()


@pytest.mark.parametrize("vocab,k", [(900, 300), (2500, 512), (5000, 40), (5000, 1000), (70001, 33)])
@pytest.mark.parametrize("limit", ["1", "3"])
def test_distill_many_rows_a_block(vocab, k, limit, monkeypatch):
    """Rows one after the other in few blocks, in every form: what a row leaves in
    shared memory is taken again only when its loss and gradient are through."""
    rows = 61
    z = torch.randn(rows, vocab, generator=gen(1), device="cuda").mul_(3).bfloat16()
    ids, u = teacher_of(rows, vocab, k, 2)
    labels = torch.randint(0, vocab, (rows,), generator=gen(4), device="cuda")
    monkeypatch.setenv("APC_GRID_LIMIT", limit)
    check_distill(z, ids, u, weights(rows))
    check_distill(z, ids, u, weights(rows), 2.0, 0.7, 0.3, None, labels)
    assert apc.device_status() == 0


@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("tau,wl", [(1.0, 0.5), (2.0, 0.5), (1.5, 0.0)])
def test_distill_without_the_teachers_weight(many, tau, wl):
    """A weight of 0 leaves the teacher out: entries on masked logits and a teacher
    that is not finite change nothing.  Few rows and as many as one warp each takes."""
    rows = 4 * torch.cuda.get_device_properties(0).multi_processor_count + 3 if many else 7
    vocab, k = 600, 20
    z = torch.randn(rows, vocab, generator=gen(1), device="cuda").mul_(3)
    z[:, 300:] = -math.inf
    ids, u = teacher_of(rows, vocab, k, 2, ragged=False)
    assert (ids >= 300).any(1).float().mean() > 0.9
    u[1, 2], u[2, 3] = math.nan, math.inf
    labels = torch.randint(0, 300, (rows,), generator=gen(4), device="cuda")
    kw = dict(temperature=tau, kd_weight=0.0, labels=labels, label_weight=wl)
    none = check_distill(z, ids[:, :0], u[:, :0], weights(rows), tau, 0.0, wl, None, labels)
    loss, stats = apc.distill_loss(z, ids, u, **kw)
    both = apc.distill_loss_grad(z, ids, u, weights(rows), **kw)
    assert torch.isfinite(loss).all()
    assert torch.equal(loss, none[0]) and torch.equal(stats, none[1])
    assert torch.equal(both[0], loss) and torch.equal(both[1], stats)
    assert torch.equal(apc.distill_grad(z, ids, u, stats, weights(rows), **kw), none[2])


def test_distill_grad_needs_statistics_and_weights():
    """What a call reads has to be given: it is not allocated in the caller's place."""
    z = torch.randn(4, 50, device="cuda")
    ids, u = teacher_of(4, 50, 5, 2)
    g = torch.ones(4, device="cuda")
    _, lse = apc.distill_loss(z, ids, u)
    for bad in (lambda: apc.distill_grad(z, ids, u, None, g), lambda: apc.distill_grad(z, ids, u, lse, None),
                lambda: apc.distill_loss_grad(z, ids, u, None),
                lambda: apc.distill_grad(z, ids, u, lse, g, labels=torch.zeros(4, dtype=torch.int64, device="cuda"))):
        with pytest.raises(ValueError):
            bad()


def test_outputs_of_a_given_stream_while_the_current_one_is_busy():
    """Memory that the current stream has just freed, with work on it still to
    run, is not where a call on another stream writes."""
    x = torch.randn(1024, 1024, generator=gen(1), device="cuda")
    want = apc.quantize_fp8(x)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    for stream in (s, s.cuda_stream):
        torch.cuda._sleep(20_000_000)
        for _ in range(8):
            old = [torch.empty_like(want[0]), torch.empty_like(want[1])]
            for t in old:
                t.view(torch.uint8).fill_(0x11)
            del old, t
        got = apc.quantize_fp8(x, stream=stream)
        s.synchronize()
        torch.cuda.synchronize()
        assert torch.equal(got[0].view(torch.uint8), want[0].view(torch.uint8)) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("m,n,k", [(4100, 4357, 2000), (8200, 8300, 500)])
@pytest.mark.parametrize("bb", [1, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_matmul_grid_with_scales_of_both_kinds(m, n, k, bb, dtype, monkeypatch):
    """Scales that are powers of two, and others in some rows and columns: a tile's
    bits follow from its own scales, not from the tiles that its blocks had before."""
    x = torch.randn(m, k, generator=gen(1), device="cuda")
    y = torch.randn(n, k, generator=gen(2), device="cuda")
    a, sa = apc.quantize_fp8(x)
    b, sb = apc.quantize_fp8(y, block_rows=bb)
    for at in ((), (0, 1500, 1501, 3900), (m - 1,)):
        odd, odd_b = sa.clone(), sb.clone()
        odd[3, list(at)] *= 1.5
        odd_b[-1, sb.shape[1] // 2] *= 1.25 if len(at) == 4 else 1.0
        ref, size = ref_matmul(a, odd, 1, b, odd_b, bb)
        first = apc.matmul_fp8(a, odd, b, odd_b, out_dtype=dtype)
        check_matmul(first, ref, size, k)
        for limit in ("7", "40", "3"):
            monkeypatch.setenv("APC_GRID_LIMIT", limit)
            assert torch.equal(first, apc.matmul_fp8(a, odd, b, odd_b, out_dtype=dtype))
        monkeypatch.delenv("APC_GRID_LIMIT")
        # nor from other rows' scales, a tile's height away
        if at:
            apart = torch.ones(m, dtype=torch.bool, device="cuda")
            for i in at:
                apart[i // 256 * 256:i // 256 * 256 + 256] = False
            assert torch.equal(first[apart], apc.matmul_fp8(a, sa, b, odd_b, out_dtype=dtype)[apart])
    assert apc.device_status() == 0


def one_sign(m, n, k, seed=1):
    """Quantized operands of positive values, whose sums' roundings do not cancel, and their product."""
    x = torch.randn(m, k, generator=gen(seed), device="cuda").abs()
    y = torch.randn(n, k, generator=gen(seed + 1), device="cuda").abs()
    a, sa = apc.quantize_fp8(x)
    b, sb = apc.quantize_fp8(y, block_rows=128)
    return a, sa, b, sb, ref_matmul(a, sa, 1, b, sb, 128)[0]


@pytest.mark.parametrize("m,n,k", [(4096, 4096, 2048), (4096, 4096, 8192), (1500, 5000, 7777), (64, 4096, 8192)])
def test_matmul_to_32_bits_has_no_bias(m, n, k):
    """The tensor cores sum 128 products in four steps, each off by at most 2^-23 and on
    average half that: 2^-22 of the mean.  Sums over k are rounded to nearest."""
    a, sa, b, sb, ref = one_sign(m, n, k)
    off = apc.matmul_fp8(a, sa, b, sb, out_dtype=torch.float32).double() / ref - 1
    assert off.mean().abs().item() <= 2.0 ** -22
    assert off.abs().max().item() <= 2.0 ** -22 * 2 + (k / 128) ** 0.5 * 6 * 2.0 ** -24  # six deviations of the sums' own
    assert apc.device_status() == 0


@pytest.mark.parametrize("dtype,k", [(torch.float16, 16384), (torch.float16, 16500), (torch.bfloat16, 131072), (torch.bfloat16, 131200)])
def test_matmul_to_16_bits_over_long_sums(dtype, k):
    """The rounding to 16 bits, and a sixteenth of it for the sum."""
    a, sa, b, sb, ref = one_sign(2048, 2304, k)
    out = apc.matmul_fp8(a, sa, b, sb, out_dtype=dtype)
    assert ((out.double() / ref - 1).abs().max() <= UNIT[dtype] * (1 + 1 / 16)).item()
    assert apc.device_status() == 0


@pytest.mark.parametrize("m,n,k", [(1, 300, 700), (40, 333, 2000), (130, 257, 300), (777, 1001, 640), (2100, 2050, 1111),
                                   (4100, 4357, 600)])
@pytest.mark.parametrize("bb", [1, 128])
@pytest.mark.parametrize("powers", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_matmul_scales_far_apart(m, n, k, bb, powers, dtype):
    """Scales whose product leaves fp32's range, or its normal numbers, though the
    result need not: zeros stay zeros, small sums times large scales are finite, and large
    sums times small scales keep their digits.  A block's sum is rounded to fp32 times b's
    scale, at 2^-150 where that is not normal, and then times a's."""
    a, sa = operand(m, k, 1, E4M3, 1)
    b, sb = operand(n, k, bb, E4M3, 2)
    a.view(torch.uint8)[::5] = 0
    e = torch.randint(-125, 126, (m,), generator=gen(3), device="cuda")
    f = torch.randint(-125, 126, (sb.shape[1],), generator=gen(4), device="cuda")
    e[::7] = 120
    f[::3] = 100                       # with the rows above: zeros, or an overflow
    e[1::7], f[1::3] = -70, -65        # a product of scales that is not normal
    near = torch.arange(m, device="cuda") % 7 == 2
    e[near], f[2::3] = 70, 60          # beyond the range but for small sums
    small = a[near].float() * 2.0 ** -6
    a[near] = small.to(E4M3)
    room = b.float()
    room[2 * bb:3 * bb] *= 2.0 ** -8
    b.copy_(room.to(E4M3))
    sa = torch.exp2(e.double()).float() * (1.0 if powers else sa * 100)
    sb = torch.exp2(f.double()).float() * (1.0 if powers else sb * 100)
    sa, sb = sa.expand(-(-k // 128), m).contiguous(), sb.expand(-(-k // 128), f.numel()).contiguous()
    ref, size = ref_matmul(a, sa, 1, b, sb, bb)
    out = apc.matmul_fp8(a, sa, b, sb, out_dtype=dtype)
    bound = UNIT[dtype] * ref.abs() + size * (2.0 ** -23 * (128 + k / 128 + 5)) * (1 + UNIT[dtype]) + TINY[dtype] + \
        -(-k // 128) * 2.0 ** -150 * (1 + sa[0].double()[:, None])
    top = torch.finfo(dtype).max
    inside = size * torch.clamp(1 / sa[0].double()[:, None], min=1) + bound < top
    beyond = ref.abs() - bound > top * (1 + UNIT[dtype])  # between: sums that leave the range on the way
    assert not out[::5].any()
    worst = ((out.double() - ref).abs() / bound)[inside].max().item()
    assert worst <= 1.0, worst
    assert not torch.isfinite(out[beyond]).any()  # blocks' sums beyond the range, of both signs where they are a NaN
    assert apc.device_status() == 0


@pytest.mark.parametrize("k", [255, 256, 279, 280, 511, 512, 513, 700, 1024])
def test_distill_over_the_kernel_s_shapes(k, monkeypatch):
    """Every number of teachers' warps and ring of the kernel for longer rows, with
    several rows a block."""
    rows, vocab = 13, 33001
    z = torch.randn(rows, vocab, generator=gen(1), device="cuda").mul_(3).bfloat16()
    ids, u = teacher_of(rows, vocab, k, 2, wide=False)
    labels = torch.randint(0, vocab, (rows,), generator=gen(4), device="cuda")
    labels[:4] = ids[:4, 0].clamp(0, vocab - 1)
    monkeypatch.setenv("APC_GRID_LIMIT", "2")
    check_distill(z, ids, u, weights(rows))
    check_distill(z, ids, u, weights(rows), 4.0, 0.7, 0.3, None, labels)
    assert apc.device_status() == 0


@pytest.mark.parametrize("vocab,k,tau", [(1, 1, 2.0), (5, 7, 4.0), (100, 10, 2.5), (513, 40, 1.0), (2049, 256, 4.0), (4095, 33, 2.0)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_distill_one_warp_a_row(vocab, k, tau, dtype):
    """As many rows as take a warp each (four for each SM), a few blocks going through
    several: masks of both kinds, rows without a student or a teacher, equal ids, labels
    on them and beyond the vocabulary, odd starts of the rows, every power of the temperature."""
    rows = 4 * torch.cuda.get_device_properties(0).multi_processor_count + 3
    z = torch.randn(rows, vocab, generator=gen(1), device="cuda").mul_(3)
    z[::7, vocab // 2:] = -math.inf
    z[1::7, vocab // 2:] = torch.finfo(dtype).min
    z[2::31] = -math.inf
    z[3::37] = torch.finfo(dtype).min
    z = strided(z.to(dtype), 1, 3)
    ids, u = teacher_of(rows, vocab, k, 2, wide=vocab % 2 == 0)
    ids[::7] = ids[::7].clamp(max=max(0, vocab // 2 - 1)) if vocab > 1 else -1  # not on the masked half
    ids[4::41] = -1
    ids[5::43, k // 2:] = ids[5::43, :1]
    u[5::43] = 1.0
    labels = torch.randint(0, max(1, vocab // 2), (rows,), generator=gen(4), device="cuda")
    on = (ids[:, 0] >= 0) & (ids[:, 0] < max(1, vocab // 2))
    labels = torch.where(on & (torch.arange(rows, device="cuda") % 2 == 0), ids[:, 0].to(labels.dtype), labels)
    if vocab == 1:
        labels[::7] = -1
    labels[::5] = -100
    g = torch.rand(rows, generator=gen(5), device="cuda") - 0.3
    g[::11] = 0.0
    check_distill(z, ids, u, g)
    check_distill(z, ids, u, g, tau, 0.7, 0.3, torch.full((rows,), 4.0, device="cuda") if k == 40 else None, labels)


@pytest.mark.parametrize("vocab", [100, 4095])
def test_distill_one_warp_a_row_does_not_depend_on_the_grid(vocab, monkeypatch):
    rows = 5 * torch.cuda.get_device_properties(0).multi_processor_count
    z = torch.randn(rows, vocab, generator=gen(1), device="cuda").bfloat16()
    ids, u = teacher_of(rows, vocab, 30, 2)
    g = weights(rows)
    first = apc.distill_loss_grad(z, ids, u, g, temperature=2.0)
    grad = apc.distill_grad(z, ids, u, first[1], g, temperature=2.0)
    monkeypatch.setenv("APC_GRID_LIMIT", "2")
    for x, y in zip(first, apc.distill_loss_grad(z, ids, u, g, temperature=2.0)):
        assert torch.equal(x, y)
    assert torch.equal(apc.distill_loss(z, ids, u, temperature=2.0)[0], first[0])
    assert torch.equal(apc.distill_grad(z, ids, u, first[1], g, temperature=2.0), grad)


def test_columns_of_one_buffer():
    """Logits and their gradient as two halves of a buffer."""
    rows, vocab, k = 9, 5000, 12
    z = torch.randn(rows, vocab, generator=gen(1), device="cuda").bfloat16()
    ids, u = teacher_of(rows, vocab, k, 2)
    want = apc.distill_loss_grad(z, ids, u, weights(rows))
    room = torch.zeros(rows, 2 * vocab, dtype=torch.bfloat16, device="cuda")
    room[:, :vocab] = z
    got = apc.distill_loss_grad(room[:, :vocab], ids, u, weights(rows), out=room[:, vocab:])
    assert torch.equal(got[0], want[0]) and torch.equal(room[:, vocab:], want[2]) and torch.equal(room[:, :vocab], z)
