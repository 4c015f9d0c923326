"""The root-mean-square norm and its gradient against plain implementations in
64 bits, on the GPU.

Bounds, in units u = 2^-24 of a rounding to fp32.  rstd is rounded once from a
mean that is right to 2^-40 of itself: off by u, and some 2^-16 more.
Everything behind rstd has a fixed order of fp32 operations, which the same
operations in torch repeat bit for bit."""
import math

import pytest
import torch

import paper_2609_18178_gb300 as apc

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}
TYPES = [torch.bfloat16, torch.float16, torch.float32]
SIZES = [(1, 1), (1, 8), (3, 7), (5, 128), (2, 129), (7, 255), (9, 1000), (1, 4096), (33, 4096), (2, 4099), (1, 8192), (160, 2048),
         (200, 5003), (300, 64), (700, 264), (5, 16384), (3, 16385), (2, 40001)]
# enough rows to walk them: (rows, columns)
MANY = [(305, 513), (700, 1000), (400, 1024), (333, 4096), (1000, 2047), (350, 5003), (306, 9001), (310, 16384), (320, 16377)]


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


def inputs(r, c, dtype, wdtype, seed=0):
    g = gen(r * 100_003 + c + seed)
    x = torch.randn(r, c, generator=g, device="cuda")
    x[:, ::37] *= 20
    w = torch.randn(c, generator=g, device="cuda") * 0.2 + 1
    return x.to(dtype), torch.randn(r, c, generator=g, device="cuda").mul_(3).to(dtype), w.to(wdtype)


def check_rstd(h, eps, rstd):
    want = 1 / (h.double().square().mean(1) + eps).sqrt()
    assert ((rstd.double() - want).abs() <= (1 + 2.0 ** -8) * U * want + 2.0 ** -150).all()


def y_of(h, rstd, w):
    return h.float() * rstd[:, None] * w.float()


@pytest.mark.parametrize("r,c", SIZES + MANY)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("residual", [False, True])
def test_norm(r, c, dtype, residual):
    # packed; at odds with each other; alike within 16 bytes, but at no boundary
    for extra, offset, wdtype in ((0, 0, dtype), (5 if c % 2 else 8, 3 if c % 2 else 8, torch.float32), (8, 3, dtype)):
        x, res, w = inputs(r, c, dtype, wdtype)
        x, res = strided(x, extra, offset), strided(res, 2 * extra, offset) if residual else None
        total = strided(torch.zeros_like(x), extra, offset if extra == 8 else 0) if residual else None
        out = strided(torch.zeros_like(x), 3 * extra, offset)
        y, h, rstd = apc.rms_norm(x, w, eps=1e-5, residual=res, out=out, sum=total)
        assert y is out and rstd.shape == (r,) and rstd.dtype == torch.float32
        want = (x.float() + res.float()).to(dtype) if residual else x
        assert h is (total if residual else x) and torch.equal(h, want)
        check_rstd(h, 1e-5, rstd)
        assert torch.equal(y, y_of(h, rstd, w).to(dtype))
        surround = y.as_strided((r, c + 3 * extra), (c + 3 * extra, 1), y.storage_offset())[:, c:]
        assert surround.isnan().all()  # what lies behind the columns is left as it was


@pytest.mark.parametrize("r,c", SIZES + MANY)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("fmt", [torch.float8_e4m3fn, torch.float8_e5m2])
@pytest.mark.parametrize("transposed", [False, True])
def test_norm_to_8_bits(r, c, dtype, fmt, transposed):
    x, res, w = inputs(r, c, dtype, torch.float32 if transposed else dtype, 1)
    res = res if r % 2 else None
    if c % 3 == 0:
        x = strided(x, 3, 1)
    elif c % 3 == 1:  # alike, at no boundary
        x, res = strided(x, 8, 5), None if res is None else strided(res, 16, 5)
    total = None if res is None else strided(torch.zeros_like(x), 0, x.storage_offset()) if c % 3 == 1 else torch.empty_like(res)
    *got, h, rstd = apc.rms_norm_fp8(x, w, eps=1e-6, residual=res, sum=total, dtype=fmt, transposed=transposed)
    assert torch.equal(h, x if res is None else (x.float() + res.float()).to(dtype))
    check_rstd(h, 1e-6, rstd)
    want = apc.quantize_fp8(y_of(h, rstd, w), dtype=fmt, transposed=transposed)
    assert len(got) == len(want)
    for a, b in zip(got, want):
        assert a.dtype == b.dtype and torch.equal(a.float(), b.float())
    if r <= 9 and c <= 1000:  # and the definition itself
        y = y_of(h, rstd, w).double()
        top = {torch.float8_e4m3fn: 448.0, torch.float8_e5m2: 57344.0}[fmt]
        for i in range(-(-c // 128)):
            m = y[:, 128 * i:128 * i + 128].abs().amax(1)
            s = got[1][i].double()
            assert ((m <= s * top) & ((m > s * top / 2) | (m == 0))).all()


def test_same_bits_however_rows_lie():
    """Few rows, many rows, aligned or not: rstd is rounded once, whatever the layout."""
    x, res, w = inputs(400, 3000, torch.bfloat16, torch.bfloat16)
    a = apc.rms_norm(x, w, residual=res)
    b = apc.rms_norm(strided(x, 1, 1), w, residual=strided(res, 1, 0))
    c = [apc.rms_norm(x[i:i + 1], w, residual=res[i:i + 1]) for i in range(100)]
    assert torch.equal(a[2], b[2]) and torch.equal(a[2][:100], torch.cat([t[2] for t in c]))
    assert torch.equal(a[2], (1 / (a[1].double().square().mean(1) + 1e-6).sqrt()).float())
    for dtype, r, cols in ((torch.bfloat16, 3000, 4096), (torch.float16, 9000, 200), (torch.float32, 2000, 1111)):
        x, _, w = inputs(r, cols, dtype, dtype)
        rstd = apc.rms_norm(x, w)[2]
        off = rstd != (1 / (x.double().square().mean(1) + 1e-6).sqrt()).float()
        assert off.sum() <= 1  # 2^-15 of the rows lie so near a border


@pytest.mark.parametrize("r,c,dtype", [(100_000, 200, torch.float32), (100_000, 200, torch.bfloat16), (50_000, 500, torch.float16),
                                       (10_000, 4096, torch.bfloat16), (5000, 9001, torch.float16), (5000, 4096, torch.float32),
                                       (1000, 20_000, torch.float32)])
def test_layouts_differ_at_borders_alone(r, c, dtype):
    """Sums within 2^-38 of themselves, so values within 2^-39, and 2^-40 for what follows: bits turn only that near a
    border.  (The mean in 64 bits is off by 2^-50 at most.)"""
    x, _, w = inputs(r, c, dtype, dtype, 13)
    some = slice(0, 120)
    exact = torch.cat([1 / (t.double().square().mean(1) + 1e-6).sqrt() for t in x.split(8192)])
    for got, want in ((apc.rms_norm(x, w)[2], exact), (apc.rms_norm(strided(x, 1, 1), w)[2], exact),
                      (apc.rms_norm(x[some], w)[2], exact[some])):
        turned = got != want.float()
        border = (got.double() + want.float().double())[turned] / 2
        assert ((border - want[turned]).abs() <= (2.0 ** -39 + 2.0 ** -40) * want[turned]).all()


@pytest.mark.parametrize("c", [264, 1000, 1003])
def test_norm_does_not_depend_on_the_grid(monkeypatch, c):
    x, res, w = inputs(1500, c, torch.bfloat16, torch.float32)
    a = apc.rms_norm_fp8(x, w, residual=res, transposed=True)
    d = apc.rms_norm_grad(res, x, w, a[-1])
    for limit in ("1", "7", "100"):
        monkeypatch.setenv("APC_GRID_LIMIT", limit)
        for p, q in zip(a, apc.rms_norm_fp8(x, w, residual=res, transposed=True)):
            assert torch.equal(p.float(), q.float())
        for p, q in zip(d, apc.rms_norm_grad(res, x, w, a[-1])):
            assert torch.equal(p, q)


@pytest.mark.parametrize("place", ["x", "residual"])
def test_sum_in_place(place):
    for r, c in ((9, 1000), (9, 40_000), (400, 1000), (400, 1003)):
        x, res, w = inputs(r, c, torch.bfloat16, torch.bfloat16)
        want = apc.rms_norm(x, w, residual=res)
        a, b = x.clone(), res.clone()
        got = apc.rms_norm(a, w, residual=b, sum=a if place == "x" else b)
        for p, q in zip(got, want):
            assert torch.equal(p, q)


@pytest.mark.parametrize("place", ["x", "residual"])
@pytest.mark.parametrize("r,c", [(9, 1003), (200, 1003), (300, 131), (1500, 203), (2000, 1200), (2100, 1003), (40, 20_003), (110, 20_003)])
@pytest.mark.parametrize("dtype", TYPES)
def test_sum_in_place_and_transposed(place, r, c, dtype):
    """The transpose is made of sums that a kernel still running stored where its input was, in sectors that rows share;
    below 2^21 elements the second kernel waits beside the first, above it starts as that one ends."""
    for extra, offset in ((0, 0), (1, 3), (8, 1)):
        x, res, w = inputs(r, c, dtype, dtype, 7)
        want = apc.rms_norm_fp8(x, w, residual=res, transposed=True)
        check_rstd(want[4], 1e-6, want[5])
        a, b = strided(x, extra, offset), strided(res, extra, offset)
        for _ in range(3):
            a.copy_(x), b.copy_(res)
            *got, rstd = apc.rms_norm_fp8(a, w, residual=b, sum=a if place == "x" else b, transposed=True)
            assert torch.equal(got[4], want[4])
            # rstd's bits may follow the layout, in a row near a border
            check_rstd(want[4], 1e-6, rstd)
            ref = apc.quantize_fp8(y_of(want[4], rstd, w), transposed=True)
            for p, q in zip(got, ref):
                assert torch.equal(p.float(), q.float())


@pytest.mark.parametrize("c", [1 << 19, 655_360, (1 << 20) + 3, 1 << 22])
@pytest.mark.parametrize("dtype", TYPES)
def test_long_rows_of_one_value(dtype, c):
    """What the additions of equal squares lose has one sign, and adds up over a row; huge values are summed scaled."""
    values = (torch.rand(24, generator=gen(c), device="cuda") * 1.5 + 0.5).to(dtype)
    if dtype != torch.float16:
        values[20:] *= 1e25
    x = values[:, None].expand(24, c).contiguous()
    rstd = apc.rms_norm(x, torch.ones(c, device="cuda", dtype=dtype))[2]
    # the mean of equal squares is the square: bounds as above
    want = 1 / (values.double().square() + 1e-6).sqrt()
    assert ((rstd.double() - want).abs() <= (1 + 2.0 ** -8) * U * want).all()


@pytest.mark.parametrize("r", [6, 400])
@pytest.mark.parametrize("c", [100, 1000, 4096, 5003, 20_000])
def test_rows_of_huge_values(r, c):
    """Squares that overflow binary32 are taken scaled; beside them ordinary rows, and tiny ones that eps rules."""
    x, _, w = inputs(r, c, torch.float32, torch.float32)
    x[0] *= 1e25
    x[1] *= 1e-25
    x[2] = 0
    x[3, ::3] = 3e38 * torch.sign(x[3, ::3])
    x[4, 0] = 1e20
    for dtype in (torch.float32, torch.bfloat16):
        h = x.to(dtype)
        y, _, rstd = apc.rms_norm(h, w, eps=1e-6)
        check_rstd(h, 1e-6, rstd)
        want = h.double() * rstd.double()[:, None] * w.double()
        assert ((y.double() - want).abs() <= (UNIT[dtype] + 3 * U) * want.abs() + TINY[dtype] * 2).all()


@pytest.mark.parametrize("r", [8, 400, 2000])
@pytest.mark.parametrize("c", [1, 100, 4096, 5003, 20_000])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_any_eps(r, c, dtype):
    """eps counts beside squares that overflow, and a mean and an eps whose sum does are no infinity."""
    if r * c > 10_000_000:
        r = 400
    x, _, w = inputs(r, c, dtype, dtype)
    for i, size in enumerate((1e16, 1e19, 1.2e19, 1e20, 1e28)):
        x[i] *= size / x[i].float().abs().max()
    x[5], x[5, 0] = 0, 2e19  # one element whose square overflows
    x[6], x[6, ::2] = 0, 1.8e19
    x[7] = 1.3e19
    for eps in (1e-20, 1e-5, 1.0, 1e10, 1e25, 1e36, 1e38, 3e38):
        check_rstd(x, eps, apc.rms_norm(x, w, eps=eps)[2])


@pytest.mark.parametrize("r", [8, 400])
@pytest.mark.parametrize("c", [100, 4096, 5003, 20_000])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_that_are_not_finite(r, c, dtype):
    x, res, w = inputs(r, c, dtype, dtype)
    x[1, c // 2] = math.inf
    x[3, 7] = math.nan
    x[5, c - 1] = -math.inf
    x[6, 3] = math.inf
    res[6, 3] = -math.inf  # their sum is a NaN
    y, h, rstd = apc.rms_norm(x, w, residual=res)
    assert rstd[[1, 5]].eq(0).all() and rstd[[3, 6]].isnan().all()
    fine = [0, 2, 4, 7, r - 1]
    check_rstd(h[fine], 1e-6, rstd[fine])
    want = y_of(h, rstd, w).to(dtype)
    assert torch.equal(y.isnan(), want.isnan()) and torch.equal(y.nan_to_num(), want.nan_to_num())
    assert y[1].isnan().sum() == 1 and (y[1].nan_to_num() == 0).all() and y[3].isnan().all()
    for fmt in (torch.float8_e4m3fn, torch.float8_e5m2):
        *got, _, _ = apc.rms_norm_fp8(x, w, residual=res, dtype=fmt, transposed=True)
        ref = apc.quantize_fp8(y_of(h, rstd, w), dtype=fmt, transposed=True)
        for a, b in zip(got, ref):
            assert torch.equal(a.float().isnan(), b.float().isnan())
            assert torch.equal(a.float().nan_to_num(), b.float().nan_to_num())
    w[5] = math.inf  # in a weight
    got = apc.rms_norm_fp8(res, w)
    ref = apc.quantize_fp8(y_of(res, got[-1], w))
    for a, b in zip(got, ref):
        assert torch.equal(a.float().nan_to_num(7.0), b.float().nan_to_num(7.0))


def test_nothing():
    w = torch.ones(16, device="cuda")
    x = torch.ones(0, 16, device="cuda")
    y, h, rstd = apc.rms_norm(x, w)
    assert y.shape == (0, 16) and rstd.shape == (0,)
    dw = torch.full((16,), 7.0, device="cuda")
    dx, dw = apc.rms_norm_grad(x, x, w, rstd, dweight=dw)
    assert dx.shape == (0, 16) and (dw == 0).all()  # a sum over no rows
    e = torch.ones(5, 0, device="cuda")
    assert apc.rms_norm(e, w[:0])[0].shape == (5, 0)
    assert apc.rms_norm_grad(e, e, w[:0], torch.ones(5, device="cuda"))[1].shape == (0,)


# ---- gradient

def check_grad(d, x, w, rstd, dres, dx, dw, parts):
    r, c = x.shape
    z, g = x.double() * rstd.double()[:, None], d.double() * w.double()
    mean = (g * z).mean(1, keepdim=True)
    want = (g - z * mean) * rstd.double()[:, None]
    # 16 products a thread for each 16,384 columns, 12 additions between threads, 8 roundings more
    k = 16 * max(1, c / 16384) + 20
    size = (g.abs() + z.abs() * (g * z).abs().mean(1, keepdim=True)) * rstd.double()[:, None]
    if dres is not None:
        want, size = want + dres.double(), size + dres.double().abs()
    assert ((dx.double() - want).abs() <= k * U * size + UNIT[x.dtype] * want.abs() + TINY[x.dtype]).all()
    if dw is not None:
        want, size = (d.double() * z).sum(0), (d.double() * z).abs().sum(0)
        # a part's rows, the parts of a warp, the warps; of few rows up to 8 a part, 256 parts
        k = r / parts + parts / 8 + 8 if parts else 8 + 256 + 4
        assert ((dw.double() - want).abs() <= k * U * size + UNIT[dw.dtype] * want.abs() + TINY[dw.dtype]).all()


@pytest.mark.parametrize("r,c", SIZES + MANY + [(3000, 200), (1500, 4096), (3000, 999)])
@pytest.mark.parametrize("dtype", TYPES)
def test_grad(r, c, dtype):
    for k, wdtype in enumerate((dtype, torch.float32, dtype)):
        x, d, w = inputs(r, c, dtype, wdtype, 2)
        d = (d * 1e-2).to(dtype)
        if r > 2:
            d[1] = 0  # a position that does not count
        dres = None if k == 0 else torch.randn(r, c, generator=gen(5), device="cuda").mul_(1e-2).to(dtype)
        rstd = apc.rms_norm(x, w)[2]
        # packed; at odds with each other; alike within 16 bytes, but at no boundary
        extra, offset, at = ((0, 0, 0), (5, 3, 0), (8, 5, 5))[k]
        out = strided(torch.zeros_like(x), extra, at)
        dx, dw = apc.rms_norm_grad(strided(d, extra, offset), strided(x, 2 * extra, at), w, rstd, out=out,
                                   dresidual=None if dres is None else strided(dres, extra, offset))
        assert out.as_strided((r, c + extra), (c + extra, 1), out.storage_offset())[:, c:].isnan().all()
        assert dx.dtype == dtype and dw.dtype == wdtype
        parts = apc.operators.rms_norm_grad_workspace(r, c) // c
        check_grad(d, x, w, rstd, dres, dx, dw, parts)
        if r > 2 and dres is None:
            assert (dx[1] == 0).all()
        only, none = apc.rms_norm_grad(d, x, w, rstd, dresidual=dres, weight_grad=False)
        assert none is None
        check_grad(d, x, w, rstd, dres, only, None, parts)


@pytest.mark.parametrize("r,c", [(9, 1000), (300, 1000), (700, 1003), (400, 9000), (400, 9003), (5000, 100), (5000, 500), (7, 20_000), (80, 16_390)])
def test_grad_in_place_and_types(r, c):
    x, d, w = inputs(r, c, torch.bfloat16, torch.bfloat16)
    rstd = apc.rms_norm(x, w)[2]
    dres = d * 0.5
    want = apc.rms_norm_grad(d, x, w, rstd, dresidual=dres, dweight=torch.empty(c, device="cuda"))
    for place in ("dout", "dresidual"):
        a, b = d.clone(), dres.clone()
        got = apc.rms_norm_grad(a, x, w, rstd, dresidual=b, out=a if place == "dout" else b,
                                dweight=torch.empty(c, dtype=torch.half, device="cuda"))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1].half())


@pytest.mark.parametrize("dtype", TYPES)
def test_dx_does_not_depend_on_dweight(dtype):
    """A frozen weight leaves dx's bits as they are, in the ring, by plain loads and where a cluster makes both."""
    for r, c in ((3, 40), (60, 500), (400, 601), (310, 840), (330, 784), (350, 601), (500, 513), (400, 2048), (700, 1003), (20, 12_000), (310, 9001),
                 (4, 17_000), (9000, 90)):
        x, d, w = inputs(r, c, dtype, dtype, 11)
        dres = torch.randn(r, c, generator=gen(6), device="cuda").to(dtype)
        rstd = apc.rms_norm(x, w)[2]
        for extra, offset in ((0, 0), (8, 5)):
            given = strided(d, extra, offset), strided(x, extra, offset), w, rstd
            for k in (dict(), dict(dresidual=strided(dres, extra, offset))):
                out = [strided(torch.zeros_like(x), extra, offset) for _ in range(2)]
                apc.rms_norm_grad(*given, out=out[0], **k)
                apc.rms_norm_grad(*given, out=out[1], weight_grad=False, **k)
                assert torch.equal(*out)


@pytest.mark.parametrize("dtype", TYPES)
def test_pitches_of_what_is_not_there(dtype):
    """Without a residual its pitch says nothing, not about which kernel runs either."""
    r, c = 200, 1000
    x, d, w = inputs(r, c, dtype, dtype, 17)
    kind = apc.operators._DTYPE[dtype]
    handle = torch.cuda.current_stream().cuda_stream
    rstd, dw = torch.empty(r, device="cuda"), torch.empty_like(w)
    work = torch.empty(apc.operators.rms_norm_grad_workspace(r, c), device="cuda")
    want = None
    for pitch in (0, c, 5, -3, 1 << 62):
        y, dx = torch.empty_like(x), torch.empty_like(x)
        norm = apc.operators._pack_norm(x.data_ptr(), 0, w.data_ptr(), 0, r, c, c, pitch, pitch, kind, kind, 1e-6)
        apc._check(apc.library().apc_rms_norm(norm, y.data_ptr(), c, rstd.data_ptr(), handle))
        grad = apc.operators._pack_norm_grad(d.data_ptr(), x.data_ptr(), w.data_ptr(), 0, rstd.data_ptr(), r, c, c, c, pitch, kind, kind)
        apc._check(apc.library().apc_rms_norm_grad(grad, dx.data_ptr(), c, dw.data_ptr(), kind, work.data_ptr() if work.numel() else None, handle))
        got = y, rstd.clone(), dx, dw.clone()
        want = got if want is None else want
        for p, q in zip(got, want):
            assert torch.equal(p, q)


def test_grad_against_differences():
    """The formula is the derivative of the forward definition, in 64 bits; the kernel follows the formula."""
    x, d, w = inputs(4, 96, torch.float32, torch.float32)
    eps = 1e-3
    _, h, rstd = apc.rms_norm(x, w, eps=eps)
    dx, dw = apc.rms_norm_grad(d, x, w, rstd)

    def loss(x, w):
        return (x / (x.square().mean(1, keepdim=True) + eps).sqrt() * w * d.double()).sum()

    x, w = x.double(), w.double()
    step = 1e-6
    for at, grad in ((x, dx), (w, dw)):
        for i in range(0, at.numel(), 17):
            e = torch.zeros_like(at).view(-1)
            e[i] = step
            e = e.view_as(at)
            up, down = (loss(x + s * e, w) if at is x else loss(x, w + s * e) for s in (1, -1))
            # differences: truncation step^2, cancellation 2^-53 |loss| / step; the kernel: a few hundred u
            assert abs((up - down) / (2 * step) - grad.view(-1)[i].double()) <= 1e-4 * (1 + abs(grad.view(-1)[i].item()))


def test_on_another_stream_and_in_a_graph():
    x, res, w = inputs(300, 4096, torch.bfloat16, torch.bfloat16)

    def step(**kw):
        *q, h, rstd = apc.rms_norm_fp8(x, w, residual=res, transposed=True, **kw)
        return [*q, h, rstd, *apc.rms_norm_grad(res, h, w, rstd, dresidual=x, **kw)]

    want = step()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = step(stream=s)
    torch.cuda.current_stream().wait_stream(s)
    for a, b in zip(got, want):
        assert torch.equal(a.float(), b.float())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step()
    x.copy_(res.flip(0))
    res.mul_(0.5)
    want = step()
    for _ in range(2):
        g.replay()
    for a, b in zip(got, want):
        assert torch.equal(a.float(), b.float())


def test_a_whole_step_of_two_replicas(monkeypatch):
    """Norm, product, distillation, products, the norm's gradient, the gradients' norm and the clipped step on one
    stream: the gradients against 64 bits of what each operator was given, and equal digests on any grid."""
    tokens, vocab, hidden, k, eps, most = 500, 1003, 272, 12, 1e-5, 1e-3
    x, res, _ = inputs(tokens, hidden, torch.bfloat16, torch.bfloat16, 9)
    head = torch.randn(vocab, hidden, generator=gen(2), device="cuda").mul_(0.05)
    u, ids = torch.randn(tokens, vocab, generator=gen(3), device="cuda").mul_(3).topk(k, 1)
    weights = torch.full((tokens,), 1.0 / tokens, device="cuda")

    def run():
        p = [head.clone(), torch.ones(hidden, device="cuda")]
        w = [t.bfloat16() for t in p]
        g = [torch.empty_like(t) for t in w]
        m, v = [torch.zeros_like(t) for t in p], [torch.zeros_like(t) for t in p]
        table = apc.prepare_table([apc.TensorEntry(*t, 1000 * i) for i, t in enumerate(zip(p, m, v, g, w))])
        kept = []
        for step in (1, 2):
            x8, xs, x8t, xst, h, rstd = apc.rms_norm_fp8(x, w[1], eps=eps, residual=res, transposed=True)
            w8, ws, w8t, wst = apc.quantize_fp8(w[0], block_rows=128, transposed=True)
            logits = apc.matmul_fp8(x8, xs, w8, ws)
            loss, _, d = apc.distill_loss_grad(logits, ids, u, weights, out=logits)
            d8, ds, d8t, dst = apc.quantize_fp8(d, transposed=True)
            dy = apc.matmul_fp8(d8, ds, w8t, wst)
            apc.matmul_fp8(d8t, dst, x8t, xst, out=g[0])
            dx, _ = apc.rms_norm_grad(dy, h, w[1], rstd, dweight=g[1])
            norm = apc.grad_norm(table)
            old = [t.clone() for t in p]
            digests = apc.commit_step(table, step, grad_norm=norm, max_norm=most)
            kept += [loss, dx, g[0].clone(), g[1].clone(), norm, digests] + [t.clone() for t in p + w]
            if step == 1:
                parts = apc.operators.rms_norm_grad_workspace(tokens, hidden) // hidden
                check_grad(dy, h, w[1], rstd, None, dx, g[1], parts)
                want = torch.cat([t.double().view(-1) for t in g]).norm()
                assert norm.item() > most and abs(norm.item() - want.item()) <= 2.0 ** -20 * want.item()
                # AdamW's first step from zero moments: every parameter moves by lr at most, and by nothing without a gradient
                for a, b, q in zip(old, p, g):
                    moved = (b - a * (1 - 3e-4 * 0.1)).abs()
                    assert (moved <= 3e-4 * 1.001 + a.abs() * 2.0 ** -22).all() and (moved[q != 0] > 0).float().mean() > 0.9
        return kept

    a = run()
    for limit in ("3", "50"):
        monkeypatch.setenv("APC_GRID_LIMIT", limit)
        for s, t in zip(a, run()):
            assert torch.equal(s, t)
    monkeypatch.delenv("APC_GRID_LIMIT")
    assert apc.device_status() == 0
