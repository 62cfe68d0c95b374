"""Matrices in 8-bit floating point blocks on the GPU: their quantizer, a quantized layer as one, and the product, against 64-bit
forms."""
import math

import pytest

torch = pytest.importorskip("torch")
import lowbit_reference as ref

pytestmark = pytest.mark.gpu
E4, E5 = torch.float8_e4m3fn, torch.float8_e5m2
SOURCES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def ctx():
    import paper_2509_05576_amd as fobq
    c = fobq.Ctx(0)
    yield c
    c.close()


def _x(rows, cols, dtype, seed, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, cols), generator=g) * torch.exp(spread * torch.randn((rows, 1), generator=g))
    return x.to(dtype)


def _same(got, want):
    return torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(0.0), want.nan_to_num(0.0))


@pytest.mark.parametrize("per", [1, 128])
@pytest.mark.parametrize("fmt", [E4, E5])
@pytest.mark.parametrize("dtype", SOURCES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 128), (3, 130), (129, 255), (200, 1000), (128, 512), (257, 641)])
def test_quantize(ctx, rows, cols, dtype, fmt, per):
    x = _x(rows, cols, dtype, rows + cols)
    m = ctx.fp8_quantize(x.cuda(), fmt, per)
    q, scales = ref.quantize(x, fmt, per)
    assert m.values.dtype == fmt and m.values.shape == x.shape and m.values.stride(0) % 16 == 0
    got = m.values.cpu().double()
    assert (m.scales.cpu().double() - scales).abs().le(scales * 2.0 ** -24 * 1.0001).all()
    if dtype != torch.float32:
        # few bits: no quotient is nearer to a border than 2^-20 unless it lies on it
        assert _same(got, ref.round8(q, fmt))
    else:
        # the quotient to 2 units of fp32, then half a step
        assert (got - q).abs().le(ref.step8(q, fmt) / 2 + q.abs() * 2 * ref.U * 1.01).all()


@pytest.mark.parametrize("fmt", [E4, E5])
@pytest.mark.parametrize("per", [1, 128])
def test_quantize_extremes(ctx, fmt, per):
    x = torch.zeros((3, 128 * 8), dtype=torch.float32)
    x[:, 128:256] = 3.0e38                       # the largest values
    x[1, 256] = math.inf
    x[1, 384] = math.nan
    x[:, 512:640] = 1.0e-44                      # denormal
    x[:, 640:768] = torch.linspace(-1e-37, 1e-37, 128)
    x[2, 768:896] = torch.linspace(-448, 448, 128)
    x[0, 768] = -0.0
    m = ctx.fp8_quantize(x.cuda(), fmt, per)
    q, scales = ref.quantize(x, fmt, per)
    s = m.scales.cpu().double()
    assert torch.equal(s.isnan(), scales.isnan())
    assert (s - scales).abs().nan_to_num(0.0).le(scales.nan_to_num(0.0) * 2.0 ** -24 * 1.0001).all()
    got = m.values.cpu().double()
    assert torch.equal(got.isnan(), q.isnan())
    assert (got - q).nan_to_num(0.0).abs().le((ref.step8(q.nan_to_num(0.0), fmt) / 2 + q.nan_to_num(0.0).abs() * 2 * ref.U * 1.01)).all()
    assert got.nan_to_num(0.0).abs().max() <= ref.TOP[fmt]


@pytest.mark.parametrize("fmt", [E4, E5])
@pytest.mark.parametrize("per", [1, 128])
def test_quotients_beside_a_border(ctx, fmt, per):
    """Values whose quotients lie on the border of two 8-bit ones, or by it, closer than fp32 tells apart: the side is the exact
    quotient's (x * top against border * largest, both exact in 64 bits), ties to the even one."""
    top, keep = (448.0, 3) if fmt == E4 else (57344.0, 2)
    g = torch.Generator().manual_seed(per)
    most = (torch.rand((1 if per == 128 else 128, 1), generator=g) + 1.0).expand(128, 1).contiguous()
    steps = torch.randint(0, 2 ** keep, (128, 511), generator=g).double()
    power = 2.0 ** torch.randint(-9 if fmt == E4 else -16, 8, (128, 511), generator=g).double()
    low_power = power.clamp(min=2.0 ** -6 if fmt == E4 else 2.0 ** -14)       # below it the values are evenly spaced
    below = torch.where(power < low_power, steps * low_power / 2 ** keep, (2 ** keep + steps) * low_power / 2 ** keep)
    above = below + low_power / 2 ** keep
    border = (below + above) / 2
    x = (border * most.double() / top).float()
    x = torch.stack((x, torch.nextafter(x, x * 2), torch.nextafter(x, x * 0)))[torch.randint(0, 3, x.shape, generator=g), torch.arange(128)[:, None], torch.arange(511)]
    first = torch.arange(511) % 128 == 127                                     # each block's largest value, in its last place
    x[:, first] = most.expand(-1, int(first.sum()))
    x = torch.cat((most, x), 1)[:, :512] * torch.where(torch.rand((128, 512), generator=g) < 0.5, -1.0, 1.0)
    got = ctx.fp8_quantize(x.cuda(), fmt, per).values.cpu().double()
    q, m = x[:, 1:].double().abs() * top, border * most.double()
    want = torch.where((q > m) | ((q == m) & (steps % 2 == 1)), above, below) * x[:, 1:].sign()
    inner = ~first
    assert torch.equal(got[:, 1:][:, inner], want[:, inner])


def test_quantize_strides_and_what_is_behind(ctx):
    import paper_2509_05576_amd as fobq
    wide = _x(70, 301, torch.bfloat16, 5).cuda()
    x = wide[:, 7:294]                           # rows an odd number of elements apart, odd start
    want = ctx.fp8_quantize(x.contiguous())
    values = torch.full((70, 304), 0x11, dtype=torch.uint8, device="cuda")
    scales = torch.full((3, 80), -1.0, device="cuda")
    out = fobq.Fp8Matrix(values.view(E4)[:, :287], scales[:, :70], 1)
    assert ctx.fp8_quantize(x, out=out) is out
    assert torch.equal(out.values.view(torch.uint8), want.values.view(torch.uint8)) and torch.equal(out.scales, want.scales)
    assert (values[:, 287:] == 0x11).all() and (scales[:, 70:] == -1).all()


@pytest.mark.parametrize("r,d,bits,group", [(1, 1, 4, 0), (64, 147, 4, 0), (33, 256, 3, 128), (100, 1024, 2, 256), (7, 2000, 4, 0)])
def test_from_codes_is_the_layer(ctx, r, d, bits, group):
    g = torch.Generator(device="cuda").manual_seed(r + d)
    W = torch.randn((r, d), generator=g, device="cuda") * math.sqrt(2.0 / d)
    X = torch.randn((d, 2 * d + 8), generator=g, device="cuda").relu_()
    ctx.hessian(X)
    layer = ctx.quantize_layer(W, bits=bits, group=group)
    m = ctx.fp8_from_codes(layer.codes, layer.scales, layer.zeros, bits=bits)
    groups = d // group if group else 1
    zero = layer.zeros.repeat_interleave(d // groups, 1)
    assert torch.equal(m.values.float(), layer.codes.float() - zero)
    assert torch.equal(m.scales, layer.scales.repeat_interleave(group // 128, 1).t() if group else layer.scales.t().expand(m.scales.shape))
    # Q is the fp64 scale times the integer, rounded once; the scale that is returned is rounded itself: two half steps of fp32
    off = (ref.expand(m.values.cpu(), m.scales.cpu(), 1) - layer.Q.cpu().double()).abs()
    assert (off <= 2 * ref.U * 1.0001 * layer.Q.cpu().double().abs()).all()


SIZES = [(1, 1, 1), (1, 64, 128), (1, 1000, 2047), (5, 33, 130), (16, 256, 4608), (17, 130, 384), (64, 512, 1024), (100, 129, 257),
         (129, 257, 640), (256, 256, 512), (300, 1000, 2304), (513, 300, 100), (40, 100, 5000), (2100, 2300, 300), (2100, 2301, 300), (4000, 4100, 260)]


@pytest.mark.parametrize("per", [1, 128])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_matmul(ctx, m, n, k, per):
    import paper_2509_05576_amd as fobq
    dtype = [torch.float32, torch.bfloat16, torch.float16][(m + n + k) % 3]
    fa, fb = [(E4, E4), (E4, E5), (E5, E4), (E5, E5)][(m + k) % 4]
    a, b = ctx.fp8_quantize(_x(m, k, torch.float32, m).cuda(), fa), ctx.fp8_quantize(_x(n, k, torch.float32, n, 0.3).cuda() * k ** -0.5, fb, per)
    y, bound = ref.matmul(ref.expand(a.values.cpu(), a.scales.cpu(), 1), ref.expand(b.values.cpu(), b.scales.cpu(), per), dtype)
    got = ctx.fp8_matmul(a, b, dtype)
    assert got.dtype == dtype and tuple(got.shape) == (m, n)
    off = (got.cpu().double() - y).abs()
    assert (off <= bound).all(), (off / bound).max()
    # what is behind the last column of the rows counts as nothing, and the result's neighbours stay as they were
    for t in (a, b):
        if t.values.stride(0) > k:
            whole = torch.as_strided(t.values.view(torch.uint8), (t.values.shape[0], t.values.stride(0)), (t.values.stride(0), 1))
            whole[:, k:] = 0x7F                  # NaN in both types
    out = torch.full((m + 1, n + 3), 7.0, dtype=dtype, device="cuda")
    ctx.fp8_matmul(a, b, out=out[:m, 1:n + 1])
    assert torch.equal(out[:m, 1:n + 1], got)
    assert (out[m] == 7).all() and (out[:, 0] == 7).all() and (out[:, n + 1:] == 7).all()


@pytest.mark.parametrize("fa", [E4, E5])
@pytest.mark.parametrize("fb", [E4, E5])
@pytest.mark.parametrize("m", [1, 40, 200])
def test_matmul_every_value(ctx, fa, fb, m):
    """All finite 8-bit values, the largest and the smallest, one product at a time."""
    import paper_2509_05576_amd as fobq
    codes = torch.arange(256, dtype=torch.uint8)
    va, vb = codes.view(fa), codes.view(fb)
    va, vb = va[va.float().isfinite()], vb[vb.float().isfinite()]
    a, b = torch.zeros((m, 128), dtype=torch.uint8), torch.zeros((256, 128), dtype=torch.uint8)
    for i in range(m):
        a[i, (5 * i) % 128] = va.view(torch.uint8)[(37 * i) % len(va)]
        a[i, (5 * i + 1) % 128] = va.view(torch.uint8)[(37 * i + 11) % len(va)]
    for j in range(256):
        b[j] = vb.view(torch.uint8)[(j + torch.arange(128) * 3) % len(vb)]
    one = lambda n, per: torch.ones((1, -(-n // per)), device="cuda")  # noqa: E731
    got = ctx.fp8_matmul(fobq.Fp8Matrix(a.cuda().view(fa), one(m, 1), 1), fobq.Fp8Matrix(b.cuda().view(fb), one(256, 128), 128), torch.float32)
    y, bound = ref.matmul(a.view(fa).double(), b.view(fb).double(), torch.float32)
    assert ((got.cpu().double() - y).abs() <= bound).all()


def test_matmul_nan_and_inf_stay_in_their_rows(ctx):
    a = _x(130, 300, torch.float32, 1)
    a[3, 7] = math.nan
    b = _x(140, 300, torch.float32, 2)
    b[5, 290] = math.inf
    y = ctx.fp8_matmul(ctx.fp8_quantize(a.cuda()), ctx.fp8_quantize(b.cuda()), torch.float32).cpu()
    bad = torch.zeros((130, 140), dtype=torch.bool)
    bad[3], bad[:, 5] = True, True
    assert torch.equal(y.isnan(), bad)


def test_empty_products(ctx):
    import paper_2509_05576_amd as fobq
    mat = lambda r, c: fobq.Fp8Matrix(torch.zeros((r, -(-c // 16) * 16), dtype=torch.uint8, device="cuda").view(E4)[:, :c],  # noqa: E731
                                      torch.ones((-(-c // 128), r), device="cuda"), 1)
    assert ctx.fp8_matmul(mat(0, 64), mat(5, 64)).shape == (0, 5)
    assert ctx.fp8_matmul(mat(4, 64), mat(0, 64)).shape == (4, 0)
    assert torch.equal(ctx.fp8_matmul(mat(4, 0), mat(5, 0), torch.float32), torch.zeros((4, 5), device="cuda"))
    assert ctx.fp8_quantize(torch.zeros((0, 40), device="cuda")).values.shape == (0, 40)


def test_a_quantized_layer_runs(ctx):
    """The calls together: quantize a layer, hold it in 8 bits, run it on quantized activations."""
    g = torch.Generator(device="cuda").manual_seed(9)
    W = torch.randn((96, 512), generator=g, device="cuda") * 0.06
    X = torch.randn((512, 2000), generator=g, device="cuda").relu_()
    ctx.hessian(X)
    layer = ctx.quantize_layer(W, bits=4, group=128)
    weights = ctx.fp8_from_codes(layer.codes, layer.scales, layer.zeros)
    acts = ctx.fp8_quantize(X.t().contiguous().to(torch.bfloat16))
    y = ctx.fp8_matmul(acts, weights, torch.float32).cpu()
    x, w = ref.expand(acts.values.cpu(), acts.scales.cpu(), 1), layer.Q.cpu().double()
    want, bound = ref.matmul(x, w, torch.float32)
    # the weights are Q to two half steps of fp32 (the scales are returned in fp32)
    assert ((y.double() - want).abs() <= bound + 2.001 * ref.U * (x.abs() @ w.abs().t())).all()
    # e4m3 activations: 2^-4 each at most, taken together well under 3 percent
    assert (y.double() - X.t().double().cpu() @ layer.Q.cpu().double().t()).norm() < 0.03 * y.double().norm()


def test_refusals(ctx):
    import paper_2509_05576_amd as fobq
    x = torch.zeros((4, 256), device="cuda")
    m = ctx.fp8_quantize(x)
    with pytest.raises(TypeError):
        ctx.fp8_quantize(x.cpu())
    with pytest.raises(TypeError):
        ctx.fp8_quantize(x.t())
    with pytest.raises(TypeError):
        ctx.fp8_quantize(x.double())
    with pytest.raises(TypeError):
        ctx.fp8_quantize(x, rows_per_scale=64)
    with pytest.raises(TypeError):
        ctx.fp8_matmul(m, ctx.fp8_quantize(torch.zeros((4, 128), device="cuda")))
    with pytest.raises(TypeError):
        ctx.fp8_matmul(m, m, torch.float64)
    with pytest.raises(fobq.FobqError) as e:
        ctx.fp8_matmul(ctx.fp8_quantize(x, rows_per_scale=128), m)
    assert e.value.code == fobq.EINVAL and "scale per row" in str(e.value)
    odd = torch.zeros((4, 264), dtype=torch.uint8, device="cuda").view(E4)
    with pytest.raises(fobq.FobqError) as e:
        ctx.fp8_matmul(fobq.Fp8Matrix(odd[:, :256], m.scales, 1), m)
    assert "multiple of 16" in str(e.value)
    with pytest.raises(fobq.FobqError) as e:
        ctx.fp8_matmul(fobq.Fp8Matrix(torch.zeros((4, 272), dtype=torch.uint8, device="cuda").view(E4)[:, 8:264], m.scales, 1), m)
    assert "aligned" in str(e.value)
    codes, s = torch.zeros((4, 256), dtype=torch.uint8, device="cuda"), torch.ones((4, 4), device="cuda")
    with pytest.raises(fobq.FobqError):
        ctx.fp8_from_codes(codes, s, s)          # groups of 64
    with pytest.raises(fobq.FobqError):
        ctx.fp8_from_codes(codes, s[:, :1].contiguous(), s[:, :1].contiguous(), bits=8)
    lib = fobq.load_library()
    import ctypes
    a = ref.Fp8Struct.from_buffer_copy(fobq.binding._fp8(ctx.handle, m, "A")[0])
    y = torch.zeros((4, 4), device="cuda")
    call = lambda a, b, ld: lib.fobq_fp8_matmul(ctx.handle, ctypes.byref(a), ctypes.byref(b), y.data_ptr(), 0, ld, None, 0)  # noqa: E731
    assert call(a, a, 4) == fobq.OK and call(a, a, 3) == fobq.EINVAL
    for field, value in [("rows", -1), ("cols", 257), ("ld", 250), ("ld_scales", 3), ("rows_per_scale", 2), ("format", 2), ("values", None), ("scales", None)]:
        b = ref.Fp8Struct.from_buffer_copy(fobq.binding._fp8(ctx.handle, m, "B")[0])
        setattr(b, field, value)
        assert call(a, b, 4) == fobq.EINVAL, field
    big = ref.Fp8Struct.from_buffer_copy(fobq.binding._fp8(ctx.handle, m, "A")[0])
    need = ctypes.c_int64(0)
    assert lib.fobq_fp8_matmul_workspace(ctx.handle, 128, 128, 1 << 20, 1, ctypes.byref(need)) == fobq.OK and need.value > 0
    assert lib.fobq_fp8_matmul_workspace(ctx.handle, 1, -1, 128, 1, ctypes.byref(need)) == fobq.EINVAL
    torch.cuda.synchronize()
