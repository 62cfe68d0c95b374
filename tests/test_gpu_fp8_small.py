"""Small values in 8-bit blocks: far below the largest of their block."""
import pytest

torch = pytest.importorskip("torch")
import lowbit_reference as ref

pytestmark = pytest.mark.gpu
E4, E5 = torch.float8_e4m3fn, torch.float8_e5m2


@pytest.fixture(scope="module")
def ctx():
    import paper_2509_05576_amd as fobq
    c = fobq.Ctx(0)
    yield c
    c.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("fmt", [E4, E5])
@pytest.mark.parametrize("per", [1, 128])
def test_values_that_vanish_beside_a_large_one(ctx, fmt, per, dtype):
    """Quotients from where 8 bits hold them to far below the smallest fp32 number: what rounds to 0 is 0, and nothing is NaN."""
    tiny = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps       # the smallest denormal
    small = torch.tensor([tiny, 2 * tiny, 1e-40, 2.0 ** -126, 1e-30, 1e-20, 1e-10, 1e-5, 1.0, 0.0])
    most = [1.0, 1024.0, 4096.0, 1e20, 1e30, 3e38, 1e-4, 1e-30]
    x = torch.zeros((7, 128 * len(most)))
    for j, m in enumerate(most):
        x[:, 128 * j:128 * j + 10] = small.clamp(max=m)
        x[:, 128 * j + 10:128 * j + 20] = -small.clamp(max=m)
        x[:, 128 * j + 40], x[:, 128 * j + 41] = m, -m
    x = x.to(dtype)
    got = ctx.fp8_quantize(x.cuda(), fmt, per)
    assert not got.values.isnan().any() and not got.scales.isnan().any()
    values = got.values.cpu().double()
    q, _ = ref.quantize(x, fmt, per)
    # the nearest ones; an fp32 quotient may be next to a border by a rounding
    assert (values - q).abs().le(ref.step8(q, fmt) / 2 + q.abs() * 2 * ref.U * 1.01).all()
    # half of the smallest value is the border to 0: 2^-9 in e4m3 (exponent -6, 3 bits), 2^-16 in e5m2 (-14, 2 bits)
    keep, low = ref.KEEP_LOW[fmt]
    below = 2.0 ** (low - keep - 1)
    vanish = (q.abs() < below * 0.99) & (x != 0)
    assert (values[vanish] == 0).all() and vanish.sum() > 7 * 20
    # and through a product: the row that holds them is finite
    y = ctx.fp8_matmul(ctx.fp8_quantize(x[:, :640].contiguous().cuda(), fmt), ctx.fp8_quantize(torch.ones((3, 640), device="cuda")), torch.float32)
    assert y.isfinite().all()


@pytest.mark.parametrize("power", [-30, -41, -60, -90, -110, -117])
@pytest.mark.parametrize("fmt", [E4, E5])
@pytest.mark.parametrize("per", [1, 128])
def test_quotients_beside_a_border_in_blocks_of_small_values(ctx, fmt, per, power):
    """Quotients on the border of two 8-bit values, or by it, closer than fp32 tells apart, where the block's largest is 2^power: the side is
    the exact quotient's (x * top against border * largest, both exact in 64 bits), ties to the even one."""
    top, keep = (448.0, 3) if fmt == E4 else (57344.0, 2)
    g = torch.Generator().manual_seed(per - power)
    most = ((torch.rand((1 if per == 128 else 128, 1), generator=g) + 1.0) * 2.0 ** power).expand(128, 1).contiguous()
    most = most.clamp(min=top * 2.0 ** -125)                       # (below it the scale is the smallest one, not the largest value's)
    low = -6 if fmt == E4 else -14
    power_of = 2.0 ** torch.randint(low - 1, 8, (128, 512), generator=g).double()
    steps, at_least = torch.randint(0, 2 ** keep, (128, 512), generator=g).double(), power_of.clamp(min=2.0 ** low)
    below = torch.where(power_of < at_least, steps * at_least / 2 ** keep, (2 ** keep + steps) * at_least / 2 ** keep)
    above = below + at_least / 2 ** keep
    border = (below + above) / 2
    x = (border * most.double() / top).float()
    near = torch.stack((x, torch.nextafter(x, x * 2), torch.nextafter(x, x * 0)))
    x = near.gather(0, torch.randint(0, 3, (1, 128, 512), generator=g))[0]
    last = torch.arange(512) % 128 == 127                          # each block's largest, in its last place
    x[:, last] = most.expand(-1, 4)
    x = x * torch.where(torch.rand((128, 512), generator=g) < 0.5, -1.0, 1.0)
    got = ctx.fp8_quantize(x.cuda(), fmt, per).values.cpu().double()
    q, m = x.double().abs() * top, border * most.double()
    want = torch.where((q > m) | ((q == m) & (steps % 2 == 1)), above, below) * x.sign()
    assert torch.equal(got[:, ~last], want[:, ~last])
    assert (got[:, last].abs() == top).all()
