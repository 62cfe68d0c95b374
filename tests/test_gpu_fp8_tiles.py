"""Products in the tiles that large calls take, over enough blocks that every stage is used again: all results against 64 bits, for every pair
of formats, both layouts of scales and all three types."""
import pytest

torch = pytest.importorskip("torch")
import lowbit_reference as ref

pytestmark = pytest.mark.gpu
E4, E5 = torch.float8_e4m3fn, torch.float8_e5m2
TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
# rows and columns of the result: those that whole tiles of 128 and 256 just do not cover, with odd edges; those that 64 take
SIZES = [(2900, 2901), (2050, 2047), (500, 411)]


@pytest.fixture(scope="module")
def ctx():
    import paper_2509_05576_amd as fobq
    c = fobq.Ctx(0)
    yield c
    c.close()


def matrix(rows, cols, seed, spread):
    g = torch.Generator(device="cuda").manual_seed(seed)
    # blocks of different size, so that one block's scale or values in another's place are far off
    x = torch.randn((rows, cols), generator=g, device="cuda") * torch.exp(spread * torch.randn((rows, -(-cols // 128)), generator=g, device="cuda")
                                                                         ).repeat_interleave(128, 1)[:, :cols]
    return x


def expanded(m):
    s = m.scales.double().t().repeat_interleave(m.rows_per_scale, 0)[:m.values.shape[0]].repeat_interleave(128, 1)[:, :m.values.shape[1]]
    return m.values.double() * s


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("fa", [E4, E5])
@pytest.mark.parametrize("fb", [E4, E5])
@pytest.mark.parametrize("per", [1, 128])
@pytest.mark.parametrize("k", [640, 1000, 1408])
@pytest.mark.parametrize("m,n", SIZES)
def test_many_blocks(ctx, m, n, k, per, fa, fb, dtype):
    import paper_2509_05576_amd as fobq
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    tile = fobq.fobq_debug_plan(fobq.PLAN_FP8_MATMUL, [cus, m, n, k, TYPES[dtype], per], 5)[0]
    if cus == 256:
        assert tile == (64 if m == 500 else 256 if m == 2900 and per == 128 and dtype != torch.float32 else 128)
    a, b = ctx.fp8_quantize(matrix(m, k, m + k, 0.5), fa), ctx.fp8_quantize(matrix(n, k, n, 0.5) * k ** -0.5, fb, per)
    got = ctx.fp8_matmul(a, b, dtype)
    y, bound = ref.matmul(expanded(a), expanded(b), dtype)
    off = (got.double() - y).abs()
    assert bool((off <= bound).all()), float((off / bound).max())
    assert torch.equal(ctx.fp8_matmul(a, b, dtype), got)
