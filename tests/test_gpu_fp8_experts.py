"""Products of experts' rows on the GPU against 64-bit forms: rows dealt evenly and not at all evenly, experts without rows, odd sizes, pairs of no
expert, strides, every pair of formats."""
import pytest

torch = pytest.importorskip("torch")
import experts_reference as eref
import lowbit_reference as ref

pytestmark = pytest.mark.gpu
E4, E5 = torch.float8_e4m3fn, torch.float8_e5m2
F32, BF, HF = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ctx():
    import paper_2509_05576_amd as fobq
    c = fobq.Ctx(0)
    yield c
    c.close()


def _matrix(ctx, rows, cols, fmt, per, seed, outliers=True):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, cols), generator=g)
    if outliers:
        x *= 1 + 9 * (torch.rand((cols,), generator=g) < 0.02)
    return ctx.fp8_quantize(x.cuda(), fmt, per)


def _weights(ctx, experts, n, k, fmt, per, seed=0):
    import paper_2509_05576_amd as fobq
    w = fobq.Fp8Experts.empty(experts, n, k, fmt, per)
    w.values.view(torch.uint8).fill_(0x7e)
    g = torch.Generator().manual_seed(seed)
    for e in range(experts):
        ctx.fp8_quantize((torch.randn((n, k), generator=g) * 0.1).cuda(), fmt, per, out=w.expert(e))
    return w


def _routing(counts, top_k, seed=0, none=0):
    """Pairs in any order, count[e] of them expert e's, `none` of no expert (a token may have an expert twice here: products do not mind)."""
    import paper_2509_05576_amd as fobq
    g = torch.Generator().manual_seed(seed)
    flat = torch.cat([torch.full((c,), e) for e, c in enumerate(counts)] + [torch.full((none,), -1)]).to(torch.int32)
    flat = flat[torch.randperm(len(flat), generator=g)]
    assert len(flat) % top_k == 0
    chosen = flat.reshape(-1, top_k)
    starts, pairs, places = eref.places(chosen, len(counts))
    return fobq.Routing(chosen.cuda(), torch.rand(chosen.shape, generator=g).cuda(), starts.cuda(), pairs.cuda(), places.cuda())


def check(ctx, a, w, r, dtype, packed, **kw):
    rows, n = r.pairs.shape[0], w.values.shape[1]
    out = torch.full((rows, n + 3), 5.0, dtype=dtype, device="cuda")[:, 1:1 + n]
    got = ctx.fp8_expert_matmul(a, w, r, packed=packed, out=out, **kw)
    assert got is out
    values, starts, pairs = a.values.cpu(), r.starts.tolist(), r.pairs.cpu()
    dense = ref.expand(values.double(), a.scales.cpu(), 1)
    out = out.cpu()
    for e in range(len(starts) - 1):
        lo, hi = starts[e], starts[e + 1]
        if lo == hi:
            continue
        rows_a = dense[lo:hi] if packed else dense[(pairs[lo:hi] // r.places.shape[1]).long()]
        m = w.expert(e)
        y, bound = ref.matmul(rows_a, ref.expand(m.values.cpu().double(), m.scales.cpu(), m.rows_per_scale), dtype)
        assert ((out[lo:hi].double() - y).abs() <= bound).all(), (e, lo, hi)
    assert bool((out[starts[-1]:] == 5).all())              # rows of no expert are left alone
    return got


COUNTS = [[1], [0, 3, 0], [5, 0, 1, 16, 17, 0, 1], [64, 65, 0, 0, 128, 129, 1, 63], [0, 300, 0, 2], [1] * 70, [0] * 63 + [9] + [0] * 100 + [70, 1]]


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("counts", COUNTS)
def test_rows_dealt(ctx, counts, dtype, packed):
    n, k = 130, 300
    top_k = next(t for t in (3, 2, 1) if sum(counts) % t == 0)
    r = _routing(counts, top_k)
    for per in (1, 128):
        w = _weights(ctx, len(counts), n, k, E4, per)
        check(ctx, _matrix(ctx, sum(counts) if packed else sum(counts) // top_k, k, E4, 1, 1), w, r, dtype, packed)


@pytest.mark.parametrize("n,k", [(1, 1), (3, 16), (64, 100), (65, 128), (16, 129), (200, 640), (257, 2304), (1000, 65)])
@pytest.mark.parametrize("counts", [[2, 0, 3], [40, 21, 5], [150, 0, 90]])
def test_sizes(ctx, counts, n, k):
    r = _routing(counts, 1 if sum(counts) % 2 else 2)
    for fa, fb, per, dtype in ((E4, E4, 128, BF), (E5, E4, 1, HF), (E4, E5, 128, F32), (E5, E5, 1, F32), (E5, E5, 128, BF)):
        w = _weights(ctx, len(counts), n, k, fb, per)
        check(ctx, _matrix(ctx, sum(counts) // r.places.shape[1], k, fa, 1, 2), w, r, dtype, False)


@pytest.mark.parametrize("per_expert", [1, 8, 16, 17, 40, 100, 200, 400, 700])
@pytest.mark.parametrize("per", [1, 128])
def test_every_tile(ctx, per_expert, per):
    """About as many rows as lead to each of the forms, in experts of very unlike sizes."""
    counts = [per_expert * 2 + 3, 0, per_expert, max(0, per_expert - 5), 1, per_expert]
    if sum(counts) % 2:
        counts[0] += 1
    r = _routing(counts, 2, none=4)
    for n, k, dtype in ((520, 512, BF), (520, 640, F32), (300, 260, HF)):
        w = _weights(ctx, len(counts), n, k, E4, per)
        check(ctx, _matrix(ctx, r.pairs.shape[0] // 2, k, E4, 1, 3), w, r, dtype, False)
        check(ctx, _matrix(ctx, r.pairs.shape[0], k, E4, 1, 4), w, r, dtype, True)


@pytest.mark.parametrize("form,counts,n,per,dtype", [
    ((16, 16), [1, 3, 0, 2], 200, 128, BF), ((16, 16), [1, 0, 17, 2], 200, 1, F32), ((64, 64), [20, 5, 64, 31], 1000, 128, BF), ((64, 64), [20, 5, 64, 31], 1000, 1, F32),
    ((64, 128), [70, 0, 300, 130], 4100, 128, HF), ((64, 128), [70, 0, 300, 130], 4100, 1, F32), ((128, 256), [500, 31, 0, 669], 4100, 128, BF),
    ((128, 256), [129, 450, 64, 557], 4100, 1, HF), ((128, 128), [1500, 500, 7, 1993], 4100, 128, F32), ((128, 128), [1500, 500, 7, 1993], 4100, 1, F32),
    ((256, 256), [1000, 64, 700, 636], 4100, 128, BF), ((256, 256), [129, 1281, 193, 797], 4100, 128, HF)])
@pytest.mark.parametrize("k", [128, 300, 2100])
def test_forms(ctx, form, counts, n, per, dtype, k):
    """Each form of the product, as the rules choose it, with tiles that are full, that have a quarter, half or three of their rows, and one."""
    import paper_2509_05576_amd as fobq
    types = {F32: 0, BF: 1, HF: 2}
    rows = sum(counts)
    assert fobq.fobq_debug_plan(fobq.PLAN_EXPERTS, [torch.cuda.get_device_properties(0).multi_processor_count, rows, len(counts), n, k, types[dtype], per], 3)[:2] == list(form)
    r = _routing(counts, 1)
    check(ctx, _matrix(ctx, rows, k, E4, 1, 5), _weights(ctx, len(counts), n, k, E4, per), r, dtype, False)


def test_pairs_of_no_expert(ctx):
    for counts, none in (([10, 0, 4], 4), ([0, 0], 8), ([100, 70], 30)):
        r = _routing(counts, 2, none=none)
        w = _weights(ctx, len(counts), 70, 256, E4, 128)
        check(ctx, _matrix(ctx, r.pairs.shape[0] // 2, 256, E4, 1, 1), w, r, BF, False)


def test_a_product_of_no_columns(ctx):
    """Zeros for the experts' rows, no others."""
    import paper_2509_05576_amd as fobq
    r = _routing([5, 0, 2], 1, none=2)
    w = fobq.Fp8Experts(torch.empty((3, 10, 0), dtype=E4, device="cuda"), torch.empty((3, 0, 1), device="cuda"), 128)
    a = fobq.Fp8Matrix(torch.empty((9, 0), dtype=E4, device="cuda"), torch.empty((0, 9), device="cuda"))
    out = torch.full((9, 10), 3.0, device="cuda")
    ctx.fp8_expert_matmul(a, w, r, out=out)
    assert bool((out[:7] == 0).all()) and bool((out[7:] == 3).all())


def test_not_finite(ctx):
    """A NaN in a token's row reaches that token's packed rows, one in an expert's weights that expert's column."""
    counts = [30, 7, 25]
    r = _routing(counts, 2)
    for dtype in (BF, F32):
        a, w = _matrix(ctx, 31, 300, E4, 1, 1), _weights(ctx, 3, 90, 300, E4, 128)
        a.values.view(torch.uint8)[4, 299] = 0x7f
        w.values.view(torch.uint8)[1, 77, 0] = 0x7f
        out = ctx.fp8_expert_matmul(a, w, r, dtype).cpu().isnan()
        pairs = r.pairs.cpu()
        want = torch.zeros_like(out)
        want[pairs // 2 == 4] = True
        want[30:37, 77] = True
        assert torch.equal(out, want)


def test_pairs_that_are_none(ctx):
    """starts and pairs that are not as they should be: kept inside, and rows without a row of A are not written."""
    import paper_2509_05576_amd as fobq
    a, w = _matrix(ctx, 10, 256, E4, 1, 1), _weights(ctx, 3, 64, 256, E4, 128)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    pairs = [3, -1, 7, 20, 2 ** 31 - 1, -2 ** 31, 19, 0, 4, 5]
    for starts in ([0, 4, 4, 10], [-7, 3, 2 ** 31 - 1, 2 ** 31 - 1], [0, 10, 3, 10], [9, 8, 7, 6], [2 ** 31 - 1] * 4, [-2 ** 31] * 4):
        r = fobq.Routing(None, None, i32(starts), i32(pairs + pairs), torch.zeros((10, 2), dtype=torch.int32, device="cuda"))
        out = torch.full((20, 64), 5.0, device="cuda")
        ctx.fp8_expert_matmul(a, w, r, out=out)
        bad = torch.tensor([p < 0 or p >= 20 for p in pairs + pairs])
        assert bool((out.cpu()[bad] == 5).all())


def test_far_apart(ctx):
    """Experts and rows whose offsets pass 32 bits (values that are not read are not initialized)."""
    import paper_2509_05576_amd as fobq
    counts, n, k = [3, 0, 20], 48, 256
    r = _routing(counts, 1)
    w = _weights(ctx, 3, n, k, E4, 128)
    apart = torch.empty((3 << 31,), dtype=torch.uint8, device="cuda").view(E4)
    far = fobq.Fp8Experts(apart.as_strided((3, n, k), ((1 << 31) + 1024, 1 << 20, 1)), w.scales, 128)
    far.values.view(torch.uint8).copy_(w.values.view(torch.uint8))
    a = _matrix(ctx, 23, k, E4, 1, 1)
    want = ctx.fp8_expert_matmul(a, w, r)
    assert torch.equal(ctx.fp8_expert_matmul(a, far, r), want)
    wide = apart.as_strided((23, k), ((1 << 24) - 16, 1))                # rows of A almost 2^24 bytes apart
    many = apart.as_strided((600, k), ((1 << 23) + 16, 1))               # the last ones behind 2^32
    wide.view(torch.uint8).copy_(a.values.view(torch.uint8))
    assert torch.equal(ctx.fp8_expert_matmul(fobq.Fp8Matrix(wide, a.scales), w, r), want)
    last = torch.arange(577, 600, device="cuda")
    many.view(torch.uint8)[last] = a.values.view(torch.uint8)
    scales = torch.zeros((2, 600), device="cuda")
    scales[:, last] = a.scales
    moved = fobq.Routing(r.chosen, r.weights, r.starts, r.pairs + 577, torch.zeros((600, 1), dtype=torch.int32, device="cuda"))
    moved.pairs = torch.cat((moved.pairs, torch.full((577,), -1, dtype=torch.int32, device="cuda")))
    near = torch.zeros((600, k), dtype=torch.uint8, device="cuda")       # (another form than that of 23 rows: compared with itself)
    near[last] = a.values.view(torch.uint8)
    want = ctx.fp8_expert_matmul(fobq.Fp8Matrix(near.view(E4), scales), w, moved)[:23]
    assert torch.equal(ctx.fp8_expert_matmul(fobq.Fp8Matrix(many, scales), w, moved)[:23], want) and float(want.float().abs().max()) > 1


def test_refusals(ctx):
    import paper_2509_05576_amd as fobq
    r = _routing([4, 6], 2)
    a, w = _matrix(ctx, 5, 256, E4, 1, 1), _weights(ctx, 2, 64, 256, E4, 128)
    full = _matrix(ctx, 10, 256, E4, 1, 1)
    bad = fobq.Fp8Experts
    for call in (lambda: ctx.fp8_expert_matmul(full, w, r), lambda: ctx.fp8_expert_matmul(a, w, r, packed=True), lambda: ctx.fp8_expert_matmul(a, w, r, torch.int32),
                 lambda: ctx.fp8_expert_matmul(_matrix(ctx, 5, 128, E4, 1, 1), w, r), lambda: ctx.fp8_expert_matmul(a, w, _routing([4, 3, 3], 2)),
                 lambda: ctx.fp8_expert_matmul(a, bad(w.values, w.scales, 1), r), lambda: ctx.fp8_expert_matmul(a, bad(w.values, w.scales[:, :1], 128), r),
                 lambda: ctx.fp8_expert_matmul(a, bad(w.values.view(torch.uint8), w.scales, 128), r),
                 lambda: ctx.fp8_expert_matmul(a, bad(w.values.transpose(1, 2), w.scales, 128), r),
                 lambda: ctx.fp8_expert_matmul(a, w, r, out=torch.empty((10, 63), device="cuda")),
                 lambda: ctx.fp8_expert_matmul(a, w, fobq.Routing(None, None, r.starts.cpu(), r.pairs, r.places))):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: ctx.fp8_expert_matmul(ctx.fp8_quantize(torch.zeros((5, 256), device="cuda"), rows_per_scale=128), w, r),
                 lambda: ctx.fp8_expert_matmul(a, bad(torch.zeros((2, 64, 264), dtype=torch.uint8, device="cuda").view(E4)[:, :, :256], w.scales, 128), r)):
        with pytest.raises(fobq.FobqError):
            call()
    none = fobq.Routing(None, None, r.starts, r.pairs[:0], r.places[:0])
    assert ctx.fp8_expert_matmul(fobq.Fp8Matrix(a.values[:0], a.scales[:, :0]), w, none).shape == (0, 64)
