"""The scale of a cache row: the range over 15, rounded up to bf16, also where the two ends of the range are of very different size."""
import pytest

torch = pytest.importorskip("torch")
import lowbit_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    import paper_2509_05576_amd as fobq
    c = fobq.Ctx(0)
    yield c
    c.close()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_a_range_just_above_fifteen_steps(ctx, dim, dtype):
    """One end is 15 bf16 numbers' worth exactly, the other a little beyond 0: less than fp32 adds to the first one, but 15 steps of that
    number do not reach any more."""
    import paper_2509_05576_amd as fobq
    ends = [(m * 15 / 16) * 2.0 ** e for m in (1.0, 17 / 16) for e in (-3, 0, 1, 4)]          # 15 times 2^n or 17/16 of it: 8 bits
    small = [2.0 ** -14, 2.0 ** -20, 2.0 ** -24] + ([2.0 ** -30, 2.0 ** -40, 3 * 2.0 ** -38] if dtype == torch.bfloat16 else [])
    rows = []
    for end in ends:
        for s in small + [0.0]:
            for sign in (1.0, -1.0):
                x = torch.linspace(0, end, dim)
                x[-1], x[3] = end, -s
                rows.append(x * sign)
    x = torch.stack(rows)[:, None].to(dtype)
    n = x.shape[0]
    cache = fobq.Kv4Cache.empty(-(-n // 16), 1, dim, 16)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32).cuda()  # noqa: E731
    batch = fobq.Kv4Batch(i32([list(range(-(-n // 16)))]), i32([n]), i32([0, n]))
    ctx.kv4_append(cache, batch, x.cuda(), x.flip(0).cuda())
    codes, scale, zero = ref.grid(x[:, 0])                     # (a range of two bf16 numbers 2^44 apart is exact in 64 bits)
    for c, g, back in ((cache.k_codes, cache.k_grids, False), (cache.v_codes, cache.v_grids, True)):
        level, got = ref.unpack(c.cpu().flatten(0, 2)[:n], g.cpu().flatten()[:n])
        level, got = (t.flip(0) if back else t for t in (level, got))
        assert torch.equal(got, scale)
        assert torch.equal(level, codes - zero[:, None])
    span = x[:, 0].double().amax(-1).clamp(min=0) - x[:, 0].double().amin(-1).clamp(max=0)
    assert (15 * scale >= span).all()
