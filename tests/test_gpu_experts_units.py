"""How far the exponentials of the gated activation and of the routing weights are off, in units of fp32's rounding (U = 2^-24): bounds that a product with log2(e)
rounded to fp32, and no more, would miss by far (half a unit of a 7-bit number's last place in the exponent, about 40 U in the result)."""
import pytest

torch = pytest.importorskip("torch")
from lowbit_reference import U

pytestmark = pytest.mark.gpu
F32, BF, HF = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ctx():
    import paper_2509_05576_amd as fobq
    c = fobq.Ctx(0)
    yield c
    c.close()


def _arguments(lo, hi, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.cat((torch.linspace(lo, hi, 4001), lo + (hi - lo) * torch.rand(4000, generator=g)))


@pytest.mark.parametrize("dtype", [F32, BF, HF])
def test_activation(ctx, dtype):
    """Rows of one column: a block's scale is its only value's magnitude over 448.  exp2 is off by a unit in the last place (2 U), what it leaves out is added (U), then 1 + e
    (U), the corrected reciprocal (U), two products (2 U) and the division by 448 (U): 8 U."""
    gate = _arguments(-80.0, 88.0, 0).to(dtype)
    up = (1 + torch.rand(len(gate), generator=torch.Generator().manual_seed(1))).to(dtype)
    m = ctx.fp8_swiglu(torch.stack((gate, up), 1).cuda())
    want = (gate.double() * torch.sigmoid(gate.double()) * up.double()).abs() / 448
    there = want >= 2.0 ** -126                              # (a scale is at least that)
    got = m.scales[0].cpu().double()
    assert int(there.sum()) > 7900
    assert ((got - want).abs() <= 8.1 * U * want)[there].all()


def test_softmax_weights(ctx):
    """Two experts: e and 1 over 1 + e, e = exp(-d) to 3 U, the sum and the division a U each."""
    d = _arguments(0.0, 80.0, 2)
    r = ctx.route(torch.stack((torch.zeros_like(d), -d), 1).cuda(), 2)
    e = torch.exp(-d.double())
    want, got = torch.stack((1 / (1 + e), e / (1 + e)), 1), r.weights.cpu().double()
    assert ((got - want).abs() <= 5.1 * U * want).all()
    r = ctx.route(torch.stack((torch.zeros_like(d), -d), 1).cuda(), 2, renormalize=True, score="softmax", groups=2, top_groups=2, group_top=1)
    assert ((r.weights.cpu().double() - want).abs() <= 5.1 * U * want).all()


@pytest.mark.parametrize("experts", [1, 300])
def test_sigmoid_weights(ctx, experts):
    """1 or e over 1 + e."""
    z = _arguments(-80.0, 80.0, 3)
    x = torch.full((len(z), experts), -100.0)
    x[:, experts // 2] = z
    r = ctx.route(x.cuda(), 1, score="sigmoid", renormalize=False)
    want = torch.sigmoid(z.double())
    assert ((r.weights[:, 0].cpu().double() - want).abs() <= 5.1 * U * want).all()
