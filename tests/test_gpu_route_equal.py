"""Routing where exact equals stand at the border of the choice: experts of the same logit and bias beside others whose keys differ by less than the first pass
resolves, saturated scores, and masks by finite values.  Logits are of few values, whose keys in 64 bits either are the same numbers or differ by far more than
their rounding."""
import math

import pytest

torch = pytest.importorskip("torch")
import experts_reference as ref

pytestmark = pytest.mark.gpu
F32, BF, HF = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ctx():
    import paper_2509_05576_amd as fobq
    c = fobq.Ctx(0)
    yield c
    c.close()


def check(ctx, logits, top_k, **kw):
    r = ctx.route(logits.cuda(), top_k, **{**kw, "bias": kw["bias"].cuda() if kw.get("bias") is not None else None})
    chosen, weights, starts, pairs, places, far = ref.route(logits, top_k, **kw)
    assert torch.equal(r.chosen.cpu(), chosen), (r.chosen.cpu() != chosen).any(1).nonzero().flatten().tolist()
    assert torch.equal(r.starts.cpu(), starts) and torch.equal(r.pairs.cpu(), pairs) and torch.equal(r.places.cpu(), places)
    bound = ref.weight_bound(weights, far, logits.shape[1])
    assert ((r.weights.cpu().double() - weights).abs() <= bound).all()


def _few(values, chances, tokens, experts, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    at = torch.multinomial(torch.tensor(chances).repeat(tokens, 1), experts, replacement=True, generator=g)
    return torch.tensor(values)[at].to(dtype)


EXPERTS = [40, 128, 256, 300, 600, 1000]


@pytest.mark.parametrize("experts", EXPERTS)
def test_a_larger_key_behind_equals(ctx, experts):
    """The only larger one stands behind equals that fp32 does not tell from it."""
    zeros = torch.zeros(experts)
    x = torch.zeros(2, experts)
    x[:, :3] = torch.tensor([20.0, 20.0, 25.0])
    check(ctx, x, 1, score="sigmoid", bias=zeros)
    check(ctx, x, 1, score="sigmoid", groups=2, group_top=2)
    x[:] = -1e4
    x[:, 4], x[:, 5] = 5.0, -20.0
    for top_k in (1, 2, 3, 14, 15):
        check(ctx, x, top_k, score="sigmoid", bias=zeros)
    x[:] = 0
    x[:, experts - 1] = 1e-7
    for top_k in (1, 2, 14, 15):
        check(ctx, x, top_k)
        check(ctx, x, top_k, score="sigmoid")
        check(ctx, x, top_k, bias=zeros)
        check(ctx, x, top_k, groups=2, top_groups=2, group_top=1)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("experts", EXPERTS)
@pytest.mark.parametrize("dtype", [F32, BF])
def test_few_values(ctx, experts, score, dtype):
    """Scores near 0 and 1 in many copies; top_k such that equals fall on either side of the last choice."""
    for i, chances in enumerate(([1, 1, 1, 1, 1, 1], [60, 1, 1, 1, 1, 1], [0.1, 0.1, 60, 1, 0.1, 0.1], [1, 1, 1, 60, 1, 0.2])):
        x = _few([-1e4, -30.0, -20.0, 20.0, 25.0, 30.0], [float(c) for c in chances], 12, experts, dtype, experts + i)
        for top_k in (1, 2, 3, 5, 8, 14, 15, 31):
            check(ctx, x, top_k, score=score, bias=torch.zeros(experts))
            check(ctx, x, top_k, score=score, groups=4, top_groups=4, group_top=2)
        check(ctx, x, 6, score=score, groups=4, top_groups=2, group_top=2)


@pytest.mark.parametrize("experts", EXPERTS)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("step", [1e-7, 1e-6, 1e-5])
def test_close_logits(ctx, experts, score, step):
    """Logits that are compared as they are: steps below, about and above those of the first pass."""
    for i, chances in enumerate(([1.0, 1.0, 1.0, 1.0], [60.0, 1.0, 1.0, 1.0], [60.0, 20.0, 0.3, 1.0])):
        x = _few([0.0, step, 2 * step, -5.0], chances, 12, experts, F32, experts + i)
        for top_k in (1, 2, 3, 8, 14, 15, 30):
            check(ctx, x, top_k, score=score)
            check(ctx, x, top_k, score=score, groups=4, top_groups=3, group_top=1)
    # the same at the lower end of what the first pass resolves, beside lower ones that are behind it
    x = _few([-16.0, -16.0 - step, -16.0 + step, -40.0], [20.0, 20.0, 1.0, 1.0], 12, experts, F32, experts)
    x[:, experts // 2] = 0
    for top_k in (1, 2, 3, 8, 14, 15):
        check(ctx, x, top_k, score=score)
        check(ctx, x, top_k, score=score, groups=4, top_groups=3, group_top=1)


@pytest.mark.parametrize("mask", [-1e4, -1e9, torch.finfo(F32).min])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("experts", EXPERTS)
def test_masks_by_finite_biases(ctx, experts, score, mask):
    """Half of the experts masked by a bias that is finite: the others' order is that of 64 bits, and the masked ones come behind them."""
    g = torch.Generator().manual_seed(experts)
    bias = torch.where(torch.rand(experts, generator=g) < 0.5, mask, 0.0)
    x = (torch.randn((12, experts), generator=g) * 2).to(BF)
    for top_k in (1, 2, 8, 14, 15):
        check(ctx, x, top_k, score=score, bias=bias)
    check(ctx, x, 6, score=score, bias=bias, groups=4, top_groups=2, group_top=2)
    check(ctx, x[:4], 15, score=score, bias=torch.where(torch.arange(experts) < 8, 0.0, mask))      # fewer than top_k are not masked


@pytest.mark.parametrize("experts", EXPERTS)
def test_all_equal(ctx, experts):
    for value in (0.0, 30.0, -30.0):
        x = torch.full((9, experts), value)
        for top_k in (1, 8, 14, 15, 31):
            for kw in (dict(), dict(bias=torch.zeros(experts)), dict(score="sigmoid", bias=torch.full((experts,), 0.5)), dict(score="sigmoid", groups=4, top_groups=4, group_top=2)):
                check(ctx, x, top_k, **kw)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("group_top", [1, 2])
@pytest.mark.parametrize("experts,groups,top_groups,top_k", [(20, 4, 1, 4), (12, 3, 1, 1), (64, 16, 3, 2), (8, 8, 5, 4), (256, 16, 9, 7), (600, 20, 3, 5), (60, 3, 1, 16)])
def test_groups_and_biases_near_the_ends_of_fp32(ctx, experts, groups, top_groups, top_k, group_top, score):
    """Groups are compared by sums that fp32 does not hold."""
    g = torch.Generator().manual_seed(experts)
    x = torch.randn((20, experts), generator=g)
    kw = dict(score=score, groups=groups, top_groups=top_groups, group_top=group_top)
    for mask in (torch.finfo(F32).min, -2e38):
        for part in (0.3, 0.5, 0.9):
            check(ctx, x, top_k, bias=torch.where(torch.rand(experts, generator=g) < part, mask, 0.0), **kw)
    # (far enough from each other that the scores, which fp32 and 64 bits lose beside them, decide nothing)
    ends = torch.tensor([-3.4e38, -2.5e38, -2e38, -1.1e38, -1e38, 0.0, 1e38, 1.4e38, 3.3e38])
    for lo, hi in ((0, 6), (0, 9), (5, 9)):
        check(ctx, x, top_k, bias=ends[torch.randint(lo, hi, (experts,), generator=g)], **kw)
