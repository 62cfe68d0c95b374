"""Routing to experts on the GPU, and the weighted sum behind it, against 64-bit forms."""
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


def _logits(tokens, experts, dtype, seed, spread=1.5):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((tokens, experts), generator=g) * spread + 0.5 * torch.randn((experts,), generator=g)).to(dtype)


def check(ctx, logits, top_k, **kw):
    r = ctx.route(logits.cuda(), top_k, **{**kw, "bias": kw["bias"].cuda() if kw.get("bias") is not None else None})
    chosen, weights, starts, pairs, places, far = ref.route(logits, top_k, **kw)
    assert torch.equal(r.chosen.cpu(), chosen) and torch.equal(r.starts.cpu(), starts) and torch.equal(r.pairs.cpu(), pairs) and torch.equal(r.places.cpu(), places)
    got = r.weights.cpu().double()
    assert torch.equal(got.isnan(), weights.isnan())
    bound = ref.weight_bound(weights, far, logits.shape[1]) * max(1.0, abs(kw.get("scale", 1.0)))
    assert ((got - weights).abs().nan_to_num(0.0) <= bound.nan_to_num(0.0)).all()
    return r


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("experts,top_k", [(1, 1), (2, 1), (7, 3), (8, 8), (64, 6), (65, 2), (128, 8), (200, 32), (256, 8), (500, 5), (513, 4), (1024, 10), (15, 15),
                                           (16, 14), (16, 16), (32, 14), (32, 15), (256, 14), (256, 15), (257, 8)])
def test_experts(ctx, experts, top_k, score):
    for i, (dtype, bias, renormalize) in enumerate(((F32, False, True), (BF, True, True), (HF, False, False), (F32, True, False))):
        b = 0.1 * _logits(1, experts, F32, 9)[0] if bias else None
        check(ctx, _logits(37, experts, dtype, experts + i), top_k, score=score, bias=b, renormalize=renormalize, scale=1.0 if i % 2 else 2.5)


@pytest.mark.parametrize("experts,groups,top_groups,top_k", [(8, 2, 1, 3), (64, 8, 3, 6), (104, 8, 4, 8), (256, 8, 4, 8), (160, 5, 2, 6), (62, 31, 7, 9), (64, 64, 20, 8),
                                                             (1024, 64, 32, 16), (990, 33, 4, 20), (48, 3, 3, 5), (12, 12, 4, 4), (256, 16, 7, 14), (256, 16, 16, 8), (272, 17, 5, 8), (250, 2, 1, 9),
                                                             (16, 16, 3, 3), (33, 3, 2, 15)])
def test_groups(ctx, experts, groups, top_groups, top_k):
    for i, (score, bias, group_top) in enumerate((("softmax", False, 1), ("sigmoid", True, 2), ("softmax", True, 1), ("softmax", False, 2), ("sigmoid", False, 2))):
        b = 0.1 * _logits(1, experts, F32, 3)[0] if bias else None
        check(ctx, _logits(29, experts, F32 if i % 2 else BF, experts + i), top_k, score=score, bias=b, groups=groups, top_groups=top_groups, group_top=group_top)


@pytest.mark.parametrize("tokens", [0, 1, 2, 15, 16, 17, 63, 64, 65, 128, 130, 1000])
def test_tokens(ctx, tokens):
    check(ctx, _logits(tokens, 40, BF, tokens), 4)
    check(ctx, _logits(tokens, 9, F32, tokens), 9, score="sigmoid", bias=torch.linspace(-1, 1, 9))


def test_many_tokens(ctx):
    """More than 64 tokens a workgroup.  (The choice against torch's, tie-free; the places against their definition.)"""
    logits = _logits(40001, 60, F32, 0)
    r = ctx.route(logits.cuda(), 3)
    assert torch.equal(r.chosen.cpu(), torch.sort(logits, dim=1, descending=True, stable=True).indices[:, :3].to(torch.int32))
    for got, want in zip((r.starts, r.pairs, r.places), ref.places(r.chosen.cpu(), 60)):
        assert torch.equal(got.cpu(), want)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("bias", [None, "zeros", "few"])
def test_ties(ctx, score, bias):
    """Logits of few values: the lowest expert, and the lowest group, first."""
    g = torch.Generator().manual_seed(1)
    x = torch.randint(-2, 3, (50, 96), generator=g).float() * 0.5
    x[x == 0] *= -1                                         # zeros of both signs
    x[::2] = x[::2].abs() * torch.where(torch.rand(25, 96, generator=g) < 0.5, 1.0, -1.0) * (x[::2] == 0) + x[::2] * (x[::2] != 0)
    b = {None: None, "zeros": torch.zeros(96), "few": torch.randint(0, 2, (96,), generator=g).float() * 0.25}[bias]
    for dtype in (F32, BF):
        check(ctx, x.to(dtype), 7, score=score, bias=b)
        check(ctx, x.to(dtype), 7, score=score, bias=b, groups=12, top_groups=5, group_top=1)
    check(ctx, torch.zeros(5, 96), 32, score=score, bias=b)


def test_close_keys(ctx):
    """Keys that differ by less than fp32 holds are told apart as 64 bits do: biases that make up for the scores but for 1e-9 of them."""
    x = _logits(64, 128, F32, 2)
    bias = (0.5 - torch.sigmoid(x[0].double())).float()
    r = ctx.route(x.cuda(), 8, score="sigmoid", bias=bias.cuda())
    key = torch.sigmoid(x.double()) + bias.double()
    apart = torch.sort(key, dim=1, descending=True).values
    sure = ((apart[:, :8] - apart[:, 1:9]).amin(1) > 1e-14)
    assert bool(sure[0]) and int(sure.sum()) > 60
    want = torch.sort(key, dim=1, descending=True, stable=True).indices[:, :8].to(torch.int32)
    assert torch.equal(r.chosen.cpu()[sure], want[sure])


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("experts,groups,top_groups,top_k", [(64, 8, 3, 6), (256, 8, 4, 8), (128, 1, 1, 8), (600, 20, 7, 9), (256, 16, 2, 14)])
def test_close_groups_and_keys(ctx, experts, groups, top_groups, top_k, score):
    """Biases that make keys, and so the groups' sums, nearly alike for some of the tokens: where they are further apart than 64 bits round, 64 bits decide."""
    g = torch.Generator().manual_seed(experts)
    base = _logits(1, experts, F32, 4)[0]
    p = torch.softmax(base.double(), 0) if score == "softmax" else torch.sigmoid(base.double())
    bias = (0.5 - p).float()                                 # the same key for all experts, but for the bias's rounding
    x = base.repeat(40, 1)
    x[20:] += 0.001 * torch.randn((20, experts), generator=g)
    r = ctx.route(x.cuda(), top_k, score=score, bias=bias.cuda(), groups=groups, top_groups=top_groups)
    p = torch.softmax(x.double(), 1) if score == "softmax" else torch.sigmoid(x.double())
    key, each, sure = p + bias.double(), experts // groups, 0
    for t in range(40):
        level = key[t].view(groups, each).sort(1, descending=True).values[:, :2].sum(1)
        order = torch.sort(level, descending=True, stable=True)
        apart = [float(order.values[top_groups - 1] - order.values[top_groups])] if top_groups < groups else []
        allowed = torch.zeros(groups, dtype=torch.bool)
        allowed[order.indices[:top_groups]] = True
        k = key[t].masked_fill(~allowed.repeat_interleave(each), -math.inf)
        best = torch.sort(k, descending=True, stable=True)
        if min(apart + (best.values[:top_k] - best.values[1:top_k + 1]).tolist()) > 1e-14:
            assert torch.equal(r.chosen[t].cpu(), best.indices[:top_k].to(torch.int32)), t
            sure += 1
    assert sure > 15


def test_far_logits(ctx):
    """Scores that no type holds: chosen by their logits, weights relative to the largest."""
    x = _logits(20, 30, F32, 5, 1.0) - 3000.0
    x[:, 7] -= 500
    for score in ("softmax", "sigmoid"):
        check(ctx, x, 4, score=score)
        check(ctx, -x, 4, score=score)
    check(ctx, x * 0.01, 4, score="sigmoid", renormalize=False)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_masked_and_not_finite(ctx, score):
    """Experts that are masked for a token or for all; tokens without any; NaN and Inf, which stay in their token."""
    x = _logits(12, 70, F32, 6)
    x[1, :] = -math.inf
    x[2, 3:] = -math.inf
    x[3, ::2] = -math.inf
    x[4, 60] = math.nan
    x[5, 11] = math.inf
    x[6, :69] = -math.inf
    x[7, ::3], x[8, :] = torch.finfo(F32).min, torch.finfo(F32).min      # masked by the lowest value: chosen where there is nothing else
    x[9, 4:], x[10, ::2] = torch.finfo(F32).min, torch.finfo(BF).min
    for kw in (dict(), dict(renormalize=False), dict(groups=7, top_groups=2, group_top=2), dict(groups=7, top_groups=3, group_top=1)):
        check(ctx, x, 5, score=score, **kw)
        bias = 0.1 * _logits(1, 70, F32, 8)[0]
        bias[20:50] = -math.inf
        check(ctx, x, 5, score=score, bias=bias, **kw)
    for bad in (math.nan, math.inf):
        bias[33] = bad
        assert bool(check(ctx, x, 5, score=score, bias=bias).weights.isnan().all())


def test_one_expert_has_all_the_weight(ctx):
    x = _logits(50, 40, F32, 2)
    for kw in (dict(), dict(score="sigmoid"), dict(score="sigmoid", bias=torch.linspace(0, 1, 40).cuda()), dict(score="sigmoid", groups=40, top_groups=1)):
        assert bool((ctx.route(x.cuda(), 1, **kw).weights == 1).all())


def test_strides_and_given_outputs(ctx):
    import paper_2509_05576_amd as fobq
    x = _logits(33, 50, BF, 3)
    wide = torch.cat((x[:, :1], x, x[:, :6]), 1).cuda()
    out = fobq.Routing.empty(33, 50, 4)
    assert ctx.route(wide[:, 1:51], 4, out=out) is out
    want = ref.route(x, 4)
    for got, w in zip((out.chosen, out.starts, out.pairs, out.places), (want[0], want[2], want[3], want[4])):
        assert torch.equal(got.cpu(), w)


def test_refusals(ctx):
    import paper_2509_05576_amd as fobq
    x = torch.zeros((4, 64), device="cuda")
    for bad in (lambda: ctx.route(x.cpu(), 2), lambda: ctx.route(x.t(), 2), lambda: ctx.route(x.double(), 2), lambda: ctx.route(x, 0), lambda: ctx.route(x, 33),
                lambda: ctx.route(x, 2.0), lambda: ctx.route(x, 2, score="max"), lambda: ctx.route(x, 2, bias=x[0, :5]), lambda: ctx.route(x, 2, bias=x[0].half()),
                lambda: ctx.route(x[:, :1], 2), lambda: ctx.route(x, 2, out=fobq.Routing.empty(4, 63, 2)), lambda: ctx.route(x, 2, out=fobq.Routing.empty(4, 64, 3))):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: ctx.route(x, 2, groups=7), lambda: ctx.route(x, 2, groups=0), lambda: ctx.route(x, 2, groups=8, top_groups=9),
                lambda: ctx.route(x, 9, groups=8, top_groups=1), lambda: ctx.route(x, 2, groups=8, group_top=3), lambda: ctx.route(x, 2, scale=math.inf),
                lambda: ctx.route(torch.zeros((1, 1025), device="cuda"), 1)):
        with pytest.raises(fobq.FobqError):
            bad()


@pytest.mark.parametrize("dtype", [F32, BF, HF])
@pytest.mark.parametrize("tokens,cols,top_k", [(1, 1, 1), (3, 7, 2), (5, 8, 3), (17, 130, 8), (9, 513, 32), (130, 1000, 5), (4, 4608, 9)])
def test_sum(ctx, tokens, cols, top_k, dtype):
    import paper_2509_05576_amd as fobq
    g = torch.Generator().manual_seed(cols)
    y = torch.randn((tokens * top_k, cols), generator=g).to(dtype)
    w = torch.randn((tokens, top_k), generator=g)
    where = torch.randperm(tokens * top_k, generator=g).to(torch.int32).reshape(tokens, top_k)
    where[torch.rand((tokens, top_k), generator=g) < 0.2] = -1          # pairs of no expert
    where.view(-1)[-1] = tokens * top_k                                  # and a place that is none
    routing = fobq.Routing(None, w.cuda(), None, None, where.cuda())
    base = torch.randn((tokens, cols), generator=g).to(dtype)
    for b in (None, base):
        want, bound = ref.expert_sum(y, w, where, b)
        got = ctx.expert_sum(y.cuda(), routing, None if b is None else b.cuda())
        assert got.dtype == dtype and ((got.cpu().double() - want).abs() <= bound).all()
    # rows of wider matrices, onto the base itself
    wide = torch.cat((base[:, :1], base, base[:, :1]), 1).cuda()
    rows = torch.cat((y[:, :1], y), 1).cuda()
    into = wide[:, 1:1 + cols]
    assert ctx.expert_sum(rows[:, 1:], routing, into, out=into) is into
    assert ((into.cpu().double() - want).abs() <= bound).all()
    assert torch.equal(wide[:, 0].cpu(), base[:, 0]) and torch.equal(wide[:, -1].cpu(), base[:, 0])


def test_sum_not_finite(ctx):
    """A NaN in a row reaches the tokens that have it, also with weight 0, and no others."""
    import paper_2509_05576_amd as fobq
    y = torch.ones((6, 300), device="cuda")
    y[4, 17] = math.nan
    routing = fobq.Routing(None, torch.zeros((3, 2), device="cuda"), None, None, torch.tensor([[0, 1], [2, 4], [3, -1]], dtype=torch.int32, device="cuda"))
    got = ctx.expert_sum(y, routing).isnan().nonzero().tolist()
    assert got == [[1, 17]]
    with pytest.raises(TypeError):
        ctx.expert_sum(y, routing, y)
    with pytest.raises(TypeError):
        ctx.expert_sum(y, routing, out=y[:3].half())
    with pytest.raises(TypeError):
        ctx.expert_sum(y.t(), routing)
