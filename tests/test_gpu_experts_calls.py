"""A feed-forward part of experts as a network calls it: its operators one after another, captured into graphs and replayed, on other streams, twice
with the same result."""
import pytest

torch = pytest.importorskip("torch")
import experts_reference as eref
import lowbit_reference as ref

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
WIDTH, HIDDEN, EXPERTS, TOP = 640, 256, 12, 3


class Part:
    """Norm, router, two products of the experts' rows with the gated activation between them, and the sum onto a shared expert's result."""

    def __init__(self, ctx, tokens, seed=0):
        import paper_2509_05576_amd as fobq
        self.ctx, self.tokens = ctx, tokens
        g = torch.Generator().manual_seed(seed)
        normal = lambda *shape: torch.randn(shape, generator=g)  # noqa: E731
        self.up, self.down = fobq.Fp8Experts.empty(EXPERTS, 2 * HIDDEN, WIDTH), fobq.Fp8Experts.empty(EXPERTS, WIDTH, HIDDEN, rows_per_scale=1)
        for e in range(EXPERTS):
            ctx.fp8_quantize((normal(2 * HIDDEN, WIDTH) * 0.05).cuda(), rows_per_scale=128, out=self.up.expert(e))
            ctx.fp8_quantize((normal(WIDTH, HIDDEN) * 0.08).cuda(), out=self.down.expert(e))
        self.shared_up = ctx.fp8_quantize((normal(2 * HIDDEN, WIDTH) * 0.05).cuda(), rows_per_scale=128)
        self.shared_down = ctx.fp8_quantize((normal(WIDTH, HIDDEN) * 0.08).cuda(), rows_per_scale=128)
        self.router = ctx.fp8_quantize((normal(EXPERTS, WIDTH) * 0.1).cuda())
        self.weight, self.bias = (1 + 0.1 * normal(WIDTH)).to(BF).cuda(), (0.02 * normal(EXPERTS)).cuda()
        self.x, self.residual = (torch.zeros((tokens, WIDTH), dtype=BF, device="cuda") for _ in range(2))
        torch.cuda.synchronize()

    def reset(self, seed):
        g = torch.Generator().manual_seed(seed)
        for t in (self.x, self.residual):
            t.copy_(torch.randn(t.shape, generator=g))
        torch.cuda.synchronize()

    def run(self):
        ctx = self.ctx
        h, total = ctx.fp8_rms_norm(self.x, self.weight, self.residual)
        routing = ctx.route(ctx.fp8_matmul(h, self.router, torch.float32), TOP, score="sigmoid", bias=self.bias, groups=4, top_groups=2, scale=1.5)
        inner = ctx.fp8_swiglu(ctx.fp8_expert_matmul(h, self.up, routing))
        rows = ctx.fp8_expert_matmul(inner, self.down, routing, packed=True)
        shared = ctx.fp8_matmul(ctx.fp8_swiglu(ctx.fp8_matmul(h, self.shared_up)), self.shared_down)
        out = ctx.expert_sum(rows, routing, base=shared)
        return [out, total, routing.chosen, routing.weights, routing.starts, routing.pairs, routing.places, rows, shared, inner.values.view(torch.uint8), inner.scales,
                h.values.view(torch.uint8), h.scales]


@pytest.fixture(scope="module")
def ctx():
    import paper_2509_05576_amd as fobq
    c = fobq.Ctx(0)
    yield c
    c.close()


SIZES = [1, 7, 70, 500]


@pytest.mark.parametrize("tokens", SIZES)
def test_a_part_of_a_network(ctx, tokens):
    """Each step against 64 bits from what the step before gave."""
    import paper_2509_05576_amd as fobq
    p = Part(ctx, tokens)
    p.reset(0)
    out, total, chosen, weights, starts, pairs, places, rows, shared, iv, iscale, hv, hscale = (t.cpu() for t in p.run())
    E4 = torch.float8_e4m3fn
    s, y = eref.rms_norm(p.x.cpu(), p.weight.cpu(), p.residual.cpu(), 1e-6)
    eref.check_blocks(hv.view(E4), hscale, y, y.abs() * 6.1 * ref.U, E4)
    h, inner = ref.expand(hv.view(E4).double(), hscale, 1), ref.expand(iv.view(E4).double(), iscale, 1)
    assert (starts[1:] >= starts[:-1]).all() and int(starts[-1]) == tokens * TOP and sorted(pairs.tolist()) == list(range(tokens * TOP))
    assert torch.equal(chosen.flatten()[pairs.long()], torch.repeat_interleave(torch.arange(EXPERTS, dtype=torch.int32), starts.diff().long()))
    assert torch.equal(pairs[places.long().flatten()], torch.arange(tokens * TOP, dtype=torch.int32))
    dense = lambda m: ref.expand(m.values.cpu().double(), m.scales.cpu(), m.rows_per_scale)  # noqa: E731
    for e in range(EXPERTS):
        lo, hi = int(starts[e]), int(starts[e + 1])
        if lo == hi:
            continue
        want, bound = ref.matmul(inner[lo:hi], dense(p.down.expert(e)), BF)
        assert ((rows[lo:hi].double() - want).abs() <= bound).all()
        # the first product in 64 bits: its bound passes through the activation (whose slope is at most 1.1 |up| + |silu|) and 8 bits
        first, bound = ref.matmul(h[(pairs[lo:hi] // TOP).long()], dense(p.up.expert(e)), BF)
        y, _, _ = eref.swiglu(first)
        gate, up = first.chunk(2, 1)
        off = bound[:, :HIDDEN] * 1.1 * (up.abs() + bound[:, HIDDEN:]) + bound[:, HIDDEN:] * (gate.abs() + bound[:, :HIDDEN]) + y.abs() * 1e-5
        got = inner[lo:hi]
        most = (y.abs() + off).unflatten(1, (-1, 128)).amax(2).repeat_interleave(128, 1)
        assert ((got - y).abs() <= off + (y.abs() + off) * 2.0 ** -4 + most / 448 * 2.0 ** -9).all()
    want, bound = eref.expert_sum(rows, weights, places, shared)
    assert ((out.double() - want).abs() <= bound).all()
    logits = ctx.fp8_matmul(fobq.Fp8Matrix(hv.view(E4).cuda(), hscale.cuda()), p.router, torch.float32).cpu()
    want = eref.route(logits, TOP, score="sigmoid", bias=p.bias.cpu(), groups=4, top_groups=2, scale=1.5)
    assert torch.equal(chosen, want[0]) and ((weights.double() - want[1]).abs() <= eref.weight_bound(want[1], want[5], EXPERTS)).all()


@pytest.mark.parametrize("tokens", SIZES)
def test_twice_the_same(ctx, tokens):
    p, got = Part(ctx, tokens), []
    for _ in range(2):
        p.reset(3)
        got.append([t.clone() for t in p.run()])
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_routes_of_many_tokens_captured(ctx):
    """Two launches and scratch between them, replayed several times with eager calls between."""
    import paper_2509_05576_amd as fobq
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        c = fobq.Ctx(0)
        x = torch.zeros((3000, 96), device="cuda")
        inputs = [torch.randn((3000, 96), generator=torch.Generator().manual_seed(i)).cuda() for i in range(4)]
        fields = ("chosen", "weights", "starts", "pairs", "places")
        run = lambda: [getattr(r, f) for r in [c.route(x, 5, groups=8, top_groups=3)] for f in fields]  # noqa: E731
        want = []
        for t in inputs:
            x.copy_(t)
            want.append([o.clone() for o in run()])
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            outs = run()
        for i in (0, 1, 1, 3, 2, 0):
            x.copy_(inputs[i])
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(outs, want[i])), i
            x.copy_(inputs[(i + 1) % 4])
            assert all(torch.equal(a, b) for a, b in zip(run(), want[(i + 1) % 4]))
        del graph, outs
        torch.cuda.synchronize()
        c.close()


def test_captured_and_replayed():
    """Two graphs in turn, each several times, with eager work between: every replay is the eager result for what the inputs then are."""
    import paper_2509_05576_amd as fobq
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        ctx = fobq.Ctx(0)
        parts = [Part(ctx, 5), Part(ctx, 300, seed=1)]
        graphs, outs, want = [], [], []
        for p in parts:
            want.append({})
            for seed in range(4):
                p.reset(seed)
                want[-1][seed] = [t.clone() for t in p.run()]
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                got = p.run()
            graphs.append(graph)
            outs.append(got)
        for step, (i, seed) in enumerate([(0, 0), (1, 1), (0, 1), (0, 2), (1, 3), (1, 0), (0, 3), (0, 3), (1, 2)]):
            parts[i].reset(seed)
            for t in outs[i]:
                t.fill_(7)
            torch.cuda.synchronize()
            graphs[i].replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(outs[i], want[i][seed])), (step, i, seed)
            other = parts[1 - i]
            other.reset(step % 4)
            again = [t.clone() for t in other.run()]
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(again, want[1 - i][step % 4]))
        del graphs, outs
        torch.cuda.synchronize()
        ctx.close()


@pytest.mark.parametrize("tokens", [7, 500])
def test_a_context_on_another_stream(ctx, tokens):
    import paper_2509_05576_amd as fobq
    here = Part(ctx, tokens)
    here.reset(1)
    want = [t.clone() for t in here.run()]
    side = torch.cuda.Stream()
    other = fobq.Ctx(0, side.cuda_stream)
    p = Part(ctx, tokens)
    p.ctx = other
    for _ in range(3):
        p.reset(1)
        noise = torch.full((1 << 22,), 3.0, device="cuda")              # the current stream's own work and memory meanwhile
        got = p.run()
        for _ in range(4):
            noise = noise * 1.5 - 2.0
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        del got
    torch.cuda.synchronize()
    other.close()


def test_two_streams_at_once(ctx):
    import paper_2509_05576_amd as fobq
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    ctxs = [fobq.Ctx(0, s.cuda_stream) for s in streams]
    want, parts = [], []
    for i, tokens in enumerate((9, 400)):
        p = Part(ctx, tokens, seed=i)
        p.reset(2)
        want.append([t.clone() for t in p.run()])
        torch.cuda.synchronize()
        p.ctx = ctxs[i]
        parts.append(p)
    kept = []
    for _ in range(10):
        kept += [(i, p.run()) for i, p in enumerate(parts)]
    torch.cuda.synchronize()
    for i, got in kept:
        assert all(torch.equal(a, b) for a, b in zip(got, want[i]))
    for c in ctxs:
        c.close()


@pytest.mark.parametrize("context_on_side", [False, True])
def test_memory_is_the_context_streams(monkeypatch, context_on_side):
    """Outputs and scratch belong to the context's stream, whichever stream is the current one."""
    import paper_2509_05576_amd as fobq
    seen = []

    def spy(make):
        def made(*a, **kw):
            seen.append(torch.cuda.current_stream(0).cuda_stream)
            return make(*a, **kw)
        return made

    class Torch:
        def __getattr__(self, name):
            return spy(getattr(torch, name)) if name in ("empty", "empty_strided") else getattr(torch, name)

    default, side = torch.cuda.default_stream(0), torch.cuda.Stream(0)
    home, away = (side, default) if context_on_side else (default, side)
    with torch.cuda.stream(home):
        c = fobq.Ctx(0)
        x = torch.ones((70, 64), device="cuda")
        w = fobq.Fp8Experts.empty(64, 32, 64)
        w.values.view(torch.uint8).zero_()
        w.scales.zero_()
        small, many = c.route(x[:9], 2), c.route(x, 2)
        m = c.fp8_quantize(x)
    torch.cuda.synchronize()
    monkeypatch.setattr(fobq.binding, "torch", Torch())
    with torch.cuda.stream(away):
        calls = [(lambda: c.fp8_rms_norm(x), 2), (lambda: c.fp8_rms_norm(x, None, x), 3), (lambda: c.fp8_swiglu(x), 2), (lambda: c.route(x[:9], 2), 2),
                 (lambda: c.route(x, 2), 3), (lambda: c.fp8_expert_matmul(m, w, many), 1), (lambda: c.expert_sum(x[:18], small), 1)]
        for call, count in calls:
            del seen[:]
            call()
            assert seen == [home.cuda_stream] * count
    torch.cuda.synchronize()
    c.close()


def test_rows_far_apart(ctx):
    """Rows 2^31 elements apart, so that the last begin past 32 bits: the same bits as of dense matrices."""
    import paper_2509_05576_amd as fobq
    rows, cols, apart = 3, 272, (1 << 31) + 16
    memory, used = torch.empty(2 * apart + 4096, dtype=BF, device="cuda"), [0]

    def far(t):
        to = memory.as_strided((rows, t.shape[1]), (apart, 1), used[0])
        used[0] += -(-t.shape[1] // 16) * 16
        return to.copy_(t)

    g = torch.Generator().manual_seed(5)
    x, r, z = (torch.randn(rows, cols, generator=g).to(BF).cuda() for _ in range(3))
    want, total = ctx.fp8_rms_norm(x, None, r, norm=torch.empty_like(x))
    values = torch.empty(2 * apart + 4096, dtype=torch.uint8, device="cuda")
    there = fobq.Fp8Matrix(values.as_strided((rows, cols), (apart, 1)).view(torch.float8_e4m3fn), torch.empty_like(want.scales), 1)
    m, s = ctx.fp8_rms_norm(far(x), None, far(r), sum=far(z), out=there)
    assert torch.equal(s, total) and torch.equal(m.values.view(torch.uint8), want.values.view(torch.uint8)) and torch.equal(m.scales, want.scales)
    want, m = ctx.fp8_swiglu(x), ctx.fp8_swiglu(far(x), out=fobq.Fp8Matrix(there.values[:, :cols // 2], there.scales[:2].contiguous(), 1))
    assert torch.equal(m.values.view(torch.uint8), want.values.view(torch.uint8)) and torch.equal(m.scales, want.scales)
    want, routing = ctx.route(x[:, :200], 1), ctx.route(far(x)[:, :200], 1)
    for a, b in zip((want.chosen, want.weights, want.starts, want.pairs, want.places), (routing.chosen, routing.weights, routing.starts, routing.pairs, routing.places)):
        assert torch.equal(a, b)
    base = far(z)
    assert torch.equal(ctx.expert_sum(far(x), routing, base=base, out=base), ctx.expert_sum(x, want, base=z))
