"""How the operators of a quantized network are called: one after another as a network does, captured into graphs and replayed, on other
streams than the current one, twice with the same result, with pages that several sequences share."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
HEADS, GROUP, DIM, PAGE, WIDTH = 2, 4, 128, 32, 1024
LINES = HEADS * (GROUP + 2) * DIM


class Block:
    """One attention block: q, k and v by an 8-bit product with a quantized layer's codes, the cache, attention, and a product back."""

    def __init__(self, ctx, seqs, seed=0):
        import paper_2509_05576_amd as fobq
        self.ctx, self.seqs = ctx, seqs
        g = torch.Generator().manual_seed(seed)
        codes = torch.randint(0, 16, (LINES, WIDTH), generator=g)
        scales = torch.rand((LINES, WIDTH // 128), generator=g) * 0.01 + 0.002
        zeros = torch.randint(4, 12, (LINES, WIDTH // 128), generator=g).float()
        self.w1 = ctx.fp8_from_codes(codes.to(torch.uint8).cuda(), scales.cuda(), zeros.cuda(), bits=4)
        self.w2 = ctx.fp8_quantize((torch.randn((WIDTH, HEADS * GROUP * DIM), generator=g) * 0.03).to(BF).cuda(), rows_per_scale=128)
        width = max(-(-n // PAGE) for n, _ in seqs) + 4
        self.cache = fobq.Kv4Cache.empty(width * len(seqs), HEADS, DIM, PAGE)
        for t in (self.cache.k_codes, self.cache.v_codes, self.cache.k_grids, self.cache.v_grids):
            t.zero_()
        self.table = torch.randperm(width * len(seqs), generator=g).to(torch.int32).reshape(len(seqs), width).cuda()
        self.lengths = torch.tensor([n for n, _ in seqs], dtype=torch.int32).cuda()
        self.starts = torch.tensor([0] + [new for _, new in seqs]).cumsum(0).to(torch.int32).cuda()
        self.batch = fobq.Kv4Batch(self.table, self.lengths, self.starts)
        self.rows = int(self.starts[-1])
        # tokens that are there before
        n = torch.tensor([0] + [n for n, _ in seqs]).cumsum(0).to(torch.int32)
        kv = torch.randn((int(n[-1]), 2 * HEADS, DIM), generator=g).to(BF).cuda()
        ctx.kv4_append(self.cache, fobq.Kv4Batch(self.table, self.lengths, n.cuda()), kv[:, :HEADS], kv[:, HEADS:])
        self.start = [t.clone() for t in self.state()]
        self.x = torch.zeros((self.rows, WIDTH), dtype=BF, device="cuda")
        torch.cuda.synchronize()

    def state(self):
        return self.cache.k_codes, self.cache.v_codes, self.cache.k_grids, self.cache.v_grids

    def reset(self, seed):
        for a, b in zip(self.state(), self.start):
            a.copy_(b)
        g = torch.Generator().manual_seed(seed)
        self.x.copy_(torch.randn((self.rows, WIDTH), generator=g))
        # shorter sequences too: fewer parts in the same launch
        back = torch.tensor([(seed * 797) % max(1, n - new + 1) for n, new in self.seqs], dtype=torch.int32)
        self.lengths.copy_(torch.tensor([n for n, _ in self.seqs], dtype=torch.int32) - back)
        torch.cuda.synchronize()

    def run(self):
        ctx = self.ctx
        y = ctx.fp8_matmul(ctx.fp8_quantize(self.x), self.w1).view(self.rows, HEADS * (GROUP + 2), DIM)
        q, k, v = y.split([HEADS * GROUP, HEADS, HEADS], 1)
        ctx.kv4_append(self.cache, self.batch, k, v)
        a = ctx.kv4_attention(self.cache, self.batch, q)
        out = ctx.fp8_matmul(ctx.fp8_quantize(a.view(self.rows, -1)), self.w2)
        return [out, a, *ctx.kv4_read(self.cache, self.batch, self.rows)]


DECODE, PROMPTS = [(3000, 1), (40, 1), (1500, 1)], [(200, 130), (64, 64), (2500, 9)]




@pytest.fixture(scope="module")
def ctx():
    import paper_2509_05576_amd as fobq
    c = fobq.Ctx(0)
    yield c
    c.close()


@pytest.mark.parametrize("seqs", [DECODE, PROMPTS])
def test_a_block_of_a_network(ctx, seqs):
    """The chain in 64 bits from what the matrices hold: keys and results within what 8-bit rows, 16-bit results, the matrix
    instructions (8 times 2^-13 of the products) and the cache's step take."""
    b = Block(ctx, seqs)
    b.reset(0)
    out, a, k, v = b.run()
    dense = lambda m: (m.values.float().unflatten(1, (-1, 128))  # noqa: E731
                       * m.scales.repeat_interleave(m.rows_per_scale, 1)[:, :m.values.shape[0]].t()[:, :, None]).flatten(1)
    w1, w2 = dense(b.w1).cpu().double(), dense(b.w2).cpu().double()
    x = b.x.cpu().double()
    y = (x @ w1.t()).view(b.rows, -1, DIM)
    # e4m3 with a scale per 128: half a step of each value (2^-4 of it, or of the smallest normal, 2^-6 of 448)
    dx = x.abs() * 2.0 ** -4 + x.abs().amax() / 448 * 2.0 ** -10
    dy = (dx @ w1.abs().t()).view(b.rows, -1, DIM) + y.abs() * 2.0 ** -8 + 8 * 2.0 ** -13 * (x.abs() @ w1.abs().t()).view(b.rows, -1, DIM)
    got_k, want_k = k.cpu().double(), y[:, HEADS * GROUP:HEADS * (GROUP + 1)]
    step = ((want_k + dy[:, HEADS * GROUP:HEADS * (GROUP + 1)]).amax(-1, keepdim=True).clamp(min=0)
            - (want_k - dy[:, HEADS * GROUP:HEADS * (GROUP + 1)]).amin(-1, keepdim=True).clamp(max=0)) / 15 * (1 + 2.0 ** -7)
    assert ((got_k - want_k).abs() <= dy[:, HEADS * GROUP:HEADS * (GROUP + 1)] + step * 1.01 + want_k.abs() * 2.0 ** -8).all()
    a64 = a.cpu().double().view(b.rows, -1)
    da = a64.abs() * 2.0 ** -4 + a64.abs().amax() / 448 * 2.0 ** -10
    bound = da @ w2.abs().t() + 8 * 2.0 ** -13 * (a64.abs() @ w2.abs().t())
    want = a64 @ w2.t()
    assert ((out.cpu().double() - want).abs() <= bound + want.abs() * 2.0 ** -8 + bound * 2.0 ** -8).all()


@pytest.mark.parametrize("seqs", [DECODE, PROMPTS])
def test_twice_the_same(ctx, seqs):
    b = Block(ctx, seqs)
    got = []
    for _ in range(2):
        b.reset(3)
        got.append([t.clone() for t in b.run()])
    assert all(torch.equal(x, y) for x, y in zip(*got))


def test_captured_and_replayed():
    """Two graphs in turn, each several times, with eager work between: every replay is the eager result for what the inputs then are."""
    import paper_2509_05576_amd as fobq
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        ctx = fobq.Ctx(0)
        blocks = [Block(ctx, DECODE), Block(ctx, PROMPTS, seed=1)]
        graphs, outs, want = [], [], []
        for b in blocks:
            want.append({})
            for seed in range(4):
                b.reset(seed)
                want[-1][seed] = [t.clone() for t in b.run()] + [t.clone() for t in b.state()]
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                got = b.run()
            graphs.append(graph)
            outs.append(got)
        for step, (i, seed) in enumerate([(0, 0), (1, 1), (0, 1), (0, 2), (1, 3), (1, 0), (0, 3), (0, 3), (1, 2)]):
            b = blocks[i]
            b.reset(seed)
            for t in outs[i]:
                t.fill_(7.0)
            torch.cuda.synchronize()
            graphs[i].replay()
            torch.cuda.synchronize()
            got = [t.clone() for t in outs[i]] + [t.clone() for t in b.state()]
            assert all(torch.equal(x, y) for x, y in zip(got, want[i][seed])), (step, i, seed)
            other = blocks[1 - i]
            other.reset(step % 4)
            again = [t.clone() for t in other.run()]                    # eager work between, with scratch of its own
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(again, want[1 - i][step % 4]))
        del graphs, outs
        torch.cuda.synchronize()
        ctx.close()


@pytest.mark.parametrize("seqs", [DECODE, PROMPTS])
def test_a_context_on_another_stream(ctx, seqs):
    import paper_2509_05576_amd as fobq
    here = Block(ctx, seqs)
    here.reset(1)
    want = [t.clone() for t in here.run()]
    side = torch.cuda.Stream()
    other = fobq.Ctx(0, side.cuda_stream)
    b = Block(ctx, seqs)
    b.ctx = other
    for _ in range(3):
        b.reset(1)
        noise = torch.full((1 << 22,), 3.0, device="cuda")              # the current stream's own work and memory meanwhile
        got = b.run()
        for _ in range(4):
            noise = noise * 1.5 - 2.0
        side.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want))
        del got
    torch.cuda.synchronize()
    other.close()


def test_two_streams_at_once(ctx):
    import paper_2509_05576_amd as fobq
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    ctxs = [fobq.Ctx(0, s.cuda_stream) for s in streams]
    want, blocks = [], []
    for i, seqs in enumerate((DECODE, PROMPTS)):
        b = Block(ctx, seqs, seed=i)
        b.reset(2)
        want.append([t.clone() for t in b.run()])
        torch.cuda.synchronize()
        b.ctx = ctxs[i]
        b.reset(2)
        blocks.append(b)
    kept = []
    for _ in range(10):                                                 # (a repeated call stores the same rows again)
        kept += [(i, b.run()) for i, b in enumerate(blocks)]
    torch.cuda.synchronize()
    for i, got in kept:
        assert all(torch.equal(x, y) for x, y in zip(got, want[i]))
    for c in ctxs:
        c.close()


def test_pages_that_sequences_share(ctx):
    """A prompt's pages under two sequences, each with a last page of its own: as if each had all of them."""
    import paper_2509_05576_amd as fobq
    g = torch.Generator().manual_seed(5)
    rows = torch.randn((64 + 2 * 7, 2 * HEADS, DIM), generator=g).to(BF).cuda()
    k, v = rows[:, :HEADS], rows[:, HEADS:]
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    shared, apart = fobq.Kv4Cache.empty(4, HEADS, DIM, PAGE), fobq.Kv4Cache.empty(6, HEADS, DIM, PAGE)
    ctx.kv4_append(shared, fobq.Kv4Batch(i32([[3, 1]]), i32([64]), i32([0, 64])), k[:64], v[:64])
    both = fobq.Kv4Batch(i32([[3, 1, 0], [3, 1, 2]]), i32([71, 71]), i32([0, 7, 14]))
    ctx.kv4_append(shared, both, k[64:], v[64:])
    for s in range(2):
        t = i32([[3 * s, 3 * s + 1, 3 * s + 2]])
        ctx.kv4_append(apart, fobq.Kv4Batch(t, i32([64]), i32([0, 64])), k[:64], v[:64])
        ctx.kv4_append(apart, fobq.Kv4Batch(t, i32([71]), i32([0, 7])), k[64 + 7 * s:71 + 7 * s], v[64 + 7 * s:71 + 7 * s])
    q = torch.randn((14, HEADS * GROUP, DIM), generator=g).to(BF).cuda()
    alone = fobq.Kv4Batch(i32([[0, 1, 2], [3, 4, 5]]), both.lengths, both.starts)
    assert torch.equal(ctx.kv4_attention(shared, both, q), ctx.kv4_attention(apart, alone, q))
