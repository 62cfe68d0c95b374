"""The 4-bit cache on the GPU: append, read and attention against 64-bit forms."""
import math

import pytest

torch = pytest.importorskip("torch")
import lowbit_reference as ref

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ctx():
    import paper_2509_05576_amd as fobq
    c = fobq.Ctx(0)
    yield c
    c.close()


class Case:
    """Sequences of (tokens held, new rows), with keys and values of all tokens appended in the order given."""

    def __init__(self, ctx, seqs, heads=2, dim=128, page=16, dtype=BF, seed=0, spare=2, spread=0.5):
        import paper_2509_05576_amd as fobq
        self.ctx, self.seqs, self.heads, self.dim, self.page, self.dtype = ctx, seqs, heads, dim, page, dtype
        g = torch.Generator().manual_seed(seed)
        need = [-(-n // page) for n, _ in seqs]
        width = max(1, max(need, default=1)) + 1
        self.pages = sum(need) + spare
        order = torch.randperm(self.pages, generator=g).to(torch.int32)
        self.table = torch.full((max(1, len(seqs)), width), -1, dtype=torch.int32)
        at = 0
        for i, k in enumerate(need):
            self.table[i, :k] = order[at:at + k]
            at += k
        self.cache = fobq.Kv4Cache.empty(self.pages, heads, dim, page)
        for t in (self.cache.k_codes, self.cache.v_codes):
            t.fill_(0xA5)
        for t in (self.cache.k_grids, self.cache.v_grids):
            t.fill_(0x7FC0000F)                  # NaN scales where nothing is written
        self.lengths = torch.tensor([n for n, _ in seqs], dtype=torch.int32)
        starts = [0]
        for _, new in seqs:
            starts.append(starts[-1] + new)
        self.starts, self.rows = torch.tensor(starts, dtype=torch.int32), starts[-1]
        self.kv = []
        for n, _ in seqs:
            size = torch.exp(spread * torch.randn((n, heads, 1), generator=g))
            self.kv.append([(torch.randn((n, heads, dim), generator=g) * size).to(dtype) for _ in range(2)])
        every = torch.tensor([0] + [n for n, _ in seqs]).cumsum(0).to(torch.int32)
        self.all = self.batch(starts=every)
        self.tokens = int(every[-1])
        if self.tokens:
            k, v = (torch.cat([x[j] for x in self.kv]).cuda() for j in range(2))
            ctx.kv4_append(self.cache, self.all, k, v)
        self.g = g

    def batch(self, **kw):
        import paper_2509_05576_amd as fobq
        d = dict(table=self.table, lengths=self.lengths, starts=self.starts)
        d.update(kw)
        return fobq.Kv4Batch(*(None if x is None else x.cuda() for x in (d["table"], d["lengths"], d["starts"])))

    def rows_of(self, s):
        """(code - zero, scale) of sequence s in the cache, for keys and values: heads first."""
        n = self.seqs[s][0]
        pages = self.table[s, :-(-n // self.page)].long()
        got = []
        for c, w in ((self.cache.k_codes, self.cache.k_grids), (self.cache.v_codes, self.cache.v_grids)):
            level, scale = ref.unpack(c.cpu()[pages], w.cpu()[pages])
            got.append((level.transpose(0, 1).flatten(1, 2)[:, :n], scale.transpose(0, 1).flatten(1, 2)[:, :n]))
        return got

    def queries(self, group, size=1.0):
        return (torch.randn((self.rows, self.heads * group, self.dim), generator=self.g) * size).to(self.dtype)

    def spans(self, s, causal, window):
        n, new = self.seqs[s]
        got = []
        for i in range(new):
            b = n - new + i + 1 if causal else n
            a = max(0, b - window) if window else 0
            got.append((a, max(a, b)))
        return got

    def check(self, q, out, lse, scale, causal=True, window=0):
        group, at = q.shape[1] // self.heads, 0
        out, lse = out.cpu().double(), lse.cpu().double()
        for s, (n, new) in enumerate(self.seqs):
            (kc, ks), (vc, vs) = self.rows_of(s)
            spans = self.spans(s, causal, window)
            for h in range(self.heads):
                for j in range(group):
                    hq = h * group + j
                    want, wl, bound, lbound = ref.attention(q[at:at + new, hq], (kc[h], ks[h]), (vc[h], vs[h]), scale, spans, self.dtype)
                    off = (out[at:at + new, hq] - want).abs()
                    assert (off <= bound).all(), (s, hq, (off / bound.clamp(min=1e-300)).max())
                    seen = torch.tensor([b > a for a, b in spans], dtype=torch.bool)
                    assert torch.equal(lse[at:at + new, hq][~seen], wl[~seen])
                    assert ((lse[at:at + new, hq] - wl).abs()[seen] <= lbound[seen]).all()
            at += new


def run(case, group, causal=True, window=0, scale=None, size=1.0, **kw):
    q = case.queries(group, size)
    lse = torch.full((case.rows, case.heads * group), 5.0, device="cuda")
    out = case.ctx.kv4_attention(case.cache, case.batch(), q.cuda(), causal=causal, window=window, scale=scale, lse=lse, **kw)
    case.check(q, out, lse, case.dim ** -0.5 if scale is None else scale, causal, window)
    return q, out


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads,page", [(1, 16), (3, 32), (8, 256)])
def test_append_and_read(ctx, dim, dtype, heads, page):
    c = Case(ctx, [(40, 3), (0, 0), (1, 1), (page, 2), (page + 1, 1)], heads, dim, page, dtype, seed=dim + heads)
    at = 0
    for s, (n, _) in enumerate(c.seqs):
        for (level, scale), x in zip(c.rows_of(s), c.kv[s]):
            codes, want_scale, zero = ref.grid(x.transpose(0, 1))
            assert torch.equal(scale, want_scale) and torch.equal(level, codes - zero[..., None])
    # places that no token has are as they were
    used = torch.zeros((c.pages, page), dtype=torch.bool)
    for s, (n, _) in enumerate(c.seqs):
        for t in range(n):
            used[c.table[s, t // page], t % page] = True
    for t in (c.cache.k_codes, c.cache.v_codes):
        assert (t.cpu().transpose(1, 2)[~used] == 0xA5).all()
    for t in (c.cache.k_grids, c.cache.v_grids):
        assert (t.cpu().transpose(1, 2)[~used] == 0x7FC0000F).all()
    for out in (torch.float32, BF, HF):
        k, v = ctx.kv4_read(c.cache, c.all, c.tokens, out)
        at = 0
        for s, (n, _) in enumerate(c.seqs):
            for got, (level, scale) in zip((k, v), c.rows_of(s)):
                assert torch.equal(got[at:at + n].cpu(), (level * scale[..., None]).transpose(0, 1).to(out))
            at += n


def test_append_extremes(ctx):
    """Rows of zeros, of one sign, of the largest and smallest values, and rows that are not finite."""
    import paper_2509_05576_amd as fobq
    dim, top = 64, torch.finfo(BF).max
    rows = torch.zeros((12, 1, dim), dtype=torch.float32)
    rows[1] = 2.5
    rows[2] = -0.75
    rows[3, 0, 5] = top
    rows[4, 0, 5], rows[4, 0, 6] = top, -top                  # the range passes fp32
    rows[5, 0, 5], rows[5, 0, 6] = top / 4, -top / 4
    rows[6] = torch.linspace(-1, 1, dim) * 2.0 ** -130          # denormal
    rows[7, 0, 9] = math.inf
    rows[8, 0, 9] = math.nan
    rows[9, 0, 0] = 2.0 ** -133
    rows[10] = torch.arange(dim) * 0.25 - 3
    rows[11, 0, 63] = -math.inf
    x = rows.to(BF)
    cache = fobq.Kv4Cache.empty(1, 1, dim, 16)
    batch = fobq.Kv4Batch(torch.zeros((1, 1), dtype=torch.int32).cuda(), torch.tensor([12], dtype=torch.int32).cuda(), torch.tensor([0, 12], dtype=torch.int32).cuda())
    ctx.kv4_append(cache, batch, x.cuda(), x.cuda())
    k, v = ctx.kv4_read(cache, batch, 12, torch.float32)
    assert torch.equal(k.isnan(), v.isnan())
    bad = torch.tensor([i in (4, 7, 8, 11) for i in range(12)])
    assert torch.equal(k.cpu().isnan().flatten(1).all(1), bad) and torch.equal(k.cpu().isnan().flatten(1).any(1), bad)
    codes, scale, zero = ref.grid(x[~bad])
    want = (codes - zero[..., None]) * scale[..., None]
    assert torch.equal(k.cpu()[~bad].double(), want) and torch.equal(v.cpu()[~bad].double(), want)
    assert (k.cpu()[0] == 0).all()


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("group", [1, 4, 7, 16, 40])
def test_single_tokens(ctx, dim, dtype, group):
    run(Case(ctx, [(1, 1), (0, 1), (15, 1), (16, 1), (17, 1), (33, 1), (130, 1), (700, 1)], 2, dim, 16, dtype, seed=group), group)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("seqs", [[(5, 5), (40, 2), (64, 8), (9, 1)], [(200, 70), (3, 3), (0, 0), (131, 131)], [(300, 300)]])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 33), (False, 50), (True, 1)])
def test_several_tokens(ctx, dim, dtype, seqs, causal, window):
    run(Case(ctx, seqs, 2, dim, 32, dtype, seed=len(seqs)), 3, causal, window)


@pytest.mark.parametrize("page", [16, 32, 64, 1024])
def test_long_caches_in_parts(ctx, page):
    run(Case(ctx, [(5000, 1), (2000, 1), (0, 1)], 1, 128, page, BF, seed=page), 4)
    run(Case(ctx, [(5000, 3)], 1, 64, page, HF, seed=page), 8)
    run(Case(ctx, [(3000, 40)], 1, 128, page, BF, seed=page), 2, window=700)


def test_rows_that_see_nothing(ctx):
    """More rows than tokens: the first ones lie before token 0; and a cache without a token."""
    c = Case(ctx, [(3, 6), (0, 4), (2, 1)], 1, 128, 16)
    q, out = run(c, 2)
    assert (out[:3] == 0).all() and (out[6:10] == 0).all()


def test_peaked_and_flat_scores(ctx):
    run(Case(ctx, [(900, 2), (64, 64)], 2, 128, 16, seed=1), 4, scale=3.0)        # a few tokens have all the weight
    run(Case(ctx, [(900, 2), (64, 64)], 2, 128, 16, seed=2), 4, scale=0.0)        # all the same
    run(Case(ctx, [(900, 2), (64, 64)], 2, 128, 16, HF, seed=3), 4, scale=-0.2)
    run(Case(ctx, [(900, 2), (64, 64)], 2, 64, 16, seed=4, spread=4.0), 4)        # tokens of very different size
    run(Case(ctx, [(900, 2), (64, 64)], 2, 256, 16, HF, seed=5, spread=1.5), 4)


@pytest.mark.parametrize("power", [126, 100, -40, -56])
def test_values_of_any_size(ctx, power):
    """Values near the largest and near the smallest number; and one token alone of that size, among others of size 1."""
    for seqs in ([(40, 2), (64, 64)], [(3000, 2)]):
        for one in (False, True):
            c = Case(ctx, seqs, 1, 128, 16, seed=power & 15)
            for s, (k, v) in enumerate(c.kv):
                pick = slice(7, 8) if one else slice(None)
                v[pick] = (v[pick].double().clamp(-1, 1) * 2.0 ** power).to(BF)
            ctx.kv4_append(c.cache, c.all, *(torch.cat([x[j] for x in c.kv]).cuda() for j in range(2)))
            run(c, 2)


def test_tokens_that_are_nan_touch_only_rows_that_see_them(ctx):
    import paper_2509_05576_amd as fobq
    c = Case(ctx, [(80, 40)], 1, 128, 16, seed=3)
    k, v = (x.clone() for x in c.kv[0])
    v[60, 0, 3] = math.nan
    ctx.kv4_append(c.cache, c.all, k.cuda(), v.cuda())
    q = c.queries(2)
    out = ctx.kv4_attention(c.cache, c.batch(), q.cuda()).cpu()
    assert out[20:].isnan().all() and not out[:20].isnan().any()
    k[60, 0, 3] = math.inf
    ctx.kv4_append(c.cache, c.all, k.cuda(), c.kv[0][1].cuda())
    out = ctx.kv4_attention(c.cache, c.batch(), q.cuda()).cpu()
    assert out[20:].isnan().all() and not out[:20].isnan().any()
    q[5, 1] = math.nan
    ctx.kv4_append(c.cache, c.all, c.kv[0][0].cuda(), c.kv[0][1].cuda())
    out = ctx.kv4_attention(c.cache, c.batch(), q.cuda()).cpu()
    bad = torch.zeros((40, 2), dtype=torch.bool)
    bad[5, 1] = True
    assert torch.equal(out.isnan().all(-1), bad) and torch.equal(out.isnan().any(-1), bad)


def test_strides_and_neighbours(ctx):
    """Queries, keys and values as parts of one product's rows; results into a part of a larger tensor; rows of no sequence."""
    import paper_2509_05576_amd as fobq
    heads, group, dim = 2, 3, 128
    c = Case(ctx, [(50, 3), (20, 1)], heads, dim, 16, seed=8)
    both = torch.randn((c.rows + 2, heads * group + 2 * heads, dim + 2), generator=c.g).to(BF).cuda()
    q, k, v = both[:, :heads * group, 1:dim + 1], both[:, heads * group:heads * (group + 1), 1:dim + 1], both[:, heads * (group + 1):, 1:dim + 1]
    whole = torch.full((c.rows + 2, heads * group + 1, dim + 8), 3.0, dtype=BF, device="cuda")
    out = whole[:, 1:, 8:]
    before = c.cache.k_codes.clone()
    ctx.kv4_append(c.cache, c.batch(), k, v)
    at = 0
    for s, (n, new) in enumerate(c.seqs):
        c.kv[s][0][n - new:], c.kv[s][1][n - new:] = k[at:at + new].cpu(), v[at:at + new].cpu()
        at += new
    want = Case(ctx, c.seqs, heads, dim, 16, seed=8)
    want.kv = c.kv
    ctx.kv4_append(want.cache, want.all, *(torch.cat([x[j] for x in c.kv]).cuda() for j in range(2)))
    assert torch.equal(c.cache.k_codes, want.cache.k_codes) and torch.equal(c.cache.v_grids, want.cache.v_grids) and not torch.equal(before, c.cache.k_codes)
    lse = torch.full((c.rows + 2, heads * group), 9.0, device="cuda")
    assert ctx.kv4_attention(c.cache, c.batch(), q, out=out, lse=lse) is out
    c.check(q[:c.rows].cpu(), out[:c.rows], lse[:c.rows], dim ** -0.5)
    assert (whole[:, 0] == 3).all() and (whole[:, :, :8] == 3).all() and (whole[c.rows:] == 3).all() and (lse[c.rows:] == 9).all()
    kk, vv = (torch.full((c.rows + 2, heads, dim), 4.0, device="cuda") for _ in range(2))
    ctx.kv4_read(c.cache, c.batch(), c.rows + 2, out=(kk, vv))
    assert (kk[c.rows:] == 4).all() and (vv[c.rows:] == 4).all() and not (kk[:c.rows] == 4).all()


def test_pages_that_are_none(ctx):
    """Entries outside the cache: nothing is written there, and their tokens are not there."""
    c = Case(ctx, [(100, 4)], 1, 128, 16, seed=6)
    q = c.queries(2)
    table = c.table.clone()
    table[0, 2], table[0, 4] = c.pages, -7                     # tokens 32 .. 47 and 64 .. 79
    lse = torch.zeros((4, 2), device="cuda")
    out = ctx.kv4_attention(c.cache, c.batch(table=table), q.cuda(), lse=lse).cpu().double()
    (kc, ks), (vc, vs) = c.rows_of(0)
    keep = torch.tensor([t for t in range(100) if t // 16 not in (2, 4)])
    for h in range(2):
        spans = [(0, int((keep <= 96 + i).sum())) for i in range(4)]
        want, _, bound, _ = ref.attention(q[:, h], (kc[0][keep], ks[0][keep]), (vc[0][keep], vs[0][keep]), 128 ** -0.5, spans, BF)
        assert ((out[:, h] - want).abs() <= bound).all()
    before = [t.clone() for t in (c.cache.k_codes, c.cache.v_codes, c.cache.k_grids, c.cache.v_grids)]
    table[0, 6] = 2 ** 30
    ctx.kv4_append(c.cache, c.batch(table=table), *(torch.ones((4, 1, 128), dtype=BF, device="cuda") for _ in range(2)))
    assert all(torch.equal(a, b) for a, b in zip(before, (c.cache.k_codes, c.cache.v_codes, c.cache.k_grids, c.cache.v_grids)))
    k, v = ctx.kv4_read(c.cache, c.batch(table=table), 4, torch.float32)
    assert (k == 0).all() and (v == 0).all()
    # lengths behind the table: the tokens that the table has
    short, q1 = c.table[:, :6].contiguous(), c.queries(1).cuda()
    got = [ctx.kv4_attention(c.cache, c.batch(table=short, lengths=torch.tensor([n], dtype=torch.int32)), q1, causal=False) for n in (1 << 30, 96)]
    assert torch.equal(*got) and not got[0].isnan().any()
    none = ctx.kv4_attention(c.cache, c.batch(lengths=torch.tensor([-5], dtype=torch.int32)), q1, causal=False)
    assert (none == 0).all()


def test_pages_that_are_none_and_nan_in_a_long_sequence(ctx):
    """The same where a sequence is split: parts without a token, parts that are NaN for the rows that see them only."""
    c = Case(ctx, [(4000, 3)], 1, 128, 16, seed=16)
    q = c.queries(2)
    table = c.table.clone()
    table[0, 20:150] = -1                                      # tokens 320 .. 2399
    table[0, 240] = c.pages
    lse = torch.zeros((3, 2), device="cuda")
    out = ctx.kv4_attention(c.cache, c.batch(table=table), q.cuda(), lse=lse).cpu().double()
    (kc, ks), (vc, vs) = c.rows_of(0)
    keep = torch.tensor([t for t in range(4000) if not 20 <= t // 16 < 150 and t // 16 != 240])
    for h in range(2):
        spans = [(0, int((keep <= 3997 + i).sum())) for i in range(3)]
        want, _, bound, _ = ref.attention(q[:, h], (kc[0][keep], ks[0][keep]), (vc[0][keep], vs[0][keep]), 128 ** -0.5, spans, BF)
        assert ((out[:, h] - want).abs() <= bound).all()
    table[:] = -1
    out = ctx.kv4_attention(c.cache, c.batch(table=table), q.cuda(), lse=lse)
    assert (out == 0).all() and (lse == -math.inf).all()
    k, v = (x.clone() for x in c.kv[0])
    v[3998, 0, 3] = math.nan
    ctx.kv4_append(c.cache, c.all, k.cuda(), v.cuda())
    out = ctx.kv4_attention(c.cache, c.batch(), q.cuda()).cpu()
    assert out[1:].isnan().all() and not out[:1].isnan().any()


def test_without_starts(ctx):
    c = Case(ctx, [(70, 1), (5, 1), (33, 1)], 2, 128, 16, seed=12)
    q = c.queries(4).cuda()
    assert torch.equal(ctx.kv4_attention(c.cache, c.batch(starts=None), q), ctx.kv4_attention(c.cache, c.batch(), q))
    a, b = ctx.kv4_read(c.cache, c.batch(starts=None), 3), ctx.kv4_read(c.cache, c.batch(), 3)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_without_starts_rows_behind_the_last_sequence_stay(ctx):
    for rows in (5, 5000):
        c = Case(ctx, [(70, 1), (5, 1), (33, 1)], 2, 128, 16, seed=12)
        before = [t.clone() for t in (c.cache.k_codes, c.cache.v_codes, c.cache.k_grids, c.cache.v_grids)]
        kv = torch.randn((rows, 4, 128), generator=c.g).to(BF).cuda()
        kv[:3, :2], kv[:3, 2:] = (torch.stack([x[j][-1] for x in c.kv]).cuda() for j in range(2))     # what is there already
        ctx.kv4_append(c.cache, c.batch(starts=None), kv[:, :2], kv[:, 2:])
        assert all(torch.equal(a, b) for a, b in zip(before, (c.cache.k_codes, c.cache.v_codes, c.cache.k_grids, c.cache.v_grids)))
        out = tuple(torch.full((rows, 2, 128), 4.0, device="cuda") for _ in range(2))
        k, v = ctx.kv4_read(c.cache, c.batch(starts=None), rows, out=out)
        assert (k[3:] == 4).all() and (v[3:] == 4).all() and not (k[:3] == 4).any()
        q = torch.randn((rows, 4, 128), generator=c.g).to(BF).cuda()
        o = torch.full((rows, 4, 128), 4.0, dtype=BF, device="cuda")
        ctx.kv4_attention(c.cache, c.batch(starts=None), q, out=o)
        assert (o[3:] == 4).all()
        c.check(q[:3].cpu(), o[:3], ctx_lse(ctx, c, q[:3]), 128 ** -0.5)


def ctx_lse(ctx, c, q):
    lse = torch.zeros((q.shape[0], q.shape[1]), device="cuda")
    ctx.kv4_attention(c.cache, c.batch(starts=None), q, lse=lse)
    return lse


def test_many_rows_of_many_sequences(ctx):
    """More rows than a wavefront each: sequences that end inside a group of four, empty ones between them."""
    g = torch.Generator().manual_seed(2)
    seqs = []
    while sum(n for n, _ in seqs) < 5000:
        n = int(torch.randint(0, 90, (1,), generator=g))
        seqs.append((n, min(n, int(torch.randint(0, 5, (1,), generator=g)))))
    c = Case(ctx, seqs, 1, 64, 16, seed=3)
    k, v = ctx.kv4_read(c.cache, c.all, c.tokens, torch.float32)
    at = 0
    for s, (n, _) in enumerate(c.seqs):
        for j, (got, (level, scale)) in enumerate(zip((k, v), c.rows_of(s))):
            assert torch.equal(got[at:at + n].cpu(), (level * scale[..., None]).transpose(0, 1).float())
            codes, want_scale, zero = ref.grid(c.kv[s][j].transpose(0, 1))
            assert torch.equal(scale, want_scale) and torch.equal(level, codes - zero[..., None])
        at += n
    run(c, 2)


def test_the_hint_of_the_longest_changes_no_coverage(ctx):
    c = Case(ctx, [(3000, 1)], 1, 128, 64, seed=13)
    for longest in (0, 1, 500, 3000, 1 << 20):
        run(c, 4, max_length=longest)


@pytest.mark.parametrize("count", [70, 300])
def test_prompts_of_many_sequences(ctx, count):
    """Rows of their own for every wavefront, more sequences than a wavefront has lanes, and than are put in order; empty ones between."""
    g = torch.Generator().manual_seed(count)
    seqs = [(int(n) + 60, 60) if i % 7 else (i, 0) for i, n in enumerate(torch.randint(0, 90, (count,), generator=g))]
    run(Case(ctx, seqs, 1, 64, 16, [BF, HF][count == 70], seed=count), 1)


def test_a_window_beyond_every_length(ctx):
    c = Case(ctx, [(100, 3), (40, 40)], 1, 128, 16, seed=17)
    q = c.queries(2).cuda()
    want = ctx.kv4_attention(c.cache, c.batch(), q)
    for window in (101, 1 << 20, (1 << 31) - 1, (1 << 32) + 1):
        assert torch.equal(ctx.kv4_attention(c.cache, c.batch(), q, window=window), want)


def test_starts_out_of_order_stay_in_bounds(ctx):
    """No such call has a meaning; nothing outside the arguments is touched by it, and the next one is right."""
    c = Case(ctx, [(2000, 2), (900, 1), (0, 1), (300, 2)], 2, 128, 16, seed=15)
    q = c.queries(4)
    whole = torch.full((c.rows + 4, 8, 128), 3.0, dtype=BF, device="cuda")
    for bad in ([0, 6, 0, 6, 0], [5, 4, 3, 2, 1], [-9, 2 ** 31 - 1, -5, 2 ** 31 - 1, 6], [2 ** 31 - 1] * 5):
        ctx.kv4_attention(c.cache, c.batch(starts=torch.tensor(bad, dtype=torch.int32)), q.cuda(), out=whole[2:-2])
        ctx.kv4_read(c.cache, c.batch(starts=torch.tensor(bad, dtype=torch.int32)), c.rows)
    assert (whole[:2] == 3).all() and (whole[-2:] == 3).all()
    run(c, 4)


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_ragged_sequences_in_parts_of_equal_size(ctx, dim):
    """Lengths from none to thousands in one call, several sequences in several parts, more of them than a wavefront has lanes."""
    g = torch.Generator().manual_seed(dim)
    seqs = [(int(n), 1) for n in (torch.rand(100, generator=g) ** 6 * 3000)] + [(4000, 2), (0, 1), (1500, 9), (5, 5)]
    run(Case(ctx, seqs, 1, dim, 32, [BF, HF][dim == 128], seed=dim), 2)
    run(Case(ctx, [(3000, 1), (10, 1), (2500, 70)], 2, dim, 16, BF, seed=dim), 3, window=1500)
    run(Case(ctx, [(3000, 60)], 1, dim, 64, HF, seed=dim), 5, causal=False)


def test_generation_step_by_step(ctx):
    """The calls together, as a program that generates makes them: a prompt, then single tokens, against one call over all."""
    import paper_2509_05576_amd as fobq
    heads, group, dim, page, total = 2, 4, 128, 16, 70
    g = torch.Generator(device="cuda").manual_seed(4)
    rows = torch.randn((total, heads * (group + 2), dim), generator=g, device="cuda").to(BF)
    q, k, v = rows[:, :heads * group], rows[:, heads * group:heads * (group + 1)], rows[:, heads * (group + 1):]
    cache = fobq.Kv4Cache.empty(6, heads, dim, page)
    table = torch.tensor([[3, 0, 5, 1, 2, 4]], dtype=torch.int32).cuda()
    outs = []
    for first, last in [(0, 50)] + [(i, i + 1) for i in range(50, total)]:
        batch = fobq.Kv4Batch(table, torch.tensor([last], dtype=torch.int32).cuda(), torch.tensor([0, last - first], dtype=torch.int32).cuda())
        ctx.kv4_append(cache, batch, k[first:last], v[first:last])
        outs.append(ctx.kv4_attention(cache, batch, q[first:last]))
    whole = fobq.Kv4Batch(table, torch.tensor([total], dtype=torch.int32).cuda(), torch.tensor([0, total], dtype=torch.int32).cuda())
    at_once = ctx.kv4_attention(cache, whole, q)
    # either is within a rounding and the weights' 2^-11 of the exact one; |out| is below 3 here
    assert (torch.cat(outs).float() - at_once.float()).abs().max() <= 2 * 3 * (2.0 ** -8 + 2.0 ** -10)


def test_offsets_behind_32_bits(ctx):
    """A cache whose codes take more than 4 GiB: its last pages, against the same tokens in a small cache."""
    import paper_2509_05576_amd as fobq
    small = Case(ctx, [(100, 2)], 1, 256, 64, seed=21)
    pages = (1 << 32) // (64 * 128) + 8
    big = fobq.Kv4Cache.empty(pages, 1, 256, 64)
    table = torch.tensor([[pages - 1, pages - 3, 0]], dtype=torch.int32)
    ctx.kv4_append(big, small.batch(table=table, starts=torch.tensor([0, 100], dtype=torch.int32)), small.kv[0][0].cuda(), small.kv[0][1].cuda())
    q = small.queries(2).cuda()
    assert torch.equal(ctx.kv4_attention(big, small.batch(table=table), q), ctx.kv4_attention(small.cache, small.batch(), q))
    a, b = ctx.kv4_read(big, small.batch(table=table), 2), ctx.kv4_read(small.cache, small.batch(), 2)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_refusals(ctx):
    import ctypes

    import paper_2509_05576_amd as fobq
    c = Case(ctx, [(20, 2)], 2, 128, 16)
    q = c.queries(2).cuda()
    with pytest.raises(TypeError):
        ctx.kv4_attention(c.cache, c.batch(), q.float())
    with pytest.raises(TypeError):
        ctx.kv4_attention(c.cache, c.batch(), q[:, :3])
    with pytest.raises(TypeError):
        ctx.kv4_attention(c.cache, c.batch(lengths=torch.zeros(2, dtype=torch.int32)), q)
    with pytest.raises(TypeError):
        ctx.kv4_attention(c.cache, c.batch(lengths=torch.zeros(1, dtype=torch.int64)), q)
    with pytest.raises(TypeError):
        ctx.kv4_append(c.cache, c.batch(), q, q)
    with pytest.raises(TypeError):
        ctx.kv4_append(c.cache, c.batch(), *(torch.zeros((2, 2, 128), device="cuda") for _ in range(2)))
    for kw in (dict(window=-1), dict(scale=math.nan), dict(max_length=-1)):
        with pytest.raises(fobq.FobqError) as e:
            ctx.kv4_attention(c.cache, c.batch(), q, **kw)
        assert e.value.code == fobq.EINVAL
    for pages, heads, dim, page in [(1, 1, 96, 16), (1, 1, 128, 8), (1, 1, 128, 48), (1, 1, 32, 16)]:
        with pytest.raises(fobq.FobqError) as e:
            ctx.kv4_read(fobq.Kv4Cache.empty(pages, heads, dim, page), c.batch(), 2)
        assert e.value.code == fobq.EINVAL
    cc, bb = (t.from_buffer_copy(x) for t, x in zip((ref.CacheStruct, ref.BatchStruct), fobq.binding._kv4(ctx.handle, c.cache, c.batch(), 2)))
    lib = fobq.load_library()
    z = torch.zeros((2, 2, 128), dtype=BF, device="cuda")
    call = lambda: lib.fobq_kv4_append(ctx.handle, ctypes.byref(cc), ctypes.byref(bb), 1, z.data_ptr(), 256, 128, z.data_ptr(), 256, 128)  # noqa: E731
    assert call() == fobq.OK
    for s, field, value in [(cc, "pages", 0), (cc, "heads", 0), (cc, "reserved", 1), (cc, "k_codes", None), (cc, "v_grids", cc.v_grids + 4), (bb, "rows", -1),
                            (bb, "n_seqs", -1), (bb, "max_pages", 99), (bb, "lengths", None), (bb, "table", None)]:
        old = getattr(s, field)
        setattr(s, field, value)
        assert call() == fobq.EINVAL, field
        setattr(s, field, old)
    long = Case(ctx, [(3000, 1)], 1, 128, 64)
    cc, bb = (t.from_buffer_copy(x) for t, x in zip((ref.CacheStruct, ref.BatchStruct), fobq.binding._kv4(ctx.handle, long.cache, long.batch(), 1)))
    qq = long.queries(1).cuda()
    d = ref.QueryStruct(qq.data_ptr(), qq.data_ptr(), None, 128, 128, 128, 128, 0, 1, 1, 1, 0, 1.0, 0)
    need = ctypes.c_int64(0)
    assert lib.fobq_kv4_attention_workspace(ctx.handle, ctypes.byref(cc), ctypes.byref(bb), ctypes.byref(d), ctypes.byref(need)) == fobq.OK and need.value > 0
    assert lib.fobq_kv4_attention(ctx.handle, ctypes.byref(cc), ctypes.byref(bb), ctypes.byref(d), None, 0) == fobq.EINVAL
    assert b"work must be" in lib.fobq_last_error(ctx.handle)
    torch.cuda.synchronize()
