"""Sequences that say they hold more tokens than their table has places for: nothing is stored in another token's place, and rows see the
tokens that they would see and that are there."""
import math

import pytest

torch = pytest.importorskip("torch")
import lowbit_reference as ref
from test_gpu_kv4 import BF, HF, Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    import paper_2509_05576_amd as fobq
    c = fobq.Ctx(0)
    yield c
    c.close()


def parts(cache):
    return cache.k_codes, cache.v_codes, cache.k_grids, cache.v_grids


@pytest.mark.parametrize("length,new", [(65, 1), (66, 1), (70, 10), (64 + 70, 100), (1 << 30, 3), (2 ** 31 - 1, 5)])
@pytest.mark.parametrize("page", [16, 64])
def test_append_and_read(ctx, page, length, new):
    """A table for 64 tokens, all held."""
    c = Case(ctx, [(64, 64)], 2, 128, page, seed=new)
    table, before = c.table[:, :64 // page].contiguous(), [t.clone() for t in parts(c.cache)]
    batch = c.batch(table=table, lengths=torch.tensor([length], dtype=torch.int32), starts=torch.tensor([0, new], dtype=torch.int32))
    k, v = (torch.randn((new, 2, 128), generator=c.g).to(BF).cuda() for _ in range(2))
    ctx.kv4_append(c.cache, batch, k, v)
    tokens = [length - new + i for i in range(new)]
    there = [i for i, t in enumerate(tokens) if t < 64]
    # as if the rows that have a place had been appended alone
    want = Case(ctx, [(64, 64)], 2, 128, page, seed=new)
    if there:
        first = there[0]
        assert tokens[first] == length - new and tokens[there[-1]] == 63
        want.ctx.kv4_append(want.cache, want.batch(table=table, lengths=torch.tensor([64], dtype=torch.int32), starts=torch.tensor([0, len(there)], dtype=torch.int32)),
                            k[:len(there)].contiguous(), v[:len(there)].contiguous())
    assert all(torch.equal(a, b) for a, b in zip(parts(c.cache), parts(want.cache)))
    assert all(torch.equal(a, b) for a, b in zip(parts(c.cache), before)) == (not there)
    rk, rv = ctx.kv4_read(c.cache, batch, new, torch.float32)
    assert (rk[len(there):] == 0).all() and (rv[len(there):] == 0).all()
    for got, (level, scale) in zip((rk, rv), c.rows_of(0)):
        for i in there:
            assert torch.equal(got[i].cpu(), (level * scale[..., None])[:, tokens[i]].float())


FORMS = {"few rows": ([(64, 1), (32, 9)], 2, 128), "prompts": ([(96, 90), (64, 40)], 2, 64), "wide prompts": ([(96, 70), (32, 32)], 1, 256),
         "parts": ([(2048, 3), (1024, 1)], 1, 128), "parts of prompts": ([(1536, 70)], 2, 128), "one token": ([(16, 1)], 1, 256)}


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("over", [1, 5, 60, 100])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 50), (False, 70)])
def test_attention(ctx, form, over, causal, window):
    """Every sequence's table is full, and its length passes it by `over` tokens."""
    seqs, group, dim = FORMS[form]
    c = Case(ctx, seqs, 2, dim, 16, [BF, HF][over % 2], seed=over)
    # every sequence's own pages, and none behind the shorter ones
    pages = max(n for n, _ in seqs) // 16
    table = c.table[:, :pages].contiguous()
    lengths = torch.tensor([n + over for n, _ in seqs], dtype=torch.int32)
    q = c.queries(group)
    lse = torch.full((c.rows, 2 * group), 5.0, device="cuda")
    out = ctx.kv4_attention(c.cache, c.batch(table=table, lengths=lengths), q.cuda(), causal=causal, window=window, lse=lse).cpu().double()
    lse, at = lse.cpu().double(), 0
    for s, (n, new) in enumerate(seqs):
        (kc, ks), (vc, vs) = c.rows_of(s)
        spans = []
        for i in range(new):
            end = n + over - new + i + 1 if causal else n + over
            start = max(0, end - window) if window else 0
            spans.append((start, max(start, min(end, n))))
        seen = torch.tensor([b > a for a, b in spans])
        for hq in range(2 * group):
            h = hq // group
            want, wl, bound, lbound = ref.attention(q[at:at + new, hq], (kc[h], ks[h]), (vc[h], vs[h]), dim ** -0.5, spans, c.dtype)
            off = (out[at:at + new, hq] - want).abs()
            assert (off <= bound).all(), (s, hq, (off / bound.clamp(min=1e-300)).max())
            assert (lse[at:at + new, hq][~seen] == -math.inf).all()
            assert ((lse[at:at + new, hq] - wl).abs()[seen] <= lbound[seen]).all()
        at += new


@pytest.mark.parametrize("seqs,group,dim", [([(2, 10), (40, 3)], 2, 128), ([(30, 100)], 1, 64), ([(1500, 1600)], 1, 128), ([(1500, 3), (4, 20)], 1, 128)])
def test_rows_before_token_0_under_a_window_beyond_every_length(ctx, seqs, group, dim):
    """Few rows, prompts, and split sequences: the rows before token 0 see nothing, the others all that is there up to their own."""
    c = Case(ctx, seqs, 1, dim, 16, BF, seed=dim)
    q = c.queries(group).cuda()
    lse = torch.empty((c.rows, group), device="cuda")
    want = ctx.kv4_attention(c.cache, c.batch(), q, lse=lse)
    for window in ((1 << 31) - 1, (1 << 31) - 5, (1 << 31) - 9, 1 << 30, 5000):
        got_lse = torch.empty_like(lse)
        assert torch.equal(ctx.kv4_attention(c.cache, c.batch(), q, window=window, lse=got_lse), want) and torch.equal(lse, got_lse), window
    assert (want[:max(0, seqs[0][1] - seqs[0][0])] == 0).all() and not (want[-1] == 0).all()
