"""A strong token before a long tail of weak ones: the tail's part of the result, where the strong token has none."""
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


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("seqs,dim", [([(900, 2)], 128), ([(20000, 1)], 64), ([(3000, 1)], 256), ([(2000, 140)], 128)])
@pytest.mark.parametrize("below", [10, 15, 18, 22, 25, 27])
def test_a_tail_behind_a_strong_token(ctx, below, seqs, dim, dtype):
    """Token 5 scores `below` binary orders above all others and has its values in channel 0 alone, the others theirs in the rest."""
    (n, new), = seqs
    c = Case(ctx, seqs, 1, dim, 16, dtype, seed=below, spread=0.0)
    k, v = (x.clone() for x in c.kv[0])
    k[:] = 0.0
    k[5, 0, :8] = 1.0
    v[..., 0], v[5] = 0.0, 0.0
    v[5, 0, 0] = 1.0
    v[:, 0, 1:9] = torch.where(torch.arange(n) == 5, 0.0, 1.0)[:, None]         # (and eight channels where the tail does not cancel)
    ctx.kv4_append(c.cache, c.all, k.cuda(), v.cuda())
    q = torch.zeros((new, 1, dim), dtype=dtype)
    q[..., :8] = 1.0
    (kc, ks), (vc, vs) = c.rows_of(0)
    top = float((kc[0, 5, :8] * ks[0, 5]).sum())
    scale = below * math.log(2.0) / top
    out = ctx.kv4_attention(c.cache, c.batch(), q.cuda(), scale=scale).cpu().double()
    for i, (a, b) in enumerate(c.spans(0, True, 0)):
        s = (kc[0, a:b] @ q[i, 0].double()) * ks[0, a:b] * torch.tensor(scale, dtype=torch.float32).double()
        p = (s - s.max()).exp()
        val = vc[0, a:b] * vs[0, a:b, None]
        want = p @ val / p.sum()
        # scores of up to 27 orders with sums of dim terms of 143 at most in fp32; weights times scales 2^-11 each, below 2^-20 of the largest (which has
        # one of two scales) to half of 2^-30 of it; sums of b fp32 terms; the result's rounding, also where that is denormal
        ds = (dim + 8) * ref.U * 2 * 143 * 8 * float(ks[0, 5]) * scale + 60 * ref.U * below
        fine = (2.0 ** -11 * 1.01 + 2 * ds + (b + 64) * ref.U) * (p @ val.abs())
        lost = ((p * vs[0, a:b] < 2.0 ** -19 * float(vs[0, 5]))[:, None] * vc[0, a:b].abs()).sum(0) * 2.0 ** -31 * 2 * float(vs[0, 5])
        bound = (fine + lost) / p.sum() + ref.HALF[dtype] * want.abs() * 1.01 + torch.finfo(dtype).smallest_normal * ref.HALF[dtype] * 1.01
        off = (out[i, 0] - want).abs()
        assert (off <= bound).all(), (i, float((off / bound).max()))
        # the tail is there: eight channels are its weight's share of 1, and what is lost of it is less than a fifth
        assert (want[1:9] > 0.5 * (b - 1) * 2.0 ** -below / (1 + b * 2.0 ** -below)).all()
        assert below > 25 or (off[1:9] <= 0.2 * want[1:9] + torch.finfo(dtype).smallest_normal * ref.HALF[dtype] * 1.01).all()
