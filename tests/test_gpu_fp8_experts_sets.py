"""Products of experts' rows by two sets of wavefronts that deal the blocks of columns among them: as many blocks each, one more in the first, and a rest behind."""
import pytest

torch = pytest.importorskip("torch")
import test_gpu_fp8_experts as forms

pytestmark = pytest.mark.gpu
ctx = forms.ctx
F32, BF, HF, E4, E5 = forms.F32, forms.BF, forms.HF, forms.E4, forms.E5


@pytest.mark.parametrize("counts,n", [([20, 5, 64, 31], 1000), ([100, 0, 70, 1, 30], 520)])
@pytest.mark.parametrize("dtype,per", [(BF, 128), (HF, 1), (F32, 128), (F32, 1)])
@pytest.mark.parametrize("k", [2048, 2064, 2176, 2200, 2432])
def test_blocks_dealt_to_two_sets(ctx, k, dtype, per, counts, n):
    import paper_2509_05576_amd as fobq
    cus, rows = torch.cuda.get_device_properties(0).multi_processor_count, sum(counts)
    args = [cus, rows, len(counts), n, k, {F32: 0, BF: 1, HF: 2}[dtype], per]
    tm, tn, _, sets = fobq.fobq_debug_plan(fobq.PLAN_EXPERTS, args, 4)
    assert (tm, tn, sets) == (64, 64, 2)
    args[4] = 1920
    assert fobq.fobq_debug_plan(fobq.PLAN_EXPERTS, args, 4)[3] == 1
    r = forms._routing(counts, 1, none=3)
    for fa, fb in ((E4, E4), (E5, E4)):
        forms.check(ctx, forms._matrix(ctx, rows + 3, k, fa, 1, 5), forms._weights(ctx, len(counts), n, k, fb, per), r, dtype, False)
