"""The host side of a feed-forward part of experts: what is refused, and how calls are cut into workgroups (no GPU)."""
import ctypes

import pytest

torch = pytest.importorskip("torch")
import paper_2509_05576_amd as fobq

A = 0x7000000000          # an address that nothing follows


def verdict(what, fields, change):
    assert set(change) <= set(fields)
    return fobq.fobq_debug_plan(what, list({**fields, **change}.values()), 1)


def expect(ok):
    return [fobq.OK if ok else fobq.EINVAL]


NORM = dict(rows=9, cols=300, x_ld=300, residual_ld=300, sum_ld=300, norm_ld=300, type=1, weight_type=1, eps=0, x=A, residual=A, weight=A, sum=A, norm=A)


@pytest.mark.parametrize("change,ok", [
    ({}, True), (dict(residual=0, sum=0, norm=0, weight=0), True), (dict(residual=0, residual_ld=0), True), (dict(sum=0, sum_ld=0), True),
    (dict(norm=0, norm_ld=-1), True), (dict(weight_type=0), True), (dict(type=0, weight_type=0), True), (dict(rows=0, x=0), True), (dict(cols=1), True),
    (dict(cols=32768, x_ld=32768, residual_ld=32768, sum_ld=32768, norm_ld=32768), True), (dict(x_ld=400, residual_ld=301), True), (dict(x=A + 2), True),
    (dict(cols=32769, x_ld=40000, residual_ld=40000, sum_ld=40000, norm_ld=40000), False), (dict(cols=0), False), (dict(rows=-1), False), (dict(x=0), False),
    (dict(x=A + 1), False), (dict(residual=A + 1), False), (dict(weight=A + 1), False), (dict(weight=A + 2, weight_type=0), False), (dict(sum=A + 1), False),
    (dict(norm=A + 1), False), (dict(x_ld=299), False), (dict(residual_ld=299), False), (dict(sum_ld=299), False), (dict(norm_ld=299), False), (dict(type=3), False),
    (dict(type=0), False), (dict(weight_type=2), False), (dict(eps=-1), False), (dict(eps=1), False), (dict(rows=1 << 27), False)])
def test_norms(change, ok):
    assert verdict(fobq.PLAN_NORM_CHECK, NORM, change) == expect(ok)


ROUTE = dict(tokens=5, ld=64, type=0, experts=64, top_k=8, score=0, groups=8, top_groups=4, group_top=2, reserved=0, logits=A, bias=A, chosen=A, weights=A, starts=A,
             pairs=A, places=A)


@pytest.mark.parametrize("change,ok", [
    ({}, True), (dict(bias=0), True), (dict(tokens=0, logits=0, chosen=0, weights=0, pairs=0, places=0), True), (dict(score=1, type=1), True), (dict(ld=100), True),
    (dict(experts=1024, ld=1024, groups=64, top_groups=64, top_k=32), True), (dict(groups=1, top_groups=1, top_k=32), True), (dict(top_k=32), True),
    (dict(experts=1, ld=1, groups=1, top_groups=1, top_k=1), True), (dict(tokens=(1 << 26) - 4, top_k=7), True),
    (dict(top_k=33, top_groups=8), False), (dict(top_k=0), False), (dict(top_groups=1, top_k=9), False), (dict(experts=1025, ld=2000, groups=1, top_groups=1), False),
    (dict(experts=0, groups=1, top_groups=1), False), (dict(groups=7), False), (dict(groups=0), False), (dict(experts=130, ld=130, groups=65, top_groups=65), False),
    (dict(top_groups=0), False), (dict(top_groups=9), False), (dict(group_top=0), False), (dict(group_top=3), False), (dict(score=2), False), (dict(type=3), False),
    (dict(ld=63), False), (dict(reserved=1), False), (dict(tokens=-1), False), (dict(tokens=(1 << 26) - 3, top_k=1), False), (dict(tokens=(1 << 26) - 4, top_k=9), False),
    (dict(logits=0), False), (dict(logits=A + 2), False), (dict(bias=A + 2), False), (dict(chosen=0), False), (dict(weights=A + 1), False), (dict(starts=0), False),
    (dict(starts=0, tokens=0), False), (dict(pairs=0), False), (dict(places=A + 2), False)])
def test_routers(change, ok):
    assert verdict(fobq.PLAN_ROUTE_CHECK, ROUTE, change) == expect(ok)


EXPERTS = dict(m=40, k=300, rows=100, cols=300, ld=304, expert_values=30400, expert_scales=300, experts=7, per=1, b=A, pairs=A, top_k=2, packed=80, type=1, y_ld=100)


@pytest.mark.parametrize("change,ok", [
    ({}, True), (dict(type=0), True), (dict(y_ld=200), True), (dict(pairs=0, m=80), True), (dict(pairs=0, m=81), True), (dict(packed=0), True), (dict(experts=1024), True),
    (dict(expert_values=0, expert_scales=0), True), (dict(per=128), True), (dict(pairs=0), False), (dict(k=301), False), (dict(ld=288), False), (dict(ld=305), False),
    (dict(expert_values=30401), False), (dict(expert_values=-16), False), (dict(expert_scales=-1), False), (dict(experts=0), False), (dict(experts=1025), False),
    (dict(per=64), False), (dict(b=0), False), (dict(b=A + 4), False), (dict(top_k=0), False), (dict(top_k=33), False), (dict(packed=-1), False),
    (dict(packed=(1 << 26) - 3), False), (dict(type=4), False), (dict(y_ld=99), False), (dict(ld=1 << 24), False), (dict(rows=-1), False),
    (dict(packed=(1 << 26) - 4, rows=1 << 20, y_ld=1 << 20), False)])
def test_expert_products(change, ok):
    assert verdict(fobq.PLAN_EXPERTS_CHECK, EXPERTS, change) == expect(ok)


SUM = dict(type=1, rows=80, cols=100, ld=100, tokens=40, top_k=2, base=A, base_ld=100, out_ld=100)


@pytest.mark.parametrize("change,ok", [
    ({}, True), (dict(base=0, base_ld=0), True), (dict(rows=0), True), (dict(tokens=0), True), (dict(cols=0), True), (dict(ld=200, out_ld=101), True), (dict(top_k=32), True),
    (dict(type=5), False), (dict(rows=-1), False), (dict(rows=(1 << 26) - 3), False), (dict(tokens=-1), False), (dict(cols=-1), False), (dict(ld=99), False),
    (dict(base_ld=99), False), (dict(out_ld=99), False), (dict(top_k=0), False), (dict(top_k=33), False),
    (dict(tokens=1 << 20, cols=1 << 17, ld=1 << 17, base_ld=1 << 17, out_ld=1 << 17), False)])
def test_sums(change, ok):
    assert verdict(fobq.PLAN_SUM_CHECK, SUM, change) == expect(ok)


@pytest.mark.parametrize("experts", [1, 7, 256, 1024])
def test_tokens_are_covered(experts):
    for tokens in (0, 1, 63, 64, 65, 1000, 16384, 16385, 100000, (1 << 26) - 4):
        parts, per, work = fobq.fobq_debug_plan(fobq.PLAN_ROUTE, [tokens, experts], 3)
        assert 1 <= parts <= 256 and per % 64 == 0 and parts * per >= tokens and (parts == 1 or (parts - 1) * per < tokens)
        assert work == (16 * parts * -(-experts // 4) if parts > 1 else 0)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("per", [1, 128])
def test_tiles_are_enough(dtype, per):
    """However the packed rows are dealt among the experts: the most tiles have those with one row more than whole tiles."""
    for rows in (1, 2, 15, 16, 17, 100, 999, 32768):
        for experts in (1, 2, 7, 64, 1024):
            for n in (1, 64, 65, 1000, 4096):
                tm, tn, tiles = fobq.fobq_debug_plan(fobq.PLAN_EXPERTS, [256, rows, experts, n, 2048, dtype, per], 3)
                with_rows = min(rows, experts)
                down, across = with_rows + (rows - with_rows) // tm, -(-n // tn)     # one row each, and then whole tiles
                assert down * across <= tiles <= (rows // tm + with_rows) * across


def test_null_contexts():
    lib, null, n = fobq.load_library(), ctypes.c_void_p(None), ctypes.c_int64(0)
    assert lib.fobq_fp8_rms_norm(null, None, None) == fobq.EINVAL
    assert lib.fobq_fp8_swiglu(null, null, 0, 1, None) == fobq.EINVAL
    assert lib.fobq_route(null, None, None, null, 0) == fobq.EINVAL
    assert lib.fobq_route_workspace(null, 1, 1, ctypes.byref(n)) == fobq.EINVAL
    assert lib.fobq_fp8_expert_matmul(null, None, None, null, null, 1, 1, null, 0, 1) == fobq.EINVAL
    assert lib.fobq_expert_sum(null, null, 0, 1, 1, 1, null, null, 1, 1, null, 1, null, 1) == fobq.EINVAL


def test_host_tensors_are_refused():
    x = torch.zeros((4, 128))
    m = fobq.Fp8Matrix(x.to(torch.float8_e4m3fn), torch.ones((1, 4)))
    r, e = fobq.Routing.empty(4, 2, 1, device="cpu"), fobq.Fp8Experts.empty(2, 8, 128, device="cpu")
    for call in (lambda: fobq.fobq_fp8_rms_norm(1, x), lambda: fobq.fobq_fp8_swiglu(1, x), lambda: fobq.fobq_route(1, x, 2),
                 lambda: fobq.fobq_fp8_expert_matmul(1, m, e, r), lambda: fobq.fobq_expert_sum(1, x, r)):
        with pytest.raises(TypeError):
            call()
