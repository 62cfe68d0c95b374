"""The host side of the 8-bit block products and of the 4-bit cache: what is refused, where a row's token lies, and how calls are cut into
workgroups (no GPU)."""
import ctypes

import pytest

torch = pytest.importorskip("torch")
import paper_2509_05576_amd as fobq

A = 0x7000000000          # an address that nothing follows


def plan(what, args, n):
    return fobq.fobq_debug_plan(what, args, n)


GOOD = dict(rows=100, cols=300, ld=304, ld_scales=100, per=1, format=0, values=A, scales=A)


@pytest.mark.parametrize("change,ok", [
    ({}, True), (dict(rows=0), True), (dict(cols=0), True), (dict(rows=0, values=0, scales=0), True), (dict(per=128, ld_scales=1), True),
    (dict(format=1), True), (dict(ld=320), True), (dict(ld=300), False), (dict(ld=288), False), (dict(ld=306), False), (dict(ld_scales=99), False),
    (dict(rows=129, per=128, ld_scales=1), False), (dict(per=2), False), (dict(per=0), False), (dict(format=2), False), (dict(format=-1), False),
    (dict(rows=-1), False), (dict(cols=-1), False), (dict(rows=1 << 30, ld_scales=1 << 30), False), (dict(cols=1 << 30, ld=1 << 30), False),
    (dict(rows=(1 << 26) - 4, ld_scales=1 << 26), True), (dict(rows=(1 << 26) - 3, ld_scales=1 << 26), False), (dict(rows=1 << 17, cols=1 << 18, ld=1 << 18, ld_scales=1 << 26), False),
    (dict(values=0), False), (dict(scales=0), False), (dict(values=A + 8), False), (dict(scales=A + 2), False)])
def test_matrices(change, ok):
    m = {**GOOD, **change}
    assert plan(fobq.PLAN_FP8_CHECK, list(m.values()), 1) == [fobq.OK if ok else fobq.EINVAL]


CACHE = dict(pages=10, page_size=16, heads=2, head_dim=128, reserved=0, n_seqs=3, rows=5, max_pages=4, table_ld=4, kc=A, vc=A, kg=A, vg=A, table=A, lengths=A)


@pytest.mark.parametrize("change,ok", [
    ({}, True), (dict(page_size=4096), True), (dict(head_dim=64), True), (dict(head_dim=256), True), (dict(n_seqs=0, lengths=0, table=0), True),
    (dict(rows=0, lengths=0), True), (dict(max_pages=0, table=0), True), (dict(table_ld=9), True), (dict(pages=0), False), (dict(pages=1 << 31), False),
    (dict(page_size=8), False), (dict(page_size=48), False), (dict(page_size=8192), False), (dict(page_size=0), False), (dict(heads=0), False),
    (dict(heads=1025), False), (dict(head_dim=96), False), (dict(head_dim=0), False), (dict(reserved=1), False), (dict(n_seqs=-1), False),
    (dict(rows=-1), False), (dict(max_pages=5), False), (dict(max_pages=-1), False), (dict(max_pages=1 << 26, table_ld=1 << 26), False),
    (dict(rows=(1 << 26) - 4), True), (dict(rows=(1 << 26) - 3), False),
    (dict(kc=0), False), (dict(vc=A + 8), False), (dict(kg=A + 4), False), (dict(vg=0), False), (dict(table=0), False), (dict(lengths=0), False)])
def test_caches(change, ok):
    c = {**CACHE, **change}
    assert plan(fobq.PLAN_KV4_CHECK, list(c.values()), 1) == [fobq.OK if ok else fobq.EINVAL]


def place(page, pages, lengths, starts, table, rows, row):
    width = len(table[0])
    return plan(fobq.PLAN_KV4_PLACE, [page, pages, width, len(lengths), rows, row] + lengths + starts + [e for t in table for e in t], 3)


def test_places():
    lengths, starts = [40, 3, 17, 0], [0, 2, 2, 5, 5]
    table = [[7, 2, 4], [1, -1, -1], [0, 9, -1], [-1, -1, -1]]
    at = lambda row, **kw: place(**{**dict(page=16, pages=10, lengths=lengths, starts=starts, table=table, rows=8, row=row), **kw})  # noqa: E731
    assert at(0) == [0, 4, 6] and at(1) == [0, 4, 7]                    # tokens 38 and 39
    assert at(2) == [2, 0, 14] and at(3) == [2, 0, 15] and at(4) == [2, 9, 0]     # sequence 1 has no rows
    for row in (5, 7):
        assert at(row)[1] == -1                                         # behind the last sequence
    # pages that are none, rows before token 0, lengths behind the table, starts out of order or out of range
    assert at(4, pages=9)[1] == -1 and at(0, table=[[7, 2, -4]] + table[1:])[1] == -1 and at(0, table=[[7, 2, 2 ** 31 - 1]] + table[1:])[1] == -1
    assert at(2, lengths=[40, 3, 2, 0])[1] == -1 and at(3, lengths=[40, 3, 2, 0]) == [2, 0, 0]
    assert at(1, lengths=[2 ** 31 - 1, 3, 17, 0]) == [0, 4, 15] and at(1, lengths=[-2 ** 31, 3, 17, 0])[1] == -1
    for bad in ([0, -5, 2 ** 31 - 1, 3, -1], [9, 8, 7, 6, 5], [2 ** 31 - 1] * 5, [-2 ** 31] * 5):
        for row in range(8):
            assert at(row, starts=bad)[1] in (-1, 0, 1, 2, 4, 7, 9)


@pytest.mark.parametrize("cus", [256, 64])
@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("per_scale", [1, 128])
def test_products_are_covered(cus, dtype, per_scale):
    for m in (0, 1, 3, 16, 17, 64, 100, 1000, 8192, 100000):
        for n in (1, 16, 130, 4608, 8192):
            for k in (0, 1, 128, 129, 2304, 8192, 100000):
                tm, tn, parts, per, work = plan(fobq.PLAN_FP8_MATMUL, [cus, m, n, k, dtype, per_scale], 5)
                blocks = -(-k // 128)
                assert tm >= 1 and tn >= 1 and parts >= 1 and per >= 1
                assert parts * per >= blocks and (parts - 1) * per < max(1, blocks)     # every block in one part, no part empty
                assert work == (4 * parts * m * n if parts > 1 else 0)
                assert work == plan(fobq.PLAN_FP8_MATMUL, [cus, m, n, k, dtype, 128], 5)[4]     # (asked for without the matrices)
                # parts are for calls that do not fill the chip, and their results take little against the matrices
                assert parts == 1 or -(-m // tm) * -(-n // tn) <= 2 * cus


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_attention_is_covered(dim):
    for heads in (1, 2, 8, 128):
        for group in (1, 4, 7, 64):
            for seqs in (1, 3, 64, 1000):
                for each in (0, 1, 5, 300):
                    rows = seqs * each
                    if rows * heads * group >= 1 << 29:
                        continue
                    for longest in (0, 1, 500, 16384, 1 << 20):
                        tile, share, slots, tiles, work = plan(fobq.PLAN_KV4_ATTENTION, [256, dim, heads, group, seqs, rows, longest], 5)
                        # sequences may be as ragged as they like: floor(first row * group / tile) + index, and one tile more
                        assert tiles >= rows * group // tile + seqs and tile in (16, 32, 64, 128)
                        # split: room for every tile of rows, and for further parts of some
                        assert slots == 0 or (slots > tiles and longest > 1024 and seqs <= 256 and slots < 1 << 17)
                        # sums, maxima and weights of every slot, and where each sequence's slots begin
                        assert work == (4 * heads * slots * tile * (dim + 2) + 8 * 256 if slots else 0)


def test_null_contexts():
    lib, null = fobq.load_library(), ctypes.c_void_p(None)
    n = ctypes.c_int64(0)
    assert lib.fobq_fp8_quantize(null, null, 0, 1, None) == fobq.EINVAL
    assert lib.fobq_fp8_from_codes(null, null, null, null, 4, 0, None) == fobq.EINVAL
    assert lib.fobq_fp8_matmul(null, None, None, null, 0, 1, null, 0) == fobq.EINVAL
    assert lib.fobq_fp8_matmul_workspace(null, 1, 1, 1, 0, ctypes.byref(n)) == fobq.EINVAL
    assert lib.fobq_kv4_append(null, None, None, 1, null, 0, 0, null, 0, 0) == fobq.EINVAL
    assert lib.fobq_kv4_read(null, None, None, 1, null, 0, 0, null, 0, 0) == fobq.EINVAL
    assert lib.fobq_kv4_attention(null, None, None, None, null, 0) == fobq.EINVAL
    assert lib.fobq_kv4_attention_workspace(null, None, None, None, ctypes.byref(n)) == fobq.EINVAL


def test_host_tensors_are_refused():
    x = torch.zeros((4, 128))
    m = fobq.Fp8Matrix(x.to(torch.float8_e4m3fn), torch.ones((1, 4)))
    cache = fobq.Kv4Cache.empty(2, 1, 64, 16, device="cpu")
    batch = fobq.Kv4Batch(torch.zeros((1, 2), dtype=torch.int32), torch.ones(1, dtype=torch.int32))
    rows = torch.zeros((1, 1, 64), dtype=torch.bfloat16)
    for call in (lambda: fobq.fobq_fp8_quantize(1, x), lambda: fobq.fobq_fp8_from_codes(1, x.to(torch.uint8), x[:, :1], x[:, :1]),
                 lambda: fobq.fobq_fp8_matmul(1, m, m), lambda: fobq.fobq_kv4_append(1, cache, batch, rows, rows),
                 lambda: fobq.fobq_kv4_read(1, cache, batch, 1), lambda: fobq.fobq_kv4_attention(1, cache, batch, rows)):
        with pytest.raises(TypeError):
            call()
