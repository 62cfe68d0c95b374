"""What the calls on few bits refuse, and where a row's token lies when lengths, pages and starts are not as they should be: the statements of
the host tests' test_places, with a length that passes the table as the contract has it (no GPU)."""
import pytest

pytest.importorskip("torch")
import paper_2509_05576_amd as fobq

LENGTHS, STARTS = [40, 3, 17, 0], [0, 2, 2, 5, 5]
TABLE = [[7, 2, 4], [1, -1, -1], [0, 9, -1], [-1, -1, -1]]


def at(row, page=16, pages=10, lengths=LENGTHS, starts=STARTS, table=TABLE, rows=8):
    width = len(table[0])
    return fobq.fobq_debug_plan(fobq.PLAN_KV4_PLACE, [page, pages, width, len(lengths), rows, row] + lengths + starts + [e for t in table for e in t], 3)


def test_places():
    assert at(0) == [0, 4, 6] and at(1) == [0, 4, 7]                    # tokens 38 and 39
    assert at(2) == [2, 0, 14] and at(3) == [2, 0, 15] and at(4) == [2, 9, 0]     # sequence 1 has no rows
    for row in (5, 7):
        assert at(row)[1] == -1                                         # behind the last sequence
    # pages that are none, rows before token 0, lengths below 0
    assert at(4, pages=9)[1] == -1 and at(0, table=[[7, 2, -4]] + TABLE[1:])[1] == -1 and at(0, table=[[7, 2, 2 ** 31 - 1]] + TABLE[1:])[1] == -1
    assert at(2, lengths=[40, 3, 2, 0])[1] == -1 and at(3, lengths=[40, 3, 2, 0]) == [2, 0, 0]
    assert at(1, lengths=[-2 ** 31, 3, 17, 0])[1] == -1
    # starts out of order or out of range
    for bad in ([0, -5, 2 ** 31 - 1, 3, -1], [9, 8, 7, 6, 5], [2 ** 31 - 1] * 5, [-2 ** 31] * 5):
        for row in range(8):
            assert at(row, starts=bad)[1] in (-1, 0, 1, 2, 4, 7, 9)


@pytest.mark.parametrize("length", [48, 49, 50, 51, 64, 1000, 1 << 30, 2 ** 31 - 1])
def test_a_length_that_passes_the_table(length):
    """Row i of n is token length - n + i of its sequence, whatever the table holds: three pages of 16, places for tokens 0 .. 47."""
    for count in (1, 2, 7):
        for row in range(count):
            token = length - count + row
            want = [0, TABLE[0][token // 16], token % 16] if token < 48 else [0, -1]
            assert at(row, lengths=[length, 3, 17, 0], starts=[0, count, count, count, count])[:len(want)] == want


@pytest.mark.parametrize("rows,cols,ok", [((1 << 26) - 4, 0, True), ((1 << 26) - 3, 0, False), ((1 << 29) - 1, 0, False), ((1 << 26) - 4, 512, True),
                                          ((1 << 26) - 4, 513, False)])
def test_rows_of_no_columns(rows, cols, ok):
    """A product over no columns writes zeros: as many rows as its launch has workgroups for."""
    got = fobq.fobq_debug_plan(fobq.PLAN_FP8_CHECK, [rows, cols, -(-cols // 16) * 16, rows, 1, 0, 0x7000000000, 0x7000000000], 1)
    assert got == [fobq.OK if ok else fobq.EINVAL]


@pytest.mark.parametrize("change", [dict(page=0), dict(page=8), dict(page=24), dict(page=8192), dict(page=(1 << 62) + 1), dict(page=2 ** 63 - 1), dict(page=-16),
                                    dict(pages=0), dict(pages=1 << 31), dict(rows=-1), dict(rows=1 << 40), dict(row=-1), dict(row=1 << 33)])
def test_places_are_asked_of_caches_that_there_can_be(change):
    with pytest.raises(fobq.FobqError):
        at(**{"row": 0, **change})
