"""Appending with lists that contradict each other or the call's sizes: reported, and nobody else's slots are written."""
import pytest
import torch

from paper_2607_28144_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16
PAGE, PAGES = 16, 12


def append(rows, lengths, starts, table, width=1):
    kc, vc = (torch.zeros(PAGES, PAGE, width, 64, dtype=rows.dtype, device=DEV) for _ in range(2))
    lists = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in (table, lengths, starts))
    B.regenvc_paged_append(rows, rows, kc, vc, *lists)
    return kc, vc


# Two sequences of 40 and 50 tokens on pages 0-2 and 3-6; the entries behind a sequence's last page name pages 7 and 8, which
# are other streams'.
TABLE = [[0, 1, 2, 7, 7], [3, 4, 5, 6, 8]]


@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("rows,lengths,starts", [
    (2, [40, 50], [0, 2, 1]),         # descending: row 1 is neither's
    (3, [40, 48], [0, 3, 2]),
    (8, [40, 50], [0, 5, 3]),
    (2, [40, 50], [0, 1, 900]),       # starts past the call's rows
    (2, [40, 50], [0, 2, 900]),       # ... of a sequence that has none of them
    (2, [40, 50], [-3, 1, 2]),
    (4, [40, 50], [2, 1, 4]),
    (2, [40, 1000], [0, 2, 2]),       # more tokens than the table holds, with no new ones among them
    (2, [40, -1], [0, 2, 2]),
    (70, [40, 50], [0, 60, 70]),      # fewer tokens than new ones
])
def test_contradicting_lists_are_reported(dtype, rows, lengths, starts):
    for off in (0, 1):                # rows without 16-byte alignment take the other kernel
        room = torch.ones(rows * 64 + 1, dtype=dtype, device=DEV)
        kc, vc = append(room[off:off + rows * 64].view(rows, 1, 64), lengths, starts, TABLE)
        assert B.regenvc_device_status() == B.ERR_RANGE
        for c in (kc, vc):
            assert (c[7:] == 0).all()                                # pages of nobody in the call
            for s, last in enumerate(lengths):
                slots = c[torch.tensor(TABLE[s][:4 - (s == 0)], device=DEV)].flatten(0, 1)
                assert (slots[max(0, min(last, 64)):] == 0).all()    # slots behind a sequence's length
    kc, vc = append(torch.ones(2, 1, 64, dtype=dtype, device=DEV), [40, 50], [0, 1, 2], TABLE)
    assert B.regenvc_device_status() == B.OK                         # and the next call is normal again
    assert kc.sum() == vc.sum() == 128 and (kc[2, 7] == 1).all() and (kc[6, 1] == 1).all()


@pytest.mark.parametrize("at", [0, 31, 32, 255, 256, 700, 4095])
def test_a_contradiction_of_any_of_many_sequences_is_reported(at):
    seqs = 4096
    starts, lengths = [min(i, 3) for i in range(seqs + 1)], [5] * seqs
    table = [[i % PAGES] for i in range(seqs)]
    rows = torch.ones(3, 1, 64, dtype=BF, device=DEV)
    append(rows, lengths, starts, table)
    assert B.regenvc_device_status() == B.OK
    lengths[at] = 17
    append(rows, lengths, starts, table)
    assert B.regenvc_device_status() == B.ERR_RANGE


def test_ordinary_lists_are_not_reported():
    """Empty sequences, starts behind the first row, rows behind the last sequence, a full table."""
    rows = torch.ones(9, 1, 64, dtype=BF, device=DEV)
    for lengths, starts in (([40, 80], [2, 2, 7]), ([0, 5], [0, 0, 5]), ([1, 0], [8, 9, 9]), ([80, 80], [0, 9, 9]), ([0, 0], [0, 0, 0])):
        kc, vc = append(rows, lengths, starts, [[0, 1, 2, 3, 4], [5, 6, 7, 8, 9]])
        assert B.regenvc_device_status() == B.OK
        assert (kc != 0).any(-1).sum() == (vc != 0).any(-1).sum() == starts[-1] - starts[0]
