"""Host side of the operators' binding, without a GPU: what a record keeps of
the program's own arrays, and which integers it takes."""

import numpy as np
import pytest

from paper_2406_14898_amd import BatchDesc
from paper_2406_14898_amd import flglm as F

G = 1 << 30  # addresses that nothing reads
BLOCKS = [dict(a=G, b=2 * G)]


def _slots(record, n):
    return [record.client_adapter[i] for i in range(n)]


def test_a_stack_record_keeps_its_own_slots():
    """A program that refills its slot array for the next batch leaves the record of
    this one as it was, whatever the array's type."""
    batch = BatchDesc([0, 4, 9], [0, 1, 2])
    for kind in (np.int32, np.int64):
        slots = np.array([0, -1], kind)
        record = F.stack_adapters(2, 8, 1.0, batch, slots, BLOCKS)
        slots[:] = [1, 0]
        assert _slots(record, 2) == [0, -1], kind
    slots = [0, -1]
    record = F.stack_adapters(2, 8, 1.0, batch, slots, BLOCKS)
    slots[:] = [1, 0]
    assert _slots(record, 2) == [0, -1]


NOT_INT32 = [np.array([2 ** 32, 1]), np.array([0, -2 ** 32 - 1]), np.array([0.9, 1.7]), np.array([0.0, np.nan]),
             np.array([1, 2 ** 31], np.uint32), [2 ** 32, 1], [0.9, 1], (0, 1.5), [np.float32(0.5), 1]]


@pytest.mark.parametrize("slots", NOT_INT32, ids=str)
def test_slots_that_int32_cannot_hold_are_refused(slots):
    batch = BatchDesc([0, 4, 9], [0, 1, 2])
    with pytest.raises(F.FlglmError) as e:
        F.stack_adapters(2, 8, 1.0, batch, slots, BLOCKS)
    assert e.value.code == F.FL_ERR_ARG
    with pytest.raises(F.FlglmError):
        F._client_adapter(slots, batch)


@pytest.mark.parametrize("slots", [[1, -1], (1, -1), np.array([1, -1], np.int8), np.array([1, 7, -1, 7], np.int64)[::2],
                                   np.array([1.0, -1.0]), [1.0, -1], [np.int64(1), np.int32(-1)],
                                   np.array([1, -1], ">i4")], ids=str)
def test_slots_of_every_type_that_holds_them(slots):
    batch = BatchDesc([0, 4, 9], [0, 1, 2])
    assert _slots(F.stack_adapters(2, 8, 1.0, batch, slots, BLOCKS), 2) == [1, -1]
    arr, p = F._client_adapter(slots, batch)
    assert list(p) == [1, -1]
