"""Host side of the operators' binding, without a GPU: what a record keeps of
the program's own arrays, and which integers it takes."""

import numpy as np

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
