"""Host side of the operators' binding, without a GPU: what a record keeps of
the program's own arrays, and which integers it takes."""

import os

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


@pytest.mark.parametrize("wrong", [2 ** 32 + 3, -2 ** 32 + 3, 3.5], ids=str)
def test_preference_labels_that_int32_cannot_hold_are_refused(wrong):
    """None of them is the label 3 that a cast makes of it (refused before the
    library is called: the handle and addresses below are of nothing)."""
    batch, desc = BatchDesc([0, 2, 4], [0, 2]), F.fl_preference_desc(1000, F.FL_BF16, 0.1, 0.0)
    for labels in (np.array([1, wrong, 2, -100]), [1, wrong, 2, -100]):
        with pytest.raises(F.FlglmError) as e:
            F.fl_lm_head_preference_forward(0, desc, batch, G, G, labels, None, G, G, G, None, None)
        assert e.value.code == F.FL_ERR_ARG and "labels" in str(e.value)


def test_preference_labels_of_every_type_reach_the_library():
    """Labels of other types, or read-only, pass the binding; the library refuses the
    call for its NULL handle."""
    batch, desc = BatchDesc([0, 2, 4], [0, 2]), F.fl_preference_desc(1000, F.FL_BF16, 0.1, 0.0)
    if not os.path.exists(F.LIB_PATH):
        from paper_2406_14898_amd import build
        build.build()
    fixed = np.array([1, 3, 2, -100], np.int32)
    fixed.setflags(write=False)
    for labels in ([1, 3, 2, -100], fixed, np.array([1, 3, 2, -100]), np.array([1.0, 3.0, 2.0, -100.0])):
        room = np.zeros(8, np.uint8)

        class Room:  # an address and its size
            numel, element_size = (lambda self: 8), (lambda self: 1)
            is_cuda, data_ptr = True, (lambda self: room.ctypes.data)
        with pytest.raises(F.FlglmError) as e:
            F.fl_lm_head_preference_forward(None, desc, batch, G, G, labels, None, G, G, G, Room(), Room())
        assert e.value.code == F.FL_ERR_NULL


@pytest.mark.parametrize("sizes,runs", [
    ([(16, 16), (8,), (24,)], [(0, 288)]), ([(5,), (8,), (3, 3), (16,)], [(0, 5), (8, 17), (32, 16)]),
    ([(0,), (7,), (0, 4), (1,)], [(0, 7), (8, 1)]), ([], []), ([(0,)], []),
])
def test_an_arena_knows_its_values_from_its_padding(sizes, runs):
    """What clipping scales: every tensor's elements, none between them."""
    from paper_2406_14898_amd import ParamArena
    arena = ParamArena([(str(i), s) for i, s in enumerate(sizes)], bf16_copy=False, device="cpu")
    assert arena._runs() == runs
    for a, n in arena._runs():
        arena.grad[a:a + n] = 1
    assert all((t == 1).all() for t in arena.grad_views().values())
    assert int(arena.grad.sum()) == sum(t.numel() for t in arena.grad_views().values())
