"""Calls whose buffers share memory that one of them writes: refused on the host,
before any device work (the addresses below are never dereferenced)."""

import ctypes
import os

import pytest

from paper_2406_14898_amd import BatchDesc
from paper_2406_14898_amd import flglm as F

G = 1 << 30  # arguments a GiB apart


def _lib():
    if not os.path.exists(F.LIB_PATH):
        from paper_2406_14898_amd import build
        build.build()
    return F.load()


H, RANK, N = 256, 8, 2
A_BYTES = {F.FL_BF16: 2 * N * RANK * H, F.FL_F32: 4 * N * RANK * H}
X, Y, SAVED, DY, DX, WS, AWS = G, 2 * G, 3 * G, 4 * G, 5 * G, 20 * G, 30 * G


def _stack_call(backward, layers, grads, dtype):
    """(code, message) of a stack call with these adapters; everything else in order."""
    lib = _lib()
    h = F.fl_stack_create(F.stack_desc(2, H, 4, 1024, 32, dtype))
    b = BatchDesc([0, 64, 128], [0, 1, 2])
    ws_n = F.fl_stack_workspace_bytes(h, b, False)
    L = (F.fl_layer_params * 2)(*[F.fl_layer_params(*([16] * 12))] * 2)
    rec = F.stack_adapters(N, RANK, 1.0, b, (0, 1), layers, grads)
    n = F.fl_stack_adapter_bytes(h, b, rec)
    if backward:
        frozen = (F.fl_layer_grads * 2)(F.fl_layer_grads(), F.fl_layer_grads())
        code = lib.fl_server_stack_backward_adapters(h, ctypes.byref(b.desc), L, frozen, ctypes.byref(rec), X, SAVED, DY, DX,
                                                     0, WS, ws_n, AWS, n, None)
    else:
        code = lib.fl_server_stack_forward_adapters(h, ctypes.byref(b.desc), L, ctypes.byref(rec), X, Y, SAVED, 0, WS, ws_n,
                                                    AWS, n, None)
    F.fl_stack_destroy(h)
    return code, F.fl_last_error()


def _pair(**kw):
    return dict(dict(a=11 * G, b=12 * G), **kw)


def _grad(**kw):
    return dict(dict(a=13 * G, b=14 * G), **kw)


@pytest.mark.parametrize("dtype", [F.FL_BF16, F.FL_F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("where", [Y, SAVED, WS, AWS])
@pytest.mark.parametrize("name", ["a", "b"])
@pytest.mark.parametrize("block", [0, 1])
def test_stack_forward_refuses_adapters_in_what_it_writes(where, name, block, dtype):
    layers = [_pair(), _pair()]
    layers[block] = _pair(**{name: where + 32})
    code, why = _stack_call(False, layers, None, dtype)
    assert code == F.FL_ERR_ALIAS and f"layer {block}" in why


@pytest.mark.parametrize("where", [DX, SAVED, WS, AWS])
@pytest.mark.parametrize("name", ["a", "b"])
def test_stack_backward_refuses_adapters_in_what_it_writes(where, name):
    assert _stack_call(True, [_pair(), _pair(**{name: where})], [_grad(), _grad()], F.FL_BF16)[0] == F.FL_ERR_ALIAS


@pytest.mark.parametrize("where", [X, DY, DX, SAVED, WS, AWS])
@pytest.mark.parametrize("name", ["a", "b"])
@pytest.mark.parametrize("block", [0, 1])
def test_stack_backward_refuses_gradients_in_other_buffers(where, name, block):
    grads = [_grad(), _grad()]
    grads[block] = _grad(**{name: where + 64})
    code, why = _stack_call(True, [_pair(), _pair()], grads, F.FL_BF16)
    assert code == F.FL_ERR_ALIAS and f"layer {block}" in why


@pytest.mark.parametrize("dtype", [F.FL_BF16, F.FL_F32], ids=["bf16", "f32"])
def test_stack_backward_refuses_gradients_that_run_into_each_other(dtype):
    """Another gradient of the same or of the other block, or an adapter (its last
    bytes as well as its first); two blocks' gradients that are one array are not
    meant (they add up)."""
    end_a, end_b = 4 * N * RANK * H, 12 * N * RANK * H  # bytes of the gradients
    wide = 3 * A_BYTES[dtype]                           # of an adapter b
    for grads in ([_grad(b=13 * G), _grad()],                     # b on a
                  [_grad(), _grad(a=13 * G + 16)],                # shifted into the other block's a
                  [_grad(), _grad(a=13 * G + end_a - 16)],
                  [_grad(a=15 * G), _grad(a=14 * G)],             # a at the other block's b
                  [_grad(), _grad(b=14 * G + end_b - 16)],
                  [_grad(a=11 * G), _grad()],                     # an adapter itself
                  [_grad(), _grad(b=12 * G + wide - 16)],
                  [_grad(a=12 * G - end_a + 16), _grad()],
                  [_grad(a=11 * G + 16), _grad(a=11 * G + 16)]):
        code, why = _stack_call(True, [_pair(), _pair()], grads, dtype)
        assert code == F.FL_ERR_ALIAS and "gradient" in why, grads
