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


# ---------------------------------------------------------------------------
# The head with the preference loss
# ---------------------------------------------------------------------------

VOCAB, PAIRS = 1000, dict(cu_seqlens=[0, 5, 14, 21, 22], client_seq_ptr=[0, 2, 4])
HEAD = dict(h=G, w=2 * G, ln_g=3 * G, ln_b=4 * G, ref=5 * G, logp=6 * G, loss=7 * G, total=8 * G, ws=9 * G, pws=10 * G,
            dh=11 * G, dw=12 * G, dln_g=13 * G, dln_b=14 * G)
T = 22
HEAD_BYTES = dict(h=2 * T * H, w=2 * VOCAB * H, ln_g=2 * H, ln_b=2 * H, ref=16, dh=2 * T * H, dw=4 * VOCAB * H, dln_g=4 * H,
                  dln_b=4 * H)


def _head_call(backward, **at):
    lib = _lib()
    p = dict(HEAD, **at)
    h = F.fl_client_create(VOCAB, H, F.FL_BF16)
    b, d = BatchDesc(**PAIRS), F.fl_preference_desc(VOCAB, F.FL_BF16, 0.1, 0.0)
    ws_n, pn = F.fl_client_workspace_bytes(h, T), F.fl_preference_workspace_bytes(d, b)
    if backward:
        code = lib.fl_lm_head_preference_backward(h, ctypes.byref(d), ctypes.byref(b.desc), p["h"], p["ln_g"], p["w"],
                                                  ctypes.c_float(1.0), p["dh"], p["dln_g"], p["dln_b"], p["dw"], p["ws"], ws_n,
                                                  p["pws"], pn, None)
    else:
        code = lib.fl_lm_head_preference_forward(h, ctypes.byref(d), ctypes.byref(b.desc), p["h"], p["ln_g"], p["ln_b"], p["w"],
                                                 (ctypes.c_int32 * T)(*[5] * T), p["ref"], p["logp"], p["loss"], p["total"],
                                                 p["ws"], ws_n, p["pws"], pn, None)
    F.fl_client_destroy(h)
    return code


@pytest.mark.parametrize("own", ["logp", "loss", "total", "ws", "pws"])
@pytest.mark.parametrize("other", ["h", "w", "ln_g", "ln_b", "ref"])
def test_head_preference_forward_refuses_outputs_in_what_it_reads(own, other):
    assert _head_call(False, **{own: HEAD[other]}) == F.FL_ERR_ALIAS
    end = HEAD[other] + HEAD_BYTES[other] - 16  # the last bytes
    assert _head_call(False, **{own: end}) == F.FL_ERR_ALIAS


@pytest.mark.parametrize("own,other", [("logp", "loss"), ("logp", "total"), ("loss", "total"), ("ws", "pws"), ("logp", "ws"),
                                       ("loss", "ws"), ("total", "ws"), ("logp", "pws"), ("total", "pws")])
def test_head_preference_forward_refuses_outputs_in_each_other(own, other):
    assert _head_call(False, **{own: HEAD[other]}) == F.FL_ERR_ALIAS


@pytest.mark.parametrize("own", ["ws", "pws", "dh", "dw", "dln_g", "dln_b"])
@pytest.mark.parametrize("other", ["h", "w", "ln_g", "ws", "pws", "dh", "dw", "dln_g", "dln_b"])
def test_head_preference_backward_refuses_gradients_in_other_memory(own, other):
    if own == other:
        return
    assert _head_call(True, **{own: HEAD[other]}) == F.FL_ERR_ALIAS
    if other in HEAD_BYTES:
        assert _head_call(True, **{own: HEAD[other] + HEAD_BYTES[other] - 16}) == F.FL_ERR_ALIAS
