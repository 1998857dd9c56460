"""Refusals of the adapter, preference-loss and gradient-norm entry points:
every malformed call gets its error code on the host, before any device work
(the addresses below are never dereferenced)."""

import ctypes
import math
import os

import pytest

from paper_2406_14898_amd import BatchDesc, FlglmError
from paper_2406_14898_amd import flglm as F

G = 1 << 30  # arguments a GiB apart


def _lib():
    if not os.path.exists(F.LIB_PATH):
        from paper_2406_14898_amd import build
        build.build()
    return F.load()


# ---------------------------------------------------------------------------
# Adapters
# ---------------------------------------------------------------------------

def _adesc(**kw):
    d = dict(num_adapters=4, rank=16, in_features=64, out_features=96, scale=2.0, dtype=F.FL_BF16)
    d.update(kw)
    return F.fl_adapter_desc(**d)


BATCH = dict(cu_seqlens=[0, 5, 14, 21], client_seq_ptr=[0, 2, 3])


@pytest.mark.parametrize("kw,code", [
    (dict(num_adapters=0), F.FL_ERR_SHAPE), (dict(num_adapters=(1 << 16) + 1), F.FL_ERR_SHAPE),
    (dict(rank=0), F.FL_ERR_SHAPE), (dict(rank=12), F.FL_ERR_SHAPE), (dict(rank=72), F.FL_ERR_SHAPE),
    (dict(in_features=0), F.FL_ERR_SHAPE), (dict(in_features=100), F.FL_ERR_SHAPE),
    (dict(out_features=12), F.FL_ERR_SHAPE), (dict(out_features=65544), F.FL_ERR_SHAPE),
    (dict(dtype=2), F.FL_ERR_SHAPE), (dict(scale=math.inf), F.FL_ERR_ARG), (dict(scale=math.nan), F.FL_ERR_ARG),
])
def test_adapter_descriptor(kw, code):
    _lib()
    with pytest.raises(FlglmError) as e:
        F.fl_adapter_workspace_bytes(_adesc(**kw), BatchDesc(**BATCH))
    assert e.value.code == code


def test_adapter_batch_is_checked():
    _lib()
    with pytest.raises(FlglmError) as e:
        F.fl_adapter_workspace_bytes(_adesc(), BatchDesc([0, 3, 3], [0, 2]))
    assert e.value.code == F.FL_ERR_SEQLENS


def _afwd(desc=None, batch=None, ca=(0, 1), x=G, ldx=64, a=2 * G, b=3 * G, base=4 * G, ldb=96, y=5 * G, ldy=96,
          v=6 * G, ws=7 * G, ws_bytes=None):
    desc, batch = desc or _adesc(), batch or BatchDesc(**BATCH)
    n = F.fl_adapter_workspace_bytes(desc, batch) if ws_bytes is None else ws_bytes
    p = None if ca is None else (ctypes.c_int32 * len(ca))(*ca)
    return _lib().fl_adapter_forward(ctypes.byref(desc), ctypes.byref(batch.desc), p, x, ldx, a, b, base, ldb, y, ldy, v,
                                     ws, n, None)


@pytest.mark.parametrize("kw,code", [
    (dict(ca=None), F.FL_ERR_NULL), (dict(ca=(0, 4)), F.FL_ERR_ARG), (dict(ca=(-2, 0)), F.FL_ERR_ARG),
    (dict(x=None), F.FL_ERR_NULL), (dict(a=None), F.FL_ERR_NULL), (dict(b=None), F.FL_ERR_NULL),
    (dict(y=None), F.FL_ERR_NULL), (dict(v=None), F.FL_ERR_NULL), (dict(ws=None), F.FL_ERR_NULL),
    (dict(x=G + 8), F.FL_ERR_ALIGN), (dict(base=4 * G + 2), F.FL_ERR_ALIGN), (dict(v=6 * G + 4), F.FL_ERR_ALIGN),
    (dict(ws=7 * G + 8), F.FL_ERR_ALIGN), (dict(ldx=56), F.FL_ERR_SHAPE), (dict(ldx=68), F.FL_ERR_SHAPE),
    (dict(ldy=88), F.FL_ERR_SHAPE), (dict(ldb=100), F.FL_ERR_SHAPE), (dict(ws_bytes=16), F.FL_ERR_WORKSPACE),
    (dict(y=G), F.FL_ERR_ALIAS), (dict(y=4 * G + 16), F.FL_ERR_ALIAS), (dict(y=4 * G, ldy=104), F.FL_ERR_ALIAS),
    (dict(v=5 * G), F.FL_ERR_ALIAS), (dict(v=2 * G), F.FL_ERR_ALIAS), (dict(ws=3 * G), F.FL_ERR_ALIAS),
    (dict(ws=6 * G), F.FL_ERR_ALIAS),
])
def test_adapter_forward_refusals(kw, code):
    assert _afwd(**kw) == code
    assert F.fl_last_error()


def _abwd(desc=None, batch=None, ca=(0, 1), dy=G, ldy=96, x=2 * G, ldx=64, a=3 * G, b=4 * G, v=5 * G, dres=6 * G,
          ldr=64, dx=7 * G, lddx=64, da=8 * G, db=9 * G, ws=10 * G, ws_bytes=None):
    desc, batch = desc or _adesc(), batch or BatchDesc(**BATCH)
    n = F.fl_adapter_workspace_bytes(desc, batch) if ws_bytes is None else ws_bytes
    p = None if ca is None else (ctypes.c_int32 * len(ca))(*ca)
    return _lib().fl_adapter_backward(ctypes.byref(desc), ctypes.byref(batch.desc), p, dy, ldy, x, ldx, a, b, v, dres,
                                      ldr, dx, lddx, da, db, ws, n, None)


@pytest.mark.parametrize("kw,code", [
    (dict(dy=None), F.FL_ERR_NULL), (dict(x=None), F.FL_ERR_NULL), (dict(v=None), F.FL_ERR_NULL),
    (dict(da=None), F.FL_ERR_NULL), (dict(db=None), F.FL_ERR_NULL), (dict(dx=None), F.FL_ERR_NULL),
    (dict(ca=(0, 9)), F.FL_ERR_ARG), (dict(da=8 * G + 4), F.FL_ERR_ALIGN), (dict(lddx=60), F.FL_ERR_SHAPE),
    (dict(ws_bytes=64), F.FL_ERR_WORKSPACE), (dict(dx=2 * G), F.FL_ERR_ALIAS), (dict(dx=6 * G + 16), F.FL_ERR_ALIAS),
    (dict(da=9 * G), F.FL_ERR_ALIAS), (dict(db=4 * G), F.FL_ERR_ALIAS), (dict(ws=5 * G), F.FL_ERR_ALIAS),
    (dict(ws=7 * G), F.FL_ERR_ALIAS),
])
def test_adapter_backward_refusals(kw, code):
    assert _abwd(**kw) == code


def test_columns_of_one_buffer_do_not_overlap():
    """x, base and y as columns of one buffer of 256-element rows: apart they pass
    the checks (the call is refused for the workspace only), one column into
    each other they do not."""
    at = lambda col: G + 2 * col  # noqa: E731
    ok = dict(x=at(0), ldx=256, base=at(64), ldb=256, y=at(160), ldy=256)
    assert _afwd(**ok, ws=2 * G) == F.FL_ERR_ALIAS                # a's place: everything else passed
    assert "workspace" in F.fl_last_error()
    for y in (at(56), at(152), at(168)):                          # into x, into base, over the row's end into x
        assert _afwd(**dict(ok, y=y), ws=2 * G) == F.FL_ERR_ALIAS
        assert "workspace" not in F.fl_last_error()


def test_adapter_workspace_does_not_grow_with_the_rank_of_rows_alone():
    """The partial sums of dA and dB are bounded by the slabs, not by the clients:
    256 clients of one row each ask for less than two slots' gradients a slab."""
    _lib()
    d = _adesc(num_adapters=256, in_features=4096, out_features=12288)
    many = BatchDesc(list(range(257)), list(range(257)))
    assert F.fl_adapter_workspace_bytes(d, many) < 200 << 20


def test_stack_adapter_refusals():
    lib = _lib()
    h = F.fl_stack_create(F.stack_desc(2, 256, 4, 1024, 32, F.FL_BF16))
    b = BatchDesc([0, 64, 128], [0, 1, 2])
    ws_n = F.fl_stack_workspace_bytes(h, b, False)
    L = (F.fl_layer_params * 2)(*[F.fl_layer_params(*([16] * 12))] * 2)
    ok = [dict(a=11 * G, b=12 * G)] * 2
    gr = [dict(a=13 * G, b=14 * G)] * 2

    def fwd(rec, aws=30 * G, n=None):
        n = F.fl_stack_adapter_bytes(h, b, rec) if n is None else n
        return lib.fl_server_stack_forward_adapters(h, ctypes.byref(b.desc), L, ctypes.byref(rec), G, 2 * G, None, 0,
                                                    20 * G, ws_n, aws, n, None)

    def rec(layers=ok, grads=None, ca=(0, 1), n=2, rank=8, scale=1.0):
        return F.stack_adapters(n, rank, scale, b, ca, layers, grads)

    assert fwd(rec(ca=(0, 2))) == F.FL_ERR_ARG
    assert fwd(rec(layers=[dict(a=None, b=12 * G), ok[0]])) == F.FL_ERR_NULL
    assert fwd(rec(layers=[dict(a=11 * G + 8, b=12 * G), ok[0]])) == F.FL_ERR_ALIGN
    assert fwd(rec(), n=16) == F.FL_ERR_WORKSPACE
    assert fwd(rec(), aws=None) == F.FL_ERR_NULL
    assert fwd(rec(), aws=20 * G) == F.FL_ERR_ALIAS
    assert fwd(rec(), aws=11 * G) == F.FL_ERR_ALIAS
    assert lib.fl_server_stack_forward_adapters(h, ctypes.byref(b.desc), L, None, G, 2 * G, None, 0, 20 * G, ws_n,
                                                30 * G, 1 << 20, None) == F.FL_ERR_NULL
    with pytest.raises(FlglmError) as e:
        F.fl_stack_adapter_bytes(h, b, rec(rank=7))
    assert e.value.code == F.FL_ERR_SHAPE
    with pytest.raises(FlglmError) as e:
        rec(ca=(0,))
    assert e.value.code == F.FL_ERR_ARG
    gl = (F.fl_layer_grads * 2)(F.fl_layer_grads(), F.fl_layer_grads())  # frozen weights

    def bwd(r):
        n = F.fl_stack_adapter_bytes(h, b, r)
        return lib.fl_server_stack_backward_adapters(h, ctypes.byref(b.desc), L, gl, ctypes.byref(r), G, 3 * G, 4 * G,
                                                     5 * G, 0, 20 * G, ws_n, 30 * G, n, None)

    assert bwd(rec()) == F.FL_ERR_NULL                                                  # no gradients
    assert bwd(rec(grads=[dict(a=13 * G, b=13 * G), gr[0]])) == F.FL_ERR_ALIAS
    assert bwd(rec(grads=[dict(a=13 * G, b=None), gr[0]])) == F.FL_ERR_NULL
    F.fl_stack_destroy(h)


# ---------------------------------------------------------------------------
# Preference loss
# ---------------------------------------------------------------------------

PAIRS = dict(cu_seqlens=[0, 5, 14, 21, 22], client_seq_ptr=[0, 2, 4])


def _pdesc(**kw):
    d = dict(vocab=1000, dtype=F.FL_BF16, beta=0.1, label_smoothing=0.0)
    d.update(kw)
    return F.fl_preference_desc(**d)


@pytest.mark.parametrize("kw,code", [
    (dict(vocab=1001), F.FL_ERR_SHAPE), (dict(vocab=0), F.FL_ERR_SHAPE), (dict(vocab=(1 << 24) + 8), F.FL_ERR_SHAPE),
    (dict(dtype=3), F.FL_ERR_SHAPE), (dict(beta=0.0), F.FL_ERR_ARG), (dict(beta=math.nan), F.FL_ERR_ARG),
    (dict(beta=math.inf), F.FL_ERR_ARG), (dict(label_smoothing=-0.1), F.FL_ERR_ARG),
    (dict(label_smoothing=0.6), F.FL_ERR_ARG), (dict(label_smoothing=math.nan), F.FL_ERR_ARG),
])
def test_preference_descriptor(kw, code):
    _lib()
    with pytest.raises(FlglmError) as e:
        F.fl_preference_workspace_bytes(_pdesc(**kw), BatchDesc(**PAIRS))
    assert e.value.code == code


@pytest.mark.parametrize("cu,csp", [([0, 5], [0, 1]), ([0, 5, 9, 12, 14], [0, 1, 4]), ([0, 5, 9, 12], [0, 3])])
def test_preference_needs_whole_pairs_of_every_client(cu, csp):
    _lib()
    with pytest.raises(FlglmError) as e:
        F.fl_preference_workspace_bytes(_pdesc(), BatchDesc(cu, csp))
    assert e.value.code == F.FL_ERR_CLIENTS


def _pfwd(logits=G, ld=1000, labels=2 * G, ref=3 * G, logp=4 * G, loss=5 * G, total=6 * G, ws=7 * G, n=None, desc=None):
    desc, b = desc or _pdesc(), BatchDesc(**PAIRS)
    n = F.fl_preference_workspace_bytes(desc, b) if n is None else n
    return _lib().fl_preference_forward(ctypes.byref(desc), ctypes.byref(b.desc), logits, ld, labels, ref, logp, loss,
                                        total, ws, n, None)


@pytest.mark.parametrize("kw,code", [
    (dict(logits=None), F.FL_ERR_NULL), (dict(labels=None), F.FL_ERR_NULL), (dict(logp=None), F.FL_ERR_NULL),
    (dict(loss=None), F.FL_ERR_NULL), (dict(total=None), F.FL_ERR_NULL), (dict(ws=None), F.FL_ERR_NULL),
    (dict(logits=G + 8), F.FL_ERR_ALIGN), (dict(labels=2 * G + 2), F.FL_ERR_ALIGN), (dict(ws=7 * G + 4), F.FL_ERR_ALIGN),
    (dict(ld=992), F.FL_ERR_SHAPE), (dict(ld=1004), F.FL_ERR_SHAPE), (dict(n=8), F.FL_ERR_WORKSPACE),
    (dict(logp=5 * G), F.FL_ERR_ALIAS), (dict(loss=3 * G + 4), F.FL_ERR_ALIAS), (dict(total=7 * G + 4), F.FL_ERR_ALIAS),
    (dict(ws=G), F.FL_ERR_ALIAS), (dict(ws=2 * G), F.FL_ERR_ALIAS), (dict(logp=G + 64), F.FL_ERR_ALIAS),
])
def test_preference_forward_refusals(kw, code):
    assert _pfwd(**kw) == code


def _pbwd(logits=G, ld=1000, labels=2 * G, scale=1.0, dl=3 * G, ldd=1000, width=1000, ws=7 * G, n=None):
    desc, b = _pdesc(), BatchDesc(**PAIRS)
    n = F.fl_preference_workspace_bytes(desc, b) if n is None else n
    return _lib().fl_preference_backward(ctypes.byref(desc), ctypes.byref(b.desc), logits, ld, labels,
                                         ctypes.c_float(scale), dl, ldd, width, ws, n, None)


@pytest.mark.parametrize("kw,code", [
    (dict(dl=None), F.FL_ERR_NULL), (dict(dl=3 * G + 4), F.FL_ERR_ALIGN), (dict(ldd=992), F.FL_ERR_SHAPE),
    (dict(ldd=1004), F.FL_ERR_SHAPE), (dict(width=992), F.FL_ERR_SHAPE), (dict(width=1008), F.FL_ERR_SHAPE),
    (dict(ldd=1024, width=1004), F.FL_ERR_SHAPE), (dict(scale=math.inf), F.FL_ERR_ARG),
    (dict(scale=math.nan), F.FL_ERR_ARG), (dict(n=8), F.FL_ERR_WORKSPACE), (dict(dl=G + 16), F.FL_ERR_ALIAS),
    (dict(dl=G, ldd=1024), F.FL_ERR_ALIAS), (dict(dl=2 * G), F.FL_ERR_ALIAS), (dict(dl=7 * G), F.FL_ERR_ALIAS),
    (dict(ws=G), F.FL_ERR_ALIAS),
])
def test_preference_backward_refusals(kw, code):
    assert _pbwd(**kw) == code


def test_head_preference_refusals():
    lib = _lib()
    h = F.fl_client_create(1000, 256, F.FL_BF16)
    b = BatchDesc(**PAIRS)
    T = b.total_tokens
    ws_n, d = F.fl_client_workspace_bytes(h, T), _pdesc()
    pn = F.fl_preference_workspace_bytes(d, b)

    def fwd(desc=d, labels=(5,) * T, ws=7 * G, pws=8 * G, logp=4 * G, n=ws_n, m=pn):
        lab = (ctypes.c_int32 * T)(*labels)
        return lib.fl_lm_head_preference_forward(h, ctypes.byref(desc), ctypes.byref(b.desc), G, None, None, 2 * G, lab,
                                                 None, logp, 5 * G, 6 * G, ws, n, pws, m, None)

    assert fwd(labels=(5,) * (T - 1) + (1000,)) == F.FL_ERR_ARG
    assert fwd(desc=_pdesc(vocab=1008)) == F.FL_ERR_SHAPE
    assert fwd(desc=_pdesc(dtype=F.FL_F32)) == F.FL_ERR_SHAPE
    assert fwd(n=ws_n - 1) == F.FL_ERR_WORKSPACE
    assert fwd(m=pn - 1) == F.FL_ERR_WORKSPACE
    assert fwd(pws=7 * G) == F.FL_ERR_ALIAS
    assert fwd(logp=7 * G + 64) == F.FL_ERR_ALIAS

    def bwd(dh=3 * G, scale=1.0, dw=None, pws=8 * G):
        return lib.fl_lm_head_preference_backward(h, ctypes.byref(d), ctypes.byref(b.desc), G, None, 2 * G,
                                                  ctypes.c_float(scale), dh, None, None, dw, 7 * G, ws_n, pws, pn, None)

    assert bwd(dh=None) == F.FL_ERR_NULL
    assert bwd(dh=G) == F.FL_ERR_ALIAS
    assert bwd(scale=math.nan) == F.FL_ERR_ARG
    assert bwd(pws=3 * G) == F.FL_ERR_ALIAS
    assert bwd(dw=7 * G) == F.FL_ERR_ALIAS
    with pytest.raises(FlglmError) as e:
        F.fl_lm_head_preference_forward(h, d, b, G, 2 * G, [1] * (T - 1), None, 4 * G, 5 * G, 6 * G, None, None)
    assert e.value.code == F.FL_ERR_ARG
    F.fl_client_destroy(h)


# ---------------------------------------------------------------------------
# Gradient norm
# ---------------------------------------------------------------------------

def _norm(grads=(G, 2 * G), sizes=(1000, 17), dtype=F.FL_F32, max_norm=1.0, out=3 * G, ws=4 * G, n=1 << 20):
    p = (ctypes.c_void_p * len(grads))(*grads)
    z = (ctypes.c_int64 * len(sizes))(*sizes)
    return _lib().fl_grad_norm(dtype, len(sizes), p, z, max_norm, out, ws, n, None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), F.FL_ERR_ARG), (dict(sizes=()), F.FL_ERR_ARG), (dict(sizes=(5, -1)), F.FL_ERR_ARG),
    (dict(sizes=(5, (1 << 40) + 1)), F.FL_ERR_ARG), (dict(max_norm=-1.0), F.FL_ERR_ARG),
    (dict(max_norm=math.nan), F.FL_ERR_ARG), (dict(grads=(G, None)), F.FL_ERR_NULL), (dict(out=None), F.FL_ERR_NULL),
    (dict(ws=None), F.FL_ERR_NULL), (dict(grads=(G, 2 * G + 4)), F.FL_ERR_ALIGN), (dict(out=3 * G + 4), F.FL_ERR_ALIGN),
    (dict(n=4), F.FL_ERR_WORKSPACE), (dict(out=G + 8), F.FL_ERR_ALIAS), (dict(ws=G + 16), F.FL_ERR_ALIAS),
    (dict(out=4 * G), F.FL_ERR_ALIAS),
])
def test_grad_norm_refusals(kw, code):
    assert _norm(**kw) == code


def _clip(grads=(G, 2 * G), out=(3 * G, 4 * G), sizes=(1000, 17), coef=5 * G, dtype=F.FL_F32):
    p, q = (ctypes.c_void_p * len(grads))(*grads), (ctypes.c_void_p * len(out))(*out)
    z = (ctypes.c_int64 * len(sizes))(*sizes)
    return _lib().fl_clip_grads(dtype, len(sizes), p, q, z, coef, None)


@pytest.mark.parametrize("kw,code", [
    (dict(out=(3 * G, None)), F.FL_ERR_NULL), (dict(coef=None), F.FL_ERR_NULL), (dict(out=(3 * G, 4 * G + 8)), F.FL_ERR_ALIGN),
    (dict(out=(3 * G, 3 * G)), F.FL_ERR_ALIAS),          # two outputs in one place
    (dict(grads=(G, G), out=(G, G)), F.FL_ERR_ALIAS),    # one tensor twice, in place: it would be scaled twice
    (dict(out=(G + 16, 4 * G)), F.FL_ERR_ALIAS),         # over its own gradient, shifted
    (dict(out=(2 * G, 4 * G)), F.FL_ERR_ALIAS),          # over another tensor's gradient
    (dict(grads=(G, 2 * G), out=(2 * G, G), sizes=(8, 8)), F.FL_ERR_ALIAS),  # swapped
    (dict(coef=3 * G + 8), F.FL_ERR_ALIAS), (dict(dtype=7), F.FL_ERR_ARG),
])
def test_clip_refusals(kw, code):
    assert _clip(**kw) == code


def test_host_tensors_and_wrong_tensors_are_refused():
    """The classes refuse host tensors, wrong shapes and types before the library."""
    import torch
    from paper_2406_14898_amd import ClientAdapters, GradNorm, PreferenceLoss
    _lib()
    op, b = ClientAdapters(2, 8, 16, 24), BatchDesc([0, 4], [0, 1])
    t = lambda *s, d=torch.bfloat16: torch.zeros(s, dtype=d)  # noqa: E731
    with pytest.raises(FlglmError):
        op.forward(b, [0], t(4, 16), t(2, 8, 16), t(2, 24, 8), None, t(4, 24), t(4, 8, d=torch.float32), t(8))
    with pytest.raises(FlglmError):
        GradNorm([t(5, d=torch.float32)])
    with pytest.raises(FlglmError):
        GradNorm([])
    with pytest.raises(FlglmError):
        PreferenceLoss(64).forward(BatchDesc([0, 2, 4], [0, 2]), t(4, 56), t(4, d=torch.int32), None, None, None, None,
                                   t(8))
