"""Low-rank adapters against a plain float64 computation, element by element.

Bounds (u = 2^-23, one step of an fp32 addition on the matrix cores; U = half a
step of the output's type, 2^-8 for bf16, 2^-24 for fp32): a sum of n products
is off by at most (n + 8) u times the sum of their magnitudes; a factor held in
two bf16 parts is off by 2^-16 of its size, in three parts or in fp32 by 2^-24.
"""

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
from paper_2406_14898_amd import BatchDesc, ClientAdapters, FlglmError  # noqa: E402

u = 2.0 ** -23
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
HELD = {"bf16": 2.0 ** -16, "f32": 2.0 ** -24}   # v under a result of the type


def _batch(lens_of_clients):
    cu, csp = [0], [0]
    for lens in lens_of_clients:
        for n in lens:
            cu.append(cu[-1] + n)
        csp.append(len(cu) - 1)
    return BatchDesc(cu, csp), [cu[i] for i in csp]


def _wide(t, extra, seed):
    """t in the left columns of a wider random buffer."""
    if not extra:
        return t
    g = torch.Generator().manual_seed(seed)
    buf = torch.randn((t.shape[0], t.shape[1] + extra), generator=g).to(t.dtype).to(t.device)
    buf[:, :t.shape[1]] = t
    return buf[:, :t.shape[1]]


def _inputs(T, n, r, inn, out, dt, seed, extra=0):
    g = torch.Generator().manual_seed(seed)
    f = lambda *s, std=1.0: (torch.randn(s, generator=g) * std).to(DT[dt]).cuda()  # noqa: E731
    d = dict(x=f(T, inn), a=f(n, r, inn, std=inn ** -0.5), b=f(n, out, r, std=0.3), base=f(T, out), dy=f(T, out, std=0.1),
             dres=f(T, inn, std=0.1))
    for k in ("x", "base", "dy", "dres"):
        d[k] = _wide(d[k], extra, seed + 1)
    return d


def _slices(rows, slots):
    return [(slice(rows[i], rows[i + 1]), k) for i, k in enumerate(slots) if k >= 0]


def _close(got, want, bound, what):
    got, want, bound = (np.asarray(t.double().cpu() if torch.is_tensor(t) else t) for t in (got, want, bound))
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, worst {np.nanmax(np.abs(got - want) / bound):.3g} bounds"


def _forward_check(d, rows, slots, scale, dt, y, v, base):
    x, a, b = (d[k].double() for k in ("x", "a", "b"))
    y0 = base.double() if base is not None else torch.zeros(y.shape, dtype=torch.float64, device="cuda")
    want, ev = y0.clone(), torch.zeros(v.shape, dtype=torch.float64, device="cuda")
    bound = HALF[dt] * y0.abs()
    vb = torch.zeros_like(ev)
    for t, k in _slices(rows, slots):
        inn, r = a.shape[2], a.shape[1]
        ev[t] = x[t] @ a[k].t()
        vb[t] = (inn + 8) * u * (x[t].abs() @ a[k].abs().t())
        d_ = scale * (ev[t] @ b[k].t())
        want[t] += d_
        e = abs(scale) * (vb[t] @ b[k].abs().t() + (HELD[dt] + (2 * r + 8) * u) * (ev[t].abs() @ b[k].abs().t()))
        e += u * (y0[t].abs() + d_.abs())
        bound[t] = e + HALF[dt] * (want[t].abs() + e)
    _close(v, ev, vb, "v")
    _close(y, want, bound, "y")


def _backward_check(d, v, rows, slots, scale, dt, dx, da, db, dres, da0, db0):
    x, a, b, dy = (d[k].double() for k in ("x", "a", "b", "dy"))
    v = v.double()
    r0 = dres.double() if dres is not None else torch.zeros(x.shape, dtype=torch.float64, device="cuda")
    wx, bx = r0.clone(), HALF[dt] * r0.abs()
    wa, wb = da0.double().clone(), db0.double().clone()
    ba, bb = torch.zeros_like(wa), torch.zeros_like(wb)
    na, nb, hits = torch.zeros_like(wa), torch.zeros_like(wb), {}
    for t, k in _slices(rows, slots):
        out, r, T = b.shape[1], a.shape[1], t.stop - t.start
        dv = scale * (dy[t] @ b[k])
        edv = (abs(scale) * (out + 24) * u) * (dy[t].abs() @ b[k].abs())
        dd = dv @ a[k]
        wx[t] += dd
        e = edv @ a[k].abs() + (HELD[dt] + (2 * r + 8) * u) * (dv.abs() @ a[k].abs()) + u * (r0[t].abs() + dd.abs())
        bx[t] = e + HALF[dt] * (wx[t].abs() + e)
        wa[k] += dv.t() @ x[t]
        ba[k] += edv.t() @ x[t].abs()
        na[k] += dv.abs().t() @ x[t].abs()
        wb[k] += scale * (dy[t].t() @ v[t])
        nb[k] += abs(scale) * (dy[t].abs().t() @ v[t].abs())
        hits[k] = hits.get(k, 0) + T
    for k, T in hits.items():  # three parts a product, their sums over rows and slabs, the sum with the old gradient
        ba[k] += (2.0 ** -24 + (3 * T + 64) * u) * na[k] + u * (da0[k].double().abs() + wa[k].abs())
        bb[k] += (2.0 ** -24 + (3 * T + 64) * u) * nb[k] + u * (db0[k].double().abs() + wb[k].abs())
    if dx is not None:
        _close(dx, wx, bx, "dx")
    _close(da, wa, ba, "da")
    _close(db, wb, bb, "db")
    for k in range(a.shape[0]):  # slots of no client stay as they were
        if k not in hits:
            assert torch.equal(da[k], da0[k]) and torch.equal(db[k], db0[k])


def _run(lens, slots, n, r, inn, out, dt, scale=2.0, seed=0, extra=0, base="given", dres="given", with_dx=True):
    batch, rows = _batch(lens)
    T = batch.total_tokens
    d = _inputs(T, n, r, inn, out, dt, seed, extra)
    op = ClientAdapters(n, r, inn, out, dt, scale)
    ws = op.workspace(batch)
    print(f"[adapters] T={T} clients={len(lens)} r={r} {inn}->{out} {dt}", flush=True)
    b0 = None if base == "none" else d["base"].clone() if base == "inplace" else d["base"]
    keep = None if base == "none" else d["base"].clone()
    y = b0 if base == "inplace" else _wide(torch.full((T, out), 7.0, dtype=DT[dt], device="cuda"), extra, 9)
    v = torch.full((T, r), 9.0, device="cuda")
    op.forward(batch, slots, d["x"], d["a"], d["b"], b0, y, v, ws)
    _forward_check(d, rows, slots, scale, dt, y, v, keep)
    g = torch.Generator().manual_seed(seed + 5)
    da0, db0 = torch.randn((n, r, inn), generator=g).cuda(), torch.randn((n, out, r), generator=g).cuda()
    da, db = da0.clone(), db0.clone()
    r0 = None if dres == "none" else d["dres"].clone() if dres == "inplace" else d["dres"]
    keep = None if dres == "none" else d["dres"].clone()
    dx = None
    if with_dx:
        dx = r0 if dres == "inplace" else _wide(torch.full((T, inn), 7.0, dtype=DT[dt], device="cuda"), extra, 10)
    else:
        r0 = None
    op.backward(batch, slots, d["dy"], d["x"], d["a"], d["b"], v, r0, dx, da, db, ws)
    _backward_check(d, v, rows, slots, scale, dt, dx, da, db, keep, da0, db0)
    return d, batch, rows, op, ws, y, v, dx, da, db


CASES = [
    # lens of clients, slots, n, r, in, out
    ([[1]], [0], 1, 8, 8, 8),
    ([[1]], [-1], 1, 8, 64, 24),                                        # nobody has an adapter
    ([[5, 9], [7]], [1, 0], 3, 8, 64, 96),                              # a slot of nobody
    ([[63], [64], [65]], [0, 1, 2], 3, 16, 520, 264),
    ([[31], [32], [33], [1]], [2, 2, 0, 2], 3, 24, 128, 136),           # shared, neighbours and apart
    ([[129], [1], [2], [200]], [-1, 0, -1, 0], 1, 32, 256, 768),
    ([[70, 3], [41]], [0, 1], 2, 40, 1032, 520),
    ([[257]], [0], 1, 64, 640, 1096),
    ([[700], [30]], [0, 0], 2, 16, 256, 512),                           # several slabs of one slot
]


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_adapters_match_float64(case, dt):
    _run(*CASES[case], dt, seed=case)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("r", [8, 16, 32, 48, 64])
def test_every_rank_width(r, dt):
    _run([[100], [37]], [1, 0], 2, r, 264, 328, dt, seed=r)


@pytest.mark.parametrize("base,dres,with_dx", [("none", "none", True), ("inplace", "inplace", True),
                                               ("given", "none", False)])
@pytest.mark.parametrize("slots", [[0, -1, 1], [-1, -1, -1]])
def test_bases_of_every_kind(slots, base, dres, with_dx):
    _run([[40], [21], [90]], slots, 2, 16, 96, 200, "bf16", base=base, dres=dres, with_dx=with_dx)


@pytest.mark.parametrize("slots", [[0, -1, 1], [-1, -1, -1]])
def test_projection_in_place_with_a_divided_reduction(slots):
    """Few rows of many columns: v is summed over workgroups, also the zeros of
    clients without an adapter, whose rows of y stay as they are."""
    _run([[40], [21], [90]], slots, 2, 16, 1032, 200, "bf16", base="inplace", dres="inplace")


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_rows_apart_in_memory(dt):
    """Strided x, base, y, dy, dres and dx; what lies between their rows stays."""
    batch, rows = _batch([[50], [19]])
    d = _inputs(69, 2, 16, 72, 104, dt, 3, extra=24)
    op = ClientAdapters(2, 16, 72, 104, dt, 0.5)
    ws = op.workspace(batch)
    ybuf, xbuf = (torch.full((69, w + 16), 7.0, dtype=DT[dt], device="cuda") for w in (104, 72))
    v = torch.empty((69, 16), device="cuda")
    y, dx = ybuf[:, 8:112], xbuf[:, 8:80]
    op.forward(batch, [1, 0], d["x"], d["a"], d["b"], d["base"], y, v, ws)
    _forward_check(d, rows, [1, 0], 0.5, dt, y, v, d["base"])
    da, db = torch.zeros((2, 16, 72), device="cuda"), torch.zeros((2, 104, 16), device="cuda")
    op.backward(batch, [1, 0], d["dy"], d["x"], d["a"], d["b"], v, d["dres"], dx, da, db, ws)
    _backward_check(d, v, rows, [1, 0], 0.5, dt, dx, da, db, d["dres"], torch.zeros_like(da), torch.zeros_like(db))
    for buf, w in ((ybuf, 104), (xbuf, 72)):
        assert (buf[:, :8] == 7).all() and (buf[:, 8 + w:] == 7).all()


def test_more_clients_than_one_launch_takes():
    """300 clients of one to three rows in 7 slots, spread over three launches."""
    rng = np.random.default_rng(0)
    lens = [[int(n)] for n in rng.integers(1, 4, 300)]
    slots = [int(k) for k in rng.integers(-1, 7, 300)]
    _run(lens, slots, 7, 16, 256, 384, "bf16", seed=4)


def test_one_token_each_wide():
    """A generation step at the ChatGLM-6B projection's width."""
    _run([[1]] * 40, [i % 9 - 1 for i in range(40)], 8, 16, 4096, 12288, "bf16", seed=5)


def test_long_clients_wide():
    _run([[1100], [257], [33]], [1, 0, 1], 2, 32, 4096, 4096, "bf16", seed=6)


@pytest.mark.parametrize("r", [16, 24, 64])
def test_batches_larger_than_the_cache(r):
    """Two clients at once, 139 MB a matrix, and each alone: y, v and dx of the same
    bits; dA and dB apart by their sums over the rows."""
    lens, inn, n = [8600, 8400], 4096, 2
    both, rows = _batch([[k] for k in lens])
    d = _inputs(17000, n, r, inn, inn, "bf16", 21)
    op = ClientAdapters(n, r, inn, inn, "bf16", 0.5)

    def run(batch, slots, t):
        T = batch.total_tokens
        ws, y, v = op.workspace(batch), torch.empty_like(d["base"][t]), torch.empty((T, r), device="cuda")
        op.forward(batch, slots, d["x"][t], d["a"], d["b"], d["base"][t], y, v, ws)
        da, db = torch.zeros((n, r, inn), device="cuda"), torch.zeros((n, inn, r), device="cuda")
        dx = torch.empty_like(d["dres"][t])
        op.backward(batch, slots, d["dy"][t], d["x"][t], d["a"], d["b"], v, d["dres"][t], dx, da, db, ws)
        return y, v, dx, da, db

    got = run(both, [1, 0], slice(0, 17000))
    for c, k in ((0, 1), (1, 0)):
        t, T = slice(rows[c], rows[c + 1]), lens[c]
        one = run(_batch([[T]])[0], [k], t)
        for p, q in zip(got[:3], one[:3]):
            assert torch.equal(p[t], q)
        x, dy, v = d["x"][t].double(), d["dy"][t].double(), got[1][t].double()
        dv = 0.5 * dy @ d["b"][k].double()
        # two sums of T products, each as in the module's bounds
        for p, q, size in ((got[3][k], one[3][k], dv.abs().t() @ x.abs()),
                           (got[4][k], one[4][k], 0.5 * dy.abs().t() @ v.abs())):
            assert ((p.double() - q.double()).abs() <= 2 * (3 * T + 64) * u * size).all()
    # and against the formula, on a sample of rows
    t = torch.arange(0, 17000, 331, device="cuda")
    k = (t < 8600).long()
    x, dy = d["x"][t].double(), d["dy"][t].double()
    v = torch.stack([d["a"][j].double() @ x[i] for i, j in enumerate(k)])
    y = d["base"][t].double() + 0.5 * torch.stack([d["b"][j].double() @ v[i] for i, j in enumerate(k)])
    dv = 0.5 * torch.stack([d["b"][j].double().t() @ dy[i] for i, j in enumerate(k)])
    dx = d["dres"][t].double() + torch.stack([d["a"][j].double().t() @ dv[i] for i, j in enumerate(k)])
    for p, q, e in ((got[0][t], y, y.abs() + 1), (got[2][t], dx, dx.abs() + 1)):
        # half a step of bf16, and fp32 sums of 4096 terms below it
        assert ((p.double() - q).abs() <= 2.0 ** -8 * q.abs() + 2.0 ** -12 * e).all()


def test_infinities_and_nan_stay_in_their_rows():
    """A row with an infinity or NaN spoils its own outputs and no other row's,
    a client's without an adapter none."""
    batch, rows = _batch([[20], [20], [20]])
    d = _inputs(60, 2, 16, 64, 96, "bf16", 8)
    op = ClientAdapters(2, 16, 64, 96, "bf16", 1.0)
    ws = op.workspace(batch)
    y, v = torch.empty((60, 96), dtype=torch.bfloat16, device="cuda"), torch.empty((60, 16), device="cuda")
    op.forward(batch, [0, -1, 1], d["x"], d["a"], d["b"], d["base"], y, v, ws)
    x2 = d["x"].clone()
    x2[3, 5], x2[25, 7], x2[44, 0] = float("inf"), float("nan"), float("nan")
    y2, v2 = torch.empty_like(y), torch.empty_like(v)
    op.forward(batch, [0, -1, 1], x2, d["a"], d["b"], d["base"], y2, v2, ws)
    same = torch.ones(60, dtype=torch.bool)
    same[3] = same[44] = False
    assert torch.equal(y[same], y2[same]) and torch.equal(v[same], v2[same])
    assert not torch.isfinite(v2[3]).any() and torch.isnan(y2[44].float()).all()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("r", [8, 40])
def test_nan_in_a_gradient_stays_with_its_slot(r, dt):
    """NaN and infinities in dy and x: a client without an adapter passes none on,
    a client with one spoils its slot's gradients and its own row of dx only."""
    batch, rows = _batch([[20], [20], [20], [7]])
    slots = [0, -1, 1, 0]
    d = _inputs(67, 2, r, 64, 96, dt, 8)
    op = ClientAdapters(2, r, 64, 96, dt, 1.0)
    ws = op.workspace(batch)

    def run(x, dy):
        y, v = torch.empty((67, 96), dtype=DT[dt], device="cuda"), torch.empty((67, r), device="cuda")
        op.forward(batch, slots, x, d["a"], d["b"], None, y, v, ws)
        dx = torch.empty_like(x)
        da, db = torch.zeros((2, r, 64), device="cuda"), torch.zeros((2, 96, r), device="cuda")
        op.backward(batch, slots, dy, x, d["a"], d["b"], v, d["dres"], dx, da, db, ws)
        return dx, da, db

    dx, da, db = run(d["x"], d["dy"])
    x, dy = d["x"].clone(), d["dy"].clone()
    x[25, 7], dy[26, 3], dy[39] = float("nan"), float("inf"), float("nan")  # no adapter
    for p, q in zip((dx, da, db), run(x, dy)):
        assert torch.equal(p, q)
    x[3, 5], dy[64, 2] = float("inf"), float("nan")  # slot 0
    dx2, da2, db2 = run(x, dy)
    assert torch.equal(da[1], da2[1]) and torch.equal(db[1], db2[1])
    keep = torch.ones(67, dtype=torch.bool)
    keep[64] = False
    assert torch.equal(dx[keep], dx2[keep]) and torch.isnan(dx2[64].float()).all()
    assert not torch.isfinite(da2[0]).all() and not torch.isfinite(db2[0]).all()


def test_slots_of_any_sequence():
    """A list, a tuple, and arrays that are read-only, strided or of 64 bits."""
    batch, rows = _batch([[5], [3], [4]])
    d = _inputs(12, 3, 8, 64, 96, "bf16", 2)
    op = ClientAdapters(3, 8, 64, 96, "bf16", 1.0)
    ws, outs = op.workspace(batch), []
    fixed = np.array([2, -1, 0], np.int32)
    fixed.setflags(write=False)
    for slots in ([2, -1, 0], (2, -1, 0), fixed, np.array([2, 9, -1, 9, 0, 9], np.int32)[::2], np.array([2, -1, 0])):
        y, v = torch.empty((12, 96), dtype=torch.bfloat16, device="cuda"), torch.empty((12, 8), device="cuda")
        op.forward(batch, slots, d["x"], d["a"], d["b"], d["base"], y, v, ws)
        outs.append((y, v))
    assert all(torch.equal(p, q) for o in outs[1:] for p, q in zip(outs[0], o))
    for slots in ([2, -1], [2, -1, 3], [2, -2, 0], [[2, -1, 0]], [2, -1, 2 ** 32]):
        with pytest.raises((FlglmError, OverflowError)):
            op.forward(batch, slots, d["x"], d["a"], d["b"], d["base"], y, v, ws)


def test_results_repeat_bit_for_bit():
    d, batch, rows, op, ws, y, v, dx, da, db = _run([[300], [150], [333]], [0, 1, 0], 2, 16, 512, 768, "bf16")
    first = None
    for _ in range(3):
        ws.fill_(255)  # nothing is kept in the workspace
        y2, v2, dx2 = torch.empty_like(y), torch.empty_like(v), torch.empty_like(dx)
        da2, db2 = torch.zeros_like(da), torch.zeros_like(db)
        op.forward(batch, [0, 1, 0], d["x"], d["a"], d["b"], d["base"], y2, v2, ws)
        op.backward(batch, [0, 1, 0], d["dy"], d["x"], d["a"], d["b"], v2, d["dres"], dx2, da2, db2, ws)
        now = (y2, v2, dx2, da2, db2)
        first = first or now
        assert all(torch.equal(p, q) for p, q in zip(first, now))


def test_captured_and_replayed_on_another_stream():
    batch, rows = _batch([[90], [1], [40]])
    slots = [0, 1, 0]
    d = _inputs(131, 2, 16, 256, 512, "bf16", 11)
    op = ClientAdapters(2, 16, 256, 512, "bf16", 2.0)
    ws, ws2 = op.workspace(batch), op.workspace(batch)
    out = lambda: (torch.empty((131, 512), dtype=torch.bfloat16, device="cuda"), torch.empty((131, 16), device="cuda"),  # noqa: E731
                   torch.empty((131, 256), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, 16, 256), device="cuda"),
                   torch.zeros((2, 512, 16), device="cuda"))

    def both(o, w):
        y, v, dx, da, db = o
        da.zero_()
        db.zero_()
        op.forward(batch, slots, d["x"], d["a"], d["b"], d["base"], y, v, w)
        op.backward(batch, slots, d["dy"], d["x"], d["a"], d["b"], v, d["dres"], dx, da, db, w)

    captured, eager = out(), out()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both(captured, ws)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(captured, ws)
    for i in range(4):
        d["x"].copy_(torch.randn_like(d["x"]))
        both(eager, ws2)
        for t in captured:
            t.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(captured, eager)), i


def test_two_streams_at_once():
    """Calls of one handle with a workspace each, on two streams: the results of one
    after the other."""
    parts = []
    op = ClientAdapters(2, 16, 1024, 2048, "bf16", 2.0)
    for seed, lens, slots in ((1, [[300], [41]], [1, 0]), (2, [[17], [1], [250]], [0, -1, 0])):
        batch, rows = _batch(lens)
        d = _inputs(rows[-1], 2, 16, 1024, 2048, "bf16", seed)
        parts.append((batch, slots, d, op.workspace(batch)))

    def run(batch, slots, d, ws, stream=None):
        T = batch.total_tokens
        y, v = torch.empty((T, 2048), dtype=torch.bfloat16, device="cuda"), torch.empty((T, 16), device="cuda")
        dx, da = torch.empty_like(d["x"]), torch.zeros((2, 16, 1024), device="cuda")
        db = torch.zeros((2, 2048, 16), device="cuda")
        torch.cuda.synchronize()
        return (y, v, dx, da, db), lambda: (
            op.forward(batch, slots, d["x"], d["a"], d["b"], d["base"], y, v, ws, stream),
            op.backward(batch, slots, d["dy"], d["x"], d["a"], d["b"], v, d["dres"], dx, da, db, ws, stream))

    want = []
    for p in parts:
        out, go = run(*p)
        go()
        torch.cuda.synchronize()
        want.append(out)
    streams = [torch.cuda.Stream() for _ in parts]
    both = [run(*p, s) for p, s in zip(parts, streams)]
    for _ in range(5):
        for out, _ in both:
            out[3].zero_()
            out[4].zero_()
        torch.cuda.synchronize()
        for _, go in both:
            go()
        torch.cuda.synchronize()
        for (out, _), w in zip(both, want):
            assert all(torch.equal(p, q) for p, q in zip(out, w))


def test_offsets_past_32_bits():
    """Rows 65536 elements apart: the last ones lie past 2^31 elements."""
    T, step = 40000, 65536
    batch, rows = _batch([[20000], [20000]])
    buf = torch.empty((T, step), dtype=torch.bfloat16, device="cuda")
    x = buf[:, 65536 - 64:]
    g = torch.Generator(device="cuda").manual_seed(0)
    x.copy_(torch.randn((T, 64), generator=g, device="cuda"))
    op = ClientAdapters(2, 8, 64, 64, "bf16", 1.0)
    a, b = (torch.randn(s, generator=g, device="cuda").bfloat16() for s in ((2, 8, 64), (2, 64, 8)))
    ws, v = op.workspace(batch), torch.empty((T, 8), device="cuda")
    y = buf[:, :64]
    op.forward(batch, [1, 0], x, a, b, None, y, v, ws)
    close, v2, y2 = x.contiguous(), torch.empty_like(v), torch.empty((T, 64), dtype=torch.bfloat16, device="cuda")
    op.forward(batch, [1, 0], close, a, b, None, y2, v2, ws)
    assert torch.equal(v, v2) and torch.equal(y, y2)
    dx, dx2 = buf[:, 128:192], torch.empty_like(close)
    da, db, da2, db2 = (torch.zeros(s, device="cuda") for s in ((2, 8, 64), (2, 64, 8)) * 2)
    op.backward(batch, [1, 0], y, x, a, b, v, None, dx, da, db, ws)
    op.backward(batch, [1, 0], y2, close, a, b, v, None, dx2, da2, db2, ws)
    assert torch.equal(dx, dx2) and torch.equal(da, da2) and torch.equal(db, db2)


def test_gradients_against_differences():
    """f = sum(y * g) is linear in x, in A and in B apart: its central difference
    of any width is the derivative, up to the rounding of two forwards."""
    batch, rows = _batch([[30], [17]])
    slots, scale = [1, 0], 1.5
    d = _inputs(47, 2, 8, 64, 96, "f32", 13)
    op = ClientAdapters(2, 8, 64, 96, "f32", scale)
    ws = op.workspace(batch)

    def f(x, a, b):
        y, v = torch.empty((47, 96), device="cuda"), torch.empty((47, 8), device="cuda")
        op.forward(batch, slots, x, a, b, None, y, v, ws)
        return float((y.double() * d["dy"].double()).sum()), v

    _, v = f(d["x"], d["a"], d["b"])
    dx, da, db = torch.empty_like(d["x"]), torch.zeros_like(d["a"]), torch.zeros_like(d["b"])
    op.backward(batch, slots, d["dy"], d["x"], d["a"], d["b"], v, None, dx, da, db, ws)
    for name, grad in (("x", dx), ("a", da), ("b", db)):
        step = torch.randn(d[name].shape, generator=torch.Generator().manual_seed(1)).cuda()
        args = {k: d[k] for k in ("x", "a", "b")}
        hi, lo = dict(args, **{name: args[name] + step}), dict(args, **{name: args[name] - step})
        diff = (f(**hi)[0] - f(**lo)[0]) / 2
        # every y is off by at most (in + r + 16) u times the sum of its terms' magnitudes
        size = 0.0
        for q in (hi, lo):
            for t, k in _slices(rows, slots):
                m = (q["x"][t].double().abs() @ q["a"][k].double().abs().t()) @ q["b"][k].double().abs().t()
                size += float((m * d["dy"][t].double().abs()).sum())
        bound = scale * (64 + 8 + 16) * u * size
        got = float((grad.double() * step.double()).sum())
        assert abs(got - diff) <= bound + 1e-6 * abs(diff), (name, got, diff, bound)
