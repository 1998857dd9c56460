"""Preference tuning of the split model with each client's own adapters: the
server stack with adapters against dense weights and against differences, and
one whole step (stack with adapters, head with the preference loss, backward,
clipping, Adam) as a program runs it."""

import math

import numpy as np
import pytest

import oracle
import synth
from tests.gpu_helpers import TOL, dev, rel_l2

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
from paper_2406_14898_amd import (BatchDesc, ClientHead, FlglmError, GradNorm, ParamArena, PreferenceLoss,  # noqa: E402
                                  ServerStack, StackAdapters)

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _adapters(n, r, H, layers, dt, seed, std_b=0.05):
    g = torch.Generator().manual_seed(seed)
    return [dict(a=(torch.randn((n, r, H), generator=g) * H ** -0.5).to(DT[dt]).cuda(),
                 b=(torch.randn((n, 3 * H, r), generator=g) * std_b).to(DT[dt]).cuda()) for _ in range(layers)]


def _zeros(ad):
    return [{k: torch.zeros(v.shape, device="cuda") for k, v in d.items()} for d in ad]


def _one_client_oracle(shape, layers, ad, slot, scale, x, dy, batch):
    """The dense stack whose W_qkv holds the client's adapters: its output, dx and
    the adapters' gradients from dW_qkv = dqkv^T u."""
    merged = []
    for p, d in zip(layers, ad):
        w = np.array(p["w_qkv"], np.float64)
        if slot >= 0:
            a, b = (d[k][slot].double().cpu().numpy() for k in ("a", "b"))
            w = w + scale * b @ a
        merged.append(dict(p, w_qkv=w))
    y, xs = oracle.stack_forward(merged, len(merged), x, batch, shape)
    dx, grads = oracle.stack_backward(merged, len(merged), xs, dy, batch, shape)
    ga = []
    for g, d in zip(grads, ad):
        if slot >= 0:
            a, b = (d[k][slot].double().cpu().numpy() for k in ("a", "b"))
            ga.append((scale * b.T @ g["w_qkv"], scale * g["w_qkv"] @ a.T))
        else:
            ga.append(None)
    return y, dx, ga


@pytest.mark.parametrize("recompute", [False, True])
@pytest.mark.parametrize("dt,frozen", [("f32", True), ("f32", False), ("bf16", True)])
def test_stack_with_adapters_matches_merged_weights(dt, frozen, recompute):
    """Every client's rows equal the dense stack with that client's adapters in
    its W_qkv (float64): y, dx, and dA, dB summed over the slot's clients."""
    shape = synth.StackShape(num_layers=2, hidden=256, num_heads=4, ffn_hidden=512, rotary_dim=32)
    lens, slots, scale, n, r = [[19, 33], [40], [27], [8]], [1, 0, -1, 1], 2.0, 3, 8
    cu, csp = [0], [0]
    for c in lens:
        for k in c:
            cu.append(cu[-1] + k)
        csp.append(len(cu) - 1)
    T = cu[-1]
    layers = [synth.layer_params(shape, l, seed=3, bf16=dt == "bf16") for l in range(2)]
    ad = _adapters(n, r, 256, 2, dt, 4)
    x = synth.activations(T, 256, seed=5, bf16=dt == "bf16")
    dy = synth.upstream_grad(T, 256, seed=6, bf16=dt == "bf16")
    stack = ServerStack(2, 256, 4, 512, 32, dt)
    batch = BatchDesc(cu, csp)
    params = [{k: dev(v, dt) for k, v in p.items()} for p in layers]
    grads = [{} if frozen else {k: torch.zeros(v.shape, device="cuda") for k, v in p.items()} for p in params]
    ga = _zeros(ad)
    adapters = StackAdapters(stack, batch, slots, ad, ga, scale)
    saved, ws = stack.buffers(batch, recompute)
    X, DY = dev(x, dt), dev(dy, dt)
    Y, DX = torch.empty_like(X), torch.empty_like(X)
    stack.forward(batch, params, X, Y, saved, ws, recompute, adapters=adapters)
    stack.backward(batch, params, grads, X, saved, DY, DX, ws, recompute, adapters=adapters)
    torch.cuda.synchronize()
    want = {k: [None, None] for k in range(n)}
    for c, slot in enumerate(slots):
        t = slice(cu[csp[c]], cu[csp[c + 1]])
        sub = synth.Batch(np.asarray(cu[csp[c]:csp[c + 1] + 1], np.int32) - t.start,
                          np.asarray([0, csp[c + 1] - csp[c]], np.int32))
        y, dx, g = _one_client_oracle(shape, layers, ad, slot, scale, x[t], dy[t], sub)
        assert rel_l2(Y[t].double().cpu().numpy(), y) < TOL[dt]
        assert rel_l2(DX[t].double().cpu().numpy(), dx) < TOL[dt]
        if slot >= 0:
            for l in range(2):
                old = want[slot][l]
                want[slot][l] = g[l] if old is None else (old[0] + g[l][0], old[1] + g[l][1])
    for k in range(n):
        for l in range(2):
            if want[k][l] is None:  # the slot of nobody
                assert not ga[l]["a"][k].any() and not ga[l]["b"][k].any()
                continue
            for name, w in zip(("a", "b"), want[k][l]):
                assert rel_l2(ga[l][name][k].double().cpu().numpy(), w) < TOL[dt], (k, l, name)
    stack.close()


@pytest.mark.parametrize("glm", [False, True])
def test_adapters_of_nobody_change_nothing(glm):
    """All slots -1: the bits of the calls without adapters, forward and backward."""
    shape = synth.StackShape(num_layers=2, hidden=256, num_heads=2, ffn_hidden=512, rotary_dim=64)
    kw = dict(residual_alpha=2.0, rotary_2d=True, num_prefix=16) if glm else {}
    stack = ServerStack(2, 256, 2, 512, 64, "bf16", **kw)
    batch = BatchDesc([0, 30, 71, 100], [0, 1, 3], [10, 0, 5])
    params = [{k: dev(v, "bf16") for k, v in synth.layer_params(shape, l, seed=1, bf16=True).items()} for l in range(2)]
    if glm:
        for l, p in enumerate(params):
            p.update({k: dev(v, "bf16") for k, v in synth.prefix_params(shape, l, 16, seed=1).items()})
    x, dy = (torch.randn((100, 256), generator=torch.Generator().manual_seed(s)).bfloat16().cuda() for s in (1, 2))
    ad = _adapters(1, 8, 256, 2, "bf16", 4)
    outs = []
    for use in (False, True):
        grads = [{k: torch.zeros(v.shape, device="cuda") for k, v in p.items()} for p in params]
        ga = _zeros(ad)
        adapters = StackAdapters(stack, batch, [-1, -1], ad, ga) if use else None
        saved, ws = stack.buffers(batch, False)
        y, dx = torch.empty_like(x), torch.empty_like(x)
        stack.forward(batch, params, x, y, saved, ws, adapters=adapters)
        stack.backward(batch, params, grads, x, saved, dy, dx, ws, adapters=adapters)
        torch.cuda.synchronize()
        outs.append([y, dx] + [g[k] for g in grads for k in sorted(g)])
        assert not any(t.any() for g in ga for t in g.values())
    assert all(torch.equal(p, q) for p, q in zip(*outs))
    stack.close()


class _Model:
    """Frozen blocks with trained adapters, the final linear layer and the
    preference loss on the server's output."""

    H, V, LAYERS, N, R = 256, 1000, 2, 2, 8

    def __init__(self, dt):
        shape = synth.StackShape(num_layers=self.LAYERS, hidden=self.H, num_heads=4, ffn_hidden=512, rotary_dim=32)
        self.dt = dt
        self.stack = ServerStack(self.LAYERS, self.H, 4, 512, 32, dt)
        self.params = [{k: dev(v, dt) for k, v in synth.layer_params(shape, l, seed=1, bf16=dt == "bf16").items()}
                       for l in range(self.LAYERS)]
        g = torch.Generator().manual_seed(2)
        self.w = (torch.randn((self.V, self.H), generator=g) * 0.05).to(DT[dt]).cuda()
        cu = [0, 20, 33, 50, 74, 80, 101]  # client 0 owns two pairs, client 1 one
        self.batch, self.cu = BatchDesc(cu, [0, 4, 6]), cu
        self.x = torch.randn((cu[-1], self.H), generator=g).to(DT[dt]).cuda()
        lab = torch.randint(0, self.V, (cu[-1],), generator=g).numpy().astype(np.int32)
        for a, b in zip(cu, cu[1:]):
            lab[a:a + (b - a) // 4] = -100
            lab[b - 1] = -100
        self.labels = lab
        self.head, self.loss = ClientHead(self.V, self.H, dt), PreferenceLoss(self.V, dt, 0.3, 0.1)
        names = [(f"{l}.{k}", s) for l in range(self.LAYERS)
                 for k, s in (("a", (self.N, self.R, self.H)), ("b", (self.N, 3 * self.H, self.R)))]
        self.arena = ParamArena(names, bf16_copy=dt == "bf16")
        ad = _adapters(self.N, self.R, self.H, self.LAYERS, "f32", 3)
        self.arena.load({f"{l}.{k}": ad[l][k] for l in range(self.LAYERS) for k in ("a", "b")})
        views, grads = self.arena.compute_views(), self.arena.grad_views()
        self.ad = [{k: views[f"{l}.{k}"] for k in ("a", "b")} for l in range(self.LAYERS)]
        self.ga = [{k: grads[f"{l}.{k}"] for k in ("a", "b")} for l in range(self.LAYERS)]
        self.adapters = StackAdapters(self.stack, self.batch, [1, 0], self.ad, self.ga, 1.5)
        self.saved, self.ws = self.stack.buffers(self.batch, False)
        self.hws, self.pws = self.head.workspace(cu[-1]), self.loss.workspace(self.batch)
        self.y, self.dy, self.dx = (torch.empty_like(self.x) for _ in range(3))
        self.out = self.loss.outputs(self.batch)
        self.ref = None

    def forward(self):
        self.stack.forward(self.batch, self.params, self.x, self.y, self.saved, self.ws, adapters=self.adapters)
        self.head.preference_forward(self.loss, self.batch, self.y, self.w, self.labels, self.ref, *self.out, self.hws,
                                     self.pws)
        return self.out[2]

    def backward(self):
        self.head.preference_backward(self.loss, self.batch, self.y, self.w, 1.0 / 3, self.dy, None, self.hws, self.pws)
        self.stack.backward(self.batch, self.params, [{}] * self.LAYERS, self.x, self.saved, self.dy, self.dx, self.ws,
                            adapters=self.adapters)


def test_one_step_of_preference_tuning():
    """Reference pass, loss, backward, clipping and Adam in the order of a training
    program.  At the reference's own weights every pair's loss is log 2; the
    whole gradient equals the slope of the loss along it (central differences of
    the mean loss, extrapolated); the clipped update is Adam's on the gradient
    scaled to norm 1."""
    m = _Model("f32")
    m.forward()
    m.ref = m.out[0].clone()  # the frozen reference is the model itself, before the step
    total = float(m.forward())
    assert abs(total - 3 * math.log(2)) < 1e-5
    m.backward()
    grad = m.arena.grad.clone()
    n = float(grad.double().norm())
    assert n > 1e-3
    # slope along g / |g|: the norm of the gradient
    master = m.arena.master.clone()
    d = grad / n

    def at(h):
        m.arena.master.copy_(master + h * d)
        return float(m.forward()) / 3

    h = 0.02
    wide, half = (at(h) - at(-h)) / (2 * h), (at(h / 2) - at(-h / 2)) / h
    slope = (4 * half - wide) / 3
    # losses near log 2 are rounded to 2^-24 of their size, and come from logits
    # whose fp32 errors of some 1e-6 a row, random in sign, add over 60 rows
    rounding = 0.3 * 1e-6 * math.sqrt(60) * 8 / h
    assert abs(slope - n) <= abs(wide - half) + rounding, (slope, n, wide, half)
    m.arena.master.copy_(master)
    norm = m.arena.clip_grad_norm(0.5 * n)
    assert abs(float(norm) - n) < 1e-6 * n
    assert torch.allclose(m.arena.grad, 0.5 * grad, rtol=1e-5, atol=0)
    m.arena.adam_step(lr=1e-3)
    moved = m.arena.master - master
    # Adam's first step: lr g / (|g| + eps), whatever the gradient's scale
    c = (0.5 * grad).double()
    want = -1e-3 * c / (c.abs() + 1e-8)
    assert torch.allclose(moved.double(), want, rtol=1e-3, atol=1e-7)
    assert float(m.arena.grad.abs().max()) == 0.0
    assert math.isfinite(float(m.forward()))


def test_step_in_bf16_repeats_bit_for_bit():
    outs = []
    for _ in range(2):
        m = _Model("bf16")
        m.forward()
        m.ref = m.out[0] + 1.0
        m.forward()
        m.backward()
        norm = m.arena.clip_grad_norm(1e-2)
        m.arena.adam_step(lr=1e-3)
        torch.cuda.synchronize()
        outs.append([t.clone() for t in m.out] + [norm.clone(), m.arena.master.clone(), m.arena.compute.clone(), m.dx])
    assert all(torch.equal(p, q) for p, q in zip(*outs))
    assert all(torch.isfinite(t.float()).all() for t in outs[0])


def test_adapters_of_another_stack_are_refused():
    stack = ServerStack(2, 256, 4, 512, 32, "bf16")
    batch = BatchDesc([0, 8], [0, 1])
    with pytest.raises(FlglmError):
        StackAdapters(stack, batch, [0], _adapters(1, 8, 256, 1, "bf16", 0))       # one block's adapters
    with pytest.raises(FlglmError):
        StackAdapters(stack, batch, [0], _adapters(1, 8, 512, 2, "bf16", 0))       # another width
    with pytest.raises(FlglmError):
        StackAdapters(stack, batch, [0], _adapters(1, 8, 256, 2, "f32", 0))        # another type
    with pytest.raises(FlglmError):
        StackAdapters(stack, batch, [0, 0], _adapters(1, 8, 256, 2, "bf16", 0))    # two clients' slots for one
    stack.close()


def test_adapters_of_another_batch_are_refused():
    """What the record and the workspace were not made for reaches no kernel."""
    stack, other = (ServerStack(2, 256, 4, 512, 32, "bf16") for _ in range(2))
    batch = BatchDesc([0, 8, 20], [0, 1, 2])
    ad = _adapters(1, 8, 256, 2, "bf16", 0)
    adapters = StackAdapters(stack, batch, [0, -1], ad)
    adapters.check(stack, batch)
    for s, b, backward in ((other, batch, False),                              # its workspace is another size
                           (stack, BatchDesc([0, 8, 14, 20], [0, 1, 2, 3]), False),  # three clients, two slots
                           (stack, BatchDesc([0, 8, 21], [0, 1, 2]), False),   # v of 20 rows
                           (stack, batch, True)):                              # forward only
        with pytest.raises(FlglmError):
            adapters.check(s, b, backward)
    x = torch.zeros((20, 256), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(FlglmError):
        stack.forward(BatchDesc([0, 8, 14, 20], [0, 1, 2, 3]), [{}, {}], x, torch.empty_like(x), None, x, adapters=adapters)
    with pytest.raises(FlglmError):
        stack.backward(batch, [{}, {}], [{}, {}], x, x, x, torch.empty_like(x), x, adapters=adapters)
    other.close()
    stack.close()


def test_adapters_keep_their_tensors():
    """The record holds addresses: a tensor replaced in its dict stays alive."""
    stack = ServerStack(2, 256, 4, 512, 32, "bf16")
    ad = _adapters(1, 8, 256, 2, "bf16", 0)
    adapters = StackAdapters(stack, BatchDesc([0, 8], [0, 1]), [0], ad, _zeros(ad))
    held = [t.data_ptr() for t in adapters.tensors]
    for d in ad:
        d["a"] = d["b"] = None
    assert [p for la in adapters.record.layers[:2] for p in (la.a, la.b)] == held[:4]
    assert [p for la in adapters.record.grads[:2] for p in (la.a, la.b)] == held[4:]
    stack.close()


def test_adapters_with_prefix_and_glm_blocks():
    """P-tuning prefix, scaled residual, 2-D positions and a bidirectional context:
    one client's adapters against the stack whose W_qkv holds them, both in bf16
    (each within the stack's own tolerance of the exact result)."""
    shape = synth.StackShape(num_layers=2, hidden=256, num_heads=2, ffn_hidden=512, rotary_dim=64)
    stack = ServerStack(2, 256, 2, 512, 64, "bf16", residual_alpha=2.0, rotary_2d=True, num_prefix=16)
    batch = BatchDesc([0, 30, 71], [0, 2], [10, 7])
    raw = [dict(synth.layer_params(shape, l, seed=1, bf16=True), **synth.prefix_params(shape, l, 16, seed=1))
           for l in range(2)]
    params = [{k: dev(v, "bf16") for k, v in p.items()} for p in raw]
    ad = _adapters(1, 16, 256, 2, "bf16", 4)
    merged = []
    for p, d in zip(params, ad):
        w = p["w_qkv"].double() + 1.5 * d["b"][0].double() @ d["a"][0].double()
        merged.append(dict(p, w_qkv=w.to(torch.bfloat16)))
    x, dy = (torch.randn((71, 256), generator=torch.Generator().manual_seed(s)).bfloat16().cuda() for s in (1, 2))
    outs, dw = [], None
    for use in (True, False):
        grads = [{k: torch.zeros(v.shape, device="cuda") for k, v in p.items()} for p in params]
        ga = _zeros(ad)
        adapters = StackAdapters(stack, batch, [0], ad, ga, 1.5) if use else None
        saved, ws = stack.buffers(batch, False)
        y, dx = torch.empty_like(x), torch.empty_like(x)
        stack.forward(batch, params if use else merged, x, y, saved, ws, adapters=adapters)
        stack.backward(batch, params if use else merged, grads, x, saved, dy, dx, ws, adapters=adapters)
        torch.cuda.synchronize()
        outs.append([y, dx] + [g[k] for g in grads for k in ("prefix_k", "prefix_v")])
        if use:
            got = ga
        else:
            dw = [g["w_qkv"].double() for g in grads]
    tol = 2 * TOL["bf16"]
    for p, q in zip(*outs):
        assert rel_l2(p.double().cpu().numpy(), q.double().cpu().numpy()) < tol
    for l in range(2):
        a, b = (ad[l][k][0].double() for k in ("a", "b"))
        for name, w in (("a", 1.5 * b.t() @ dw[l]), ("b", 1.5 * dw[l] @ a.t())):
            assert rel_l2(got[l][name][0].double().cpu().numpy(), w.cpu().numpy()) < tol, (l, name)
    stack.close()


@pytest.mark.parametrize("recompute", [False, True])
def test_stack_with_adapters_captured(recompute):
    """Forward, backward and clipping in one graph: every replay equals the eager
    calls on the same input, with eager work of its own workspaces between."""
    shape = synth.StackShape(num_layers=2, hidden=256, num_heads=4, ffn_hidden=512, rotary_dim=32)
    stack = ServerStack(2, 256, 4, 512, 32, "bf16")
    params = [{k: dev(v, "bf16") for k, v in synth.layer_params(shape, l, seed=1, bf16=True).items()} for l in range(2)]
    batch = BatchDesc([0, 40, 41, 90], [0, 1, 3])
    ad = _adapters(2, 8, 256, 2, "bf16", 4)
    x, dy = (torch.randn((90, 256), generator=torch.Generator().manual_seed(s)).bfloat16().cuda() for s in (1, 2))

    def side_of_one():
        ga = _zeros(ad)
        adapters = StackAdapters(stack, batch, [1, 0], ad, ga, 2.0)
        saved, ws = stack.buffers(batch, recompute)
        y, dx = torch.empty_like(x), torch.empty_like(x)
        norm = GradNorm([t for d in ga for t in d.values()])

        def run():
            for d in ga:
                for t in d.values():
                    t.zero_()
            stack.forward(batch, params, x, y, saved, ws, recompute, adapters=adapters)
            stack.backward(batch, params, [{}, {}], x, saved, dy, dx, ws, recompute, adapters=adapters)
            norm.clip(0.5)
        return run, [y, dx, norm.result] + [t for d in ga for t in d.values()]

    captured, a = side_of_one()
    eager, b = side_of_one()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        captured()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured()
    for i in range(4):
        x.copy_(torch.randn_like(x))
        eager()
        for t in a:
            t.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(a, b)), i
    stack.close()
