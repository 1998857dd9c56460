"""Global gradient norm and clipping against float64 (norm: one rounding to
fp32; a clipped value: the coefficient's rounding, the product's, and the
output type's)."""

import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
from paper_2406_14898_amd import GradNorm, ParamArena  # noqa: E402
from paper_2406_14898_amd import flglm as F  # noqa: E402

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def _grads(sizes, dt, seed=0, std=0.01):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(n, generator=g) * std).to(DT[dt]).cuda() for n in sizes]


def _norm64(grads):
    return math.sqrt(sum(float(g.double().square().sum()) for g in grads))


def _check(grads, out, norm, max_norm, dt):
    n = _norm64(grads)
    assert abs(float(norm) - n) <= 2.0 ** -23 * n + 1e-45
    c = min(1.0, max_norm / (n + 1e-6))
    for g, o in zip(grads, out):
        w = g.double() * c
        assert ((o.double() - w).abs() <= (2.0 ** -23 + HALF[dt]) * w.abs() + 2.0 ** -126).all()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("sizes", [[1], [7, 0, 1, 8], [4096], [65537, 3, 2048, 2049], [1 << 20, 5], [0, 0],
                                   [100] * 300 + [0] * 5 + [9]])
def test_norm_and_clip(sizes, dt):
    grads = _grads(sizes, dt)
    op = GradNorm(grads)
    n = _norm64(grads)
    print(f"[grad norm] {len(sizes)} tensors, {sum(sizes)} elements, {dt}", flush=True)
    for max_norm in (0.5 * n, 2 * n + 1, 0.0, math.inf):
        out = [torch.full_like(g, 7) for g in grads]
        norm = op.clip(max_norm, out=out)
        if math.isinf(max_norm) or max_norm > n:
            assert all(torch.equal(g, o) for g, o in zip(grads, out))
        _check(grads, out, norm, max_norm, dt)
        inside = [g.clone() for g in grads]
        norm2 = GradNorm(inside).clip(max_norm)
        assert torch.equal(norm, norm2) and all(torch.equal(a, b) for a, b in zip(inside, out))


def test_squares_outside_fp32():
    """Gradients whose squares overflow or vanish in fp32 have a norm all the same."""
    for big in (1e30, 1e-30):
        g = [torch.full((1000,), big, device="cuda"), torch.full((3,), -big, device="cuda")]
        assert abs(float(GradNorm(g).norm()) / (big * math.sqrt(1003)) - 1) <= 2.0 ** -22


def test_infinity_and_nan():
    g = [torch.ones(50, device="cuda"), torch.ones(9, device="cuda")]
    op = GradNorm(g)
    g[1][4] = math.inf
    out = [torch.empty_like(t) for t in g]
    assert float(op.clip(1.0, out=out)) == math.inf and float(op.result[1]) == 0.0
    assert (out[0] == 0).all() and math.isnan(float(out[1][4]))
    g[0][7] = math.nan
    assert math.isnan(float(op.clip(1.0, out=out))) and torch.isnan(out[0]).all() and torch.isnan(out[1]).all()
    assert float(op.norm(math.inf)) != 0 and float(op.result[1]) == 1.0


def test_untouched_around_unaligned_ends():
    """A tensor that ends inside a 16-byte group: what lies behind it stays."""
    buf = torch.full((64,), 2.0, device="cuda")
    out = torch.full((64,), 5.0, device="cuda")
    norm = GradNorm([buf[:13], buf[16:33]]).clip(1.0, out=[out[:13], out[16:33]])
    assert abs(float(norm) - 2 * math.sqrt(30)) < 1e-5
    assert (out[13:16] == 5).all() and (out[33:] == 5).all() and (out[:13] != 5).all()


def test_repeats_and_replays():
    grads = _grads([100000, 31, 7777], "f32")
    a, b = GradNorm(grads), GradNorm(grads)
    out, out2 = ([torch.empty_like(g) for g in grads] for _ in range(2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a.clip(1.0, out=out)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.clip(1.0, out=out)
    for i in range(4):
        for g in grads:
            g.copy_(torch.randn_like(g))
        b.clip(1.0, out=out2)
        for t in out:
            t.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a.result, b.result) and all(torch.equal(p, q) for p, q in zip(out, out2)), i


def test_more_elements_than_32_bits_count():
    n = (1 << 31) + 5
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[0], g[n - 1], g[1 << 31] = 3.0, 4.0, 12.0
    op = GradNorm([g])
    assert float(op.clip(6.5)) == 13.0
    want = 6.5 / (13 + 1e-6)
    got = [float(g[i]) for i in (0, n - 1, 1 << 31)]
    assert all(abs(p - q * want) <= (2.0 ** -8 + 2.0 ** -22) * q * want for p, q in zip(got, (3.0, 4.0, 12.0)))


def test_more_elements_than_one_launch_takes():
    """34 GB in bf16, the second of three tensors: its rest is scaled too, and the
    third behind it."""
    n = (1 << 34) + 2051
    grads = [torch.full((5,), 2.0, dtype=torch.bfloat16, device="cuda"),
             torch.zeros(n, dtype=torch.bfloat16, device="cuda"),
             torch.full((7,), 2.0, dtype=torch.bfloat16, device="cuda")]
    at = [0, (1 << 34) - 1, 1 << 34, n - 1]
    for i in at:
        grads[1][i] = 8.0
    op = GradNorm(grads)
    assert abs(float(op.clip(1.0)) - 304 ** 0.5) <= 2.0 ** -23 * 18
    coef = float(op.result[1])
    for g, i in [(grads[0], 0), (grads[2], 6)]:
        assert abs(float(g[i]) - 2 * coef) <= 2.0 ** -8 * 2 * coef
    for i in at:
        assert abs(float(grads[1][i]) - 8 * coef) <= 2.0 ** -8 * 8 * coef
    del grads, op, g
    torch.cuda.empty_cache()


def test_arena_clips_before_the_update():
    shapes = [("a", (16, 256)), ("b", (768, 16)), ("c", (5,))]
    arena = ParamArena(shapes, bf16_copy=True)
    g = torch.Generator().manual_seed(1)
    for _, t in arena.grad_views().items():
        t.copy_(torch.randn(t.shape, generator=g))
    before = arena.grad.clone()
    norm = arena.clip_grad_norm(1.0)
    _check([before], [arena.grad], norm, 1.0, "f32")
    assert abs(float(arena.clip_grad_norm(10.0)) - 1.0) < 1e-5
    arena.grad = torch.full_like(arena.grad, 2.0)  # another buffer
    assert abs(float(arena.clip_grad_norm(1.0)) - 2 * math.sqrt(arena.grad.numel())) < 1e-2
    arena.adam_step()


def test_the_workspace_is_only_as_large_as_asked():
    sizes = [1 << 20, 17]
    n = F.fl_grad_norm_workspace_bytes(sizes)
    ws = torch.full((n + 64,), 77, dtype=torch.uint8, device="cuda")
    grads = _grads(sizes, "f32")
    res = torch.empty(2, device="cuda")
    F.fl_grad_norm(F.FL_F32, grads, sizes, 1.0, res, ws, n)
    torch.cuda.synchronize()
    assert (ws[n:] == 77).all() and abs(float(res[0]) - _norm64(grads)) < 1e-4


def test_outputs_unlike_the_gradients_are_refused():
    """Nothing is launched: the gradients and outputs keep their values."""
    grads = [torch.ones(40, device="cuda"), torch.ones((4, 8), device="cuda")]
    op = GradNorm(grads)
    good = [torch.zeros(40, device="cuda"), torch.zeros((4, 8), device="cuda")]
    for bad in (good[:1], [good[0], good[1][:3]], [good[0], good[1].bfloat16()], [good[0], good[1].cpu()],
                [good[0], torch.zeros((8, 8), device="cuda")[:, ::2].t()], [good[0], good[0][:32]],
                [grads[1].new_zeros(40), grads[0][:32]]):
        with pytest.raises(F.FlglmError):
            op.clip(1.0, out=bad)
    torch.cuda.synchronize()
    assert all((g == 1).all() for g in grads) and all((o == 0).all() for o in good)
    op.clip(1.0, out=good)
    assert all((g == 1).all() for g in grads) and all(abs(float(o.max()) - 72 ** -0.5) < 1e-5 for o in good)


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_more_bytes_than_the_cache_holds(dt):
    """Past 1 GB, ragged sizes, into other tensors: each element the product
    rounded once."""
    unit = 4 // dt.itemsize << 20
    sizes = [200 * unit + 3, 1, 61 * unit - 2047, 2049, 8 * unit]
    gen = torch.Generator(device="cuda").manual_seed(3)
    grads = [torch.randn(n, generator=gen, device="cuda", dtype=torch.float32).to(dt) for n in sizes]
    out = [torch.full_like(g, 7.0) for g in grads]
    op = GradNorm(grads)
    op.clip(2.0, out=out)
    coef = op.result[1]
    for g, o in zip(grads, out):
        assert torch.equal(o, (g.float() * coef).to(dt))
