"""Adapters, preference loss and clipping where callers share memory, streams or
tables with each other."""

import math

import numpy as np
import pytest

import synth
from tests.gpu_helpers import dev

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
from paper_2406_14898_amd import BatchDesc, ParamArena, ServerStack, StackAdapters  # noqa: E402

u = 2.0 ** -23


def _randn(*shape, seed, std=1.0, dtype=torch.float32):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * std).to(dtype).cuda()


def test_blocks_that_share_a_gradient_add_up_in_it():
    """Both blocks' adapters and their gradients in one array each: the sum of what
    separate arrays receive, but for the rounding of that sum."""
    H, r = 256, 8
    shape = synth.StackShape(num_layers=2, hidden=H, num_heads=4, ffn_hidden=512, rotary_dim=32)
    stack, batch = ServerStack(2, H, 4, 512, 32, "f32"), BatchDesc([0, 21, 50], [0, 1, 2])
    params = [{k: dev(v, "f32") for k, v in synth.layer_params(shape, l, seed=1, bf16=False).items()} for l in range(2)]
    pair = dict(a=_randn(2, r, H, seed=1, std=H ** -0.5), b=_randn(2, 3 * H, r, seed=2, std=0.05))
    x, dy = _randn(50, H, seed=3), _randn(50, H, seed=4)
    zeros = lambda: {k: torch.zeros_like(v) for k, v in pair.items()}  # noqa: E731
    shared, apart = zeros(), [zeros(), zeros()]
    for grads in ([shared, shared], apart):
        adapters = StackAdapters(stack, batch, [1, 0], [pair, pair], grads, 2.0)
        saved, ws = stack.buffers(batch, False)
        y, dx = torch.empty_like(x), torch.empty_like(x)
        stack.forward(batch, params, x, y, saved, ws, adapters=adapters)
        stack.backward(batch, params, [{}, {}], x, saved, dy, dx, ws, adapters=adapters)
    for k in ("a", "b"):
        one, two = (d[k].double() for d in apart)
        # (the second block's sums start from the first one's: 50 rows' additions)
        assert ((shared[k].double() - (one + two)).abs() <= 64 * u * (one.abs() + two.abs()) + 64 * u *
                float((one + two).abs().max())).all() and shared[k].any()
    stack.close()


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_a_bad_step_leaves_an_arena_usable(bad):
    """NaN (or infinite) gradients, clipped, the update skipped and the gradients
    cleared through their views, none of a size that fills its place: the next
    norm is that of the next gradients, and the padding is still zero."""
    arena = ParamArena([("a", (3, 7)), ("b", (16,)), ("c", (13,)), ("d", (1,))], bf16_copy=False)
    views = arena.grad_views()
    for t in views.values():
        t.fill_(1.0)
    inside = arena.grad != 0
    views["c"][5] = bad
    norm = float(arena.clip_grad_norm(1.0))
    assert math.isnan(norm) if math.isnan(bad) else norm == math.inf
    assert not arena.grad[~inside].any()
    for t in views.values():
        t.zero_()
    assert float(arena.clip_grad_norm(1.0)) == 0.0
    for t in views.values():
        t.fill_(2.0)
    want = 2 * math.sqrt(21 + 16 + 13 + 1)
    assert abs(float(arena.clip_grad_norm(1.0)) - want) <= 2.0 ** -23 * want
    # coefficient and product rounded once each
    assert ((arena.grad[inside].double() - 2 / (want + 1e-6)).abs() <= 2.0 ** -22 * 2 / want).all()
    assert not arena.grad[~inside].any()
