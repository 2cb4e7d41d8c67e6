"""Calls of the training operators at the edges of what their documentation allows, against their definitions in 64 bits."""
import math

import pytest

torch = pytest.importorskip("torch")
from test_gpu_training_ops import BOTH, EPS, HALF, STEP, Layer, _clip, _dt, _gelu64, _gen, _normal, _slope64, ctx  # noqa: E402,F401
from test_gpu_training_ops import test_layernorm_backward as check_layernorm_backward, test_layernorm_forward as check_layernorm_forward  # noqa: E402

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------ gradient clipping
@pytest.mark.parametrize("dsts", ["new", "same"])
def test_clip_of_infinite_values_by_an_infinite_bound(ctx, dsts):
    """Zeros, and no number in the infinite places, as for every other bound."""
    vit, m = ctx
    sources = [_normal(_gen(5), 40000), _normal(_gen(6), 11, dtype=torch.bfloat16)]
    sources[0][33333], sources[1][2] = math.inf, -math.inf
    norm, out = _clip(vit, m, sources, math.inf, dsts)
    assert norm.item() == math.inf
    for t, at in zip(out, (33333, 2)):
        assert t[at].isnan() and t.isnan().sum() == 1 and (t.nan_to_num(0) == 0).all()


@pytest.mark.parametrize("dsts", ["new", "same"])
def test_clip_by_a_factor_that_rounds_to_a_power_of_two(ctx, dsts):
    """The factor is 2^-100 (1 - 2^-29), below the limit of factors that fit 32 bits and equal to it when rounded."""
    vit, m = ctx
    source = torch.tensor([2.0 ** 60, 2.0 ** 46, -2.0 ** 40], device="cuda")
    norm, out = _clip(vit, m, [source.clone()], 2.0 ** -40, dsts)
    want = source.double() * (2.0 ** -40 / source.double().norm())
    assert ((out[0].double() - want).abs() <= STEP * want.abs()).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("bound,size", [(1e-37, 1e36), (1e-35, 3e34), (1e-20, 1e38), (1e-36, 1e6)])
def test_clip_of_huge_values_by_tiny_bounds(ctx, bound, size, dtype):
    """Factors far below what 32 bits hold, and results in their range: the product is rounded once, to dst's type."""
    vit, m = ctx
    sources = [(_normal(_gen(7), 5).clamp(-3, 3) * size).to(dtype) for _ in range(3)]
    sources.append(torch.tensor([size], device="cuda").to(dtype))
    norm, out = _clip(vit, m, sources, bound)
    total = math.sqrt(sum(t.double().square().sum().item() for t in sources))
    bound32 = torch.tensor(bound, dtype=torch.float32).item()
    for t, o in zip(sources, out):
        want = t.double() * (bound32 / total)
        # the norm's squares are added in 64 bits where they leave the range, and 16 at a time in 32 elsewhere: 12 steps; two roundings
        assert ((o.double() - want).abs() <= (HALF[dtype] + 14 * STEP) * want.abs() + 2.0 ** -133 * (1 if dtype == torch.bfloat16 else 2.0 ** -16)).all()
        assert (o != 0).all()
