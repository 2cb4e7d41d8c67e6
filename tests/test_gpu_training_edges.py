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
