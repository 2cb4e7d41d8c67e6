"""Host-side checks of the training operators that need no GPU: size queries and refusals without a handle."""
import pytest

import paper_2110_14895_b200 as vit
from paper_2110_14895_b200 import build as vit_build


@pytest.fixture(scope="module", autouse=True)
def built():
    vit_build.build()
    vit.lib()


def test_layernorm_scratch():
    assert vit.vit_layernorm_backward_bytes(100, 64) >= 2 * 64 * 4
    assert vit.vit_layernorm_backward_bytes(0, 8) > 0
    assert vit.vit_layernorm_backward_bytes(2 ** 31 - 1, 8192) < 2 ** 26
    for rows, cols in ((-1, 64), (1, 0), (1, 4), (1, 60), (1, 8200), (1, -8)):
        assert vit.vit_layernorm_backward_bytes(rows, cols) == 0


def test_clip_scratch():
    assert vit.vit_grad_clip_bytes(-1) == 0
    sizes = [vit.vit_grad_clip_bytes(n) for n in (0, 1, 960, 961, 5000)]
    assert all(n > 0 and n % 16 == 0 for n in sizes) and sizes == sorted(sizes) and sizes[3] > sizes[2]


GOOD = dict(groups=4, rows=1000, in_features=256, out_features=512, offsets=64)


def _bytes(dtype=vit.VIT_BF16, **changed):
    return vit.vit_linear_grouped_backward_weights_bytes(dtype, vit.make_grouped_problem(**{**GOOD, **changed}))


@pytest.mark.parametrize("dtype", [vit.VIT_BF16, vit.VIT_FP32])
def test_weight_gradient_scratch(dtype):
    assert _bytes(dtype) > 0 and _bytes(dtype, rows=0) > 0 and _bytes(dtype, groups=1, offsets=0) > 0
    assert _bytes(dtype, rows=10 ** 6, in_features=4096, out_features=4096) < 2 ** 27
    for changed in (dict(groups=0), dict(groups=-3), dict(rows=-1), dict(in_features=0), dict(in_features=12), dict(out_features=4), dict(offsets=0),
                    dict(offsets=66), dict(rows=2 ** 31 - 1), dict(groups=2 ** 31 - 1), dict(in_features=2 ** 31 - 8, out_features=2 ** 31 - 8)):
        assert _bytes(dtype, **changed) == 0


def test_weight_gradient_scratch_of_no_problem():
    assert vit.vit_linear_grouped_backward_weights_bytes(vit.VIT_BF16, None) == 0
    assert _bytes(dtype=7) == 0


def test_lists_of_tensors_keep_their_entries():
    t = vit.make_tensors([(16, 32, 5, vit.VIT_BF16), (48, 0, 2 ** 40, vit.VIT_FP32)])
    assert (t[0].src, t[0].dst, t[0].count, t[0].dtype) == (16, 32, 5, 0)
    assert (t[1].src, t[1].dst, t[1].count, t[1].dtype) == (48, None, 2 ** 40, 1)
    vit.make_tensors([])


def test_calls_without_a_handle_are_refused():
    tensors = vit.make_tensors([(64, 64, 4, 1)])
    for call in (lambda: vit.vit_op_layernorm_forward(None, 0, 1, 64, 256, 64, 512, 768, 1e-6, 1024, 64, 0),
                 lambda: vit.vit_op_layernorm_backward(None, 0, 1, 64, 256, 64, 512, 768, 1024, 64, 0, 64, 2048, 64, 4096, 8192, 16384, 1 << 20),
                 lambda: vit.vit_op_linear_grouped(None, 0, vit.make_grouped_problem(**GOOD), 256, 256, 512, 0, 0, 0, 0, 1024, 512, 0, 0),
                 lambda: vit.vit_op_linear_grouped_backward_input(None, 0, vit.make_grouped_problem(**GOOD), 256, 512, 512, 0, 0, 1024, 256),
                 lambda: vit.vit_op_linear_grouped_backward_weights(None, 0, vit.make_grouped_problem(**GOOD), 256, 256, 512, 512, 1024, 0, 64, 1 << 30),
                 lambda: vit.vit_op_grad_clip(None, tensors, 1, 1.0, 256, 512, 1 << 20)):
        with pytest.raises(vit.VitError) as e:
            call()
        assert e.value.status == vit.VIT_ERR_INVALID_ARG
