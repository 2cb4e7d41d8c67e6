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


def test_lists_of_tensors_keep_their_entries():
    t = vit.make_tensors([(16, 32, 5, vit.VIT_BF16), (48, 0, 2 ** 40, vit.VIT_FP32)])
    assert (t[0].src, t[0].dst, t[0].count, t[0].dtype) == (16, 32, 5, 0)
    assert (t[1].src, t[1].dst, t[1].count, t[1].dtype) == (48, None, 2 ** 40, 1)
    vit.make_tensors([])


def test_calls_without_a_handle_are_refused():
    tensors = vit.make_tensors([(64, 64, 4, 1)])
    for call in (lambda: vit.vit_op_layernorm_forward(None, 0, 1, 64, 256, 64, 512, 768, 1e-6, 1024, 64, 0),
                 lambda: vit.vit_op_layernorm_backward(None, 0, 1, 64, 256, 64, 512, 768, 1024, 64, 0, 64, 2048, 64, 4096, 8192, 16384, 1 << 20),
                 lambda: vit.vit_op_grad_clip(None, tensors, 1, 1.0, 256, 512, 1 << 20)):
        with pytest.raises(vit.VitError) as e:
            call()
        assert e.value.status == vit.VIT_ERR_INVALID_ARG
