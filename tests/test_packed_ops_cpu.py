"""Host-side checks of the packed operators that need no GPU: size queries accept and refuse problems."""
import pytest

import paper_2110_14895_b200 as vit
from paper_2110_14895_b200 import build as vit_build


@pytest.fixture(scope="module", autouse=True)
def built():
    vit_build.build()
    vit.lib()


GOOD = dict(sequences=3, heads=4, kv_heads=2, d=64, q_rows=100, max_q=60, q_offsets=64, k_rows=90, max_k=50, k_offsets=128, scale=0.125)


def _bytes(dtype=vit.VIT_BF16, backward=True, **changed):
    return vit.vit_attention_packed_bytes(dtype, vit.make_attention_problem(**{**GOOD, **changed}), backward)


def test_backward_scratch_holds_one_float_per_query_and_head():
    for dtype in (vit.VIT_BF16, vit.VIT_FP32):
        assert _bytes(dtype) >= 4 * 100 * 4
        assert _bytes(dtype) < 4 * 100 * 4 + 4096


@pytest.mark.parametrize("changed", [dict(sequences=-1), dict(heads=0), dict(kv_heads=0), dict(kv_heads=3), dict(d=8), dict(d=40),
                                     dict(d=144), dict(q_rows=-1), dict(max_q=-1), dict(k_rows=-1), dict(max_k=-1), dict(q_offsets=0),
                                     dict(k_offsets=0), dict(q_offsets=66), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")),
                                     dict(scale=float("nan")), dict(sequences=2 ** 30, max_q=2 ** 30), dict(heads=2 ** 30, kv_heads=1)])
def test_invalid_problems_have_no_size(changed):
    assert _bytes(**changed) == 0


def test_invalid_type_has_no_size():
    assert _bytes(dtype=5) == 0
    assert vit.vit_attention_packed_bytes(vit.VIT_BF16, None, True) == 0


def test_norm_gradient_scratch():
    assert vit.vit_qk_norm_rope_backward_bytes(100, 4, 2, 64) > 0
    for args in ((-1, 4, 2, 64), (100, -1, 2, 64), (100, 4, -1, 64), (100, 4, 2, 40), (100, 4, 2, 0)):
        assert vit.vit_qk_norm_rope_backward_bytes(*args) == 0


def test_rope_needs_one_to_four_axes():
    with pytest.raises(ValueError):
        vit.make_rope((), 0, 0)
    with pytest.raises(ValueError):
        vit.make_rope((1, 1, 1, 1, 1), 0, 0)


def test_status_of_bad_offsets_has_a_text():
    assert "offsets" in vit.status_string(vit.VIT_ERR_OFFSETS)


def test_calls_without_a_handle_are_refused():
    rope = vit.make_rope((8,), 64, 64)
    problem = vit.make_attention_problem(**GOOD)
    for call in (lambda: vit.vit_op_rope_axes(None, 0, 1, 1, 64, rope, False, 256, 64, 512, 64),
                 lambda: vit.vit_op_qk_norm_rope(None, 0, 1, 1, 1, 64, 256, 256, 1e-6, rope, 256, 128, 512, 128),
                 lambda: vit.vit_op_attention_packed(None, 0, problem, 0, 256, 0, 128, 0, 128, 0, 256, 0, 0, 0)):
        with pytest.raises(vit.VitError) as e:
            call()
        assert e.value.status == vit.VIT_ERR_INVALID_ARG


ANY = 2 ** 31 - 1


@pytest.mark.parametrize("dtype", [vit.VIT_BF16, vit.VIT_FP32])
@pytest.mark.parametrize("heads,kv_heads,q_rows,k_rows", [(1, 1, 5000, 5000), (2, 1, 100, 90), (8, 2, 16388, 16388), (1, 1, 0, 7)])
def test_a_bound_beyond_the_buffers_says_what_their_rows_say(dtype, heads, kv_heads, q_rows, k_rows):
    shape = dict(dtype=dtype, sequences=1, heads=heads, kv_heads=kv_heads, q_rows=q_rows, k_rows=k_rows)
    whole = _bytes(max_q=q_rows, max_k=k_rows, **shape)
    for max_q, max_k in ((ANY, ANY), (ANY, k_rows), (q_rows, ANY), (ANY - 31, ANY - 100), (q_rows + 1, k_rows + 1)):
        assert _bytes(max_q=max_q, max_k=max_k, **shape) == whole
    assert whole > 0 or q_rows == 0
    assert _bytes(dtype=dtype, sequences=1000, heads=64, kv_heads=64, max_q=ANY, max_k=ANY) > 0


def test_rows_that_the_kernels_cannot_count_have_no_size():
    one = dict(sequences=1, heads=1, kv_heads=1, d=16, max_q=1, max_k=1)
    for rows in (ANY, ANY - 1023):
        assert _bytes(**one, q_rows=rows) == 0 and _bytes(**one, k_rows=rows) == 0
    assert _bytes(**one, q_rows=ANY - 1024, k_rows=ANY - 1024) >= 8 * (ANY - 1024)


@pytest.mark.parametrize("dtype", [vit.VIT_BF16, vit.VIT_FP32])
def test_backward_scratch_holds_two_floats_per_query_and_head(dtype):
    """Log-sum-exp and delta of every query row and head, in 32 bits each."""
    for heads, kv_heads, q_rows in ((4, 2, 100), (1, 1, 1), (12, 12, 12608), (3, 3, 2 ** 30)):
        got = _bytes(dtype, sequences=1, heads=heads, kv_heads=kv_heads, q_rows=q_rows, max_q=1, max_k=1)
        assert 8 * heads * q_rows <= got < 8 * heads * q_rows + 4096


def test_backward_scratch_holds_the_parts_of_shared_sums():
    """bf16, long sequences: 148 blocks leave two parts each, of 128 rows of dk and of dv in 32 bits."""
    rows, heads, d = 4 * 4097, 8, 128
    long = dict(sequences=4, heads=heads, kv_heads=2, d=d, q_rows=rows, max_q=4097, k_rows=rows, max_k=4097)
    assert _bytes(vit.VIT_BF16, **long) >= 8 * heads * rows + 148 * 2 * 2 * 128 * d * 4
    assert _bytes(vit.VIT_FP32, **long) < 8 * heads * rows + 4096
    assert _bytes(vit.VIT_BF16, backward=False, **long) == 0
