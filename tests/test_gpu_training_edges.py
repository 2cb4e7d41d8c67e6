"""Calls of the training operators at the edges of what their documentation allows, against their definitions in 64 bits."""
import math

import pytest

torch = pytest.importorskip("torch")
from test_gpu_training_ops import BOTH, EPS, HALF, STEP, Layer, _clip, _dt, _gelu64, _gen, _normal, _slope64, _sum_error, ctx  # noqa: E402,F401
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



# ------------------------------------------------------------------------------------ linear layers by group
@BOTH
def test_a_single_row_has_any_stride(ctx, dtype):
    """With one row, or none, nothing lies a stride further on: strides beyond what any memory holds are as good as others."""
    vit, m = ctx
    k, n, far = 72, 136, 1 << 45
    dt = _dt(vit, dtype)
    l = Layer(vit, m, [1], 0, 0, k, n, dtype)
    x, dout, residual, pre = l.some(k, k), l.some(n, n), l.some(n, n), l.some(k, k)
    calls = lambda ld: [l_forward(1, ld), l_forward(2, ld), l_input(ld), *l_weights(ld)]

    def l_forward(epilogue, ld):
        out, kept = l.blank(n), l.blank(n)
        vit.vit_op_linear_grouped(m.h, dt, l.problem, x.data_ptr(), ld or k, l.w.data_ptr(), 0, epilogue, residual.data_ptr(), ld or n, out.data_ptr(),
                                  ld or n, kept.data_ptr(), ld or n)
        return out

    def l_input(ld):
        dx = l.blank(k)
        vit.vit_op_linear_grouped_backward_input(m.h, dt, l.problem, dout.data_ptr(), ld or n, l.w.data_ptr(), pre.data_ptr(), ld or k, dx.data_ptr(), ld or k)
        return dx

    def l_weights(ld, problem=None):
        dw, db = torch.full_like(l.w, 77.0), torch.full((1, n), 77.0, device="cuda")
        size = vit.vit_linear_grouped_backward_weights_bytes(dt, problem or l.problem)
        ws = torch.empty(size, dtype=torch.uint8, device="cuda")
        vit.vit_op_linear_grouped_backward_weights(m.h, dt, problem or l.problem, x.data_ptr(), ld or k, dout.data_ptr(), ld or n, dw.data_ptr(),
                                                   db.data_ptr(), ws.data_ptr(), size)
        return dw, db

    for a, b in zip(calls(0), calls(far)):
        assert torch.equal(a, b)
    m.check()
    none = vit.make_grouped_problem(1, 0, k, n, 0)
    assert all((t == 0).all() for t in l_weights(far, none))
    m.check()


@pytest.mark.parametrize("far", [False, True])
def test_gelu_and_its_slope_in_fp32(ctx, far):
    """The error function and the exponential of the fp32 mode are CUDA's own, good to a few roundings; an approximation to 1e-7 of
    one, as the bf16 mode uses, is not."""
    vit, m = ctx
    k, rows = 64, 300
    l = Layer(vit, m, [rows], 0, 0, k, k, torch.float32)
    l.w[0] = torch.eye(k, device="cuda")
    v = _normal(l.gen, rows, k, scale=4.0 if far else 1.0)                       # products with ones and sums with zeros are exact
    a = v.double()
    # erfc is good to 4 steps (8 roundings); its argument u has two roundings, which count 2 u^2 + 1.2 times at most beyond u = 0 (u erfc'(u) / erfc(u),
    # and less than u before); three products follow
    u = a.abs() / math.sqrt(2)
    erfc = 8 + 2 * (2 * u * u + 2) + 3
    out = l.forward(v, None, 1, out=l.blank(k))
    want = _gelu64(a)
    assert ((out.double() - want).abs() <= erfc * STEP * want.abs() + 2.0 ** -140).all()
    # the exponential is good to 2 steps, its argument a^2 / 2 has a rounding; the factors before it three, the sum one
    dx = l.input_grad(torch.ones_like(v), v, l.blank(k))
    phi = a.abs() * torch.exp(-0.5 * a * a) / math.sqrt(2 * math.pi)
    want = _slope64(a)
    tol = phi * (4 + 0.5 * a * a + 3) + 0.5 * torch.erfc(-a / math.sqrt(2)) * erfc + want.abs()
    assert ((dx.double() - want).abs() <= STEP * tol + 2.0 ** -140).all()


# ------------------------------------------------------------------------------------ layer norm
# two rows to a warp from 32 to an SM on, in one to six pieces a lane (three in fp32), an odd row left over; the same with four warps to two rows
@pytest.mark.parametrize("rows,cols", [(4737, 200), (4737, 384), (4739, 768), (4999, 1000), (4741, 1024), (4801, 1280), (4736, 1536), (4735, 768),
                                       (5001, 1800), (4737, 2056), (4801, 4000)])
@BOTH
def test_layernorm_of_many_rows(ctx, rows, cols, dtype):
    check_layernorm_forward(ctx, rows, cols, dtype)
    check_layernorm_backward(ctx, rows, cols, True, dtype)


# ------------------------------------------------------------------------------------ bad offsets where clusters share the sums
@pytest.mark.parametrize("edges,rows,k,n", [([5, 3], 577, 1280, 1280), ([0, 578], 577, 1280, 1280), ([-1, 577], 577, 1280, 1024), ([0, 90, 60, 97], 97, 4096, 1544),
                                            ([0, 2 ** 31 - 1, 5, 33], 33, 2048, 1536)], ids=lambda v: "-".join(map(str, v)) if isinstance(v, list) else str(v))
@BOTH
def test_bad_offsets_of_few_tiles(ctx, edges, rows, k, n, dtype):
    """Long sums of few tiles, forwards, backwards and of the weights: bad groups are left as they were and reported, the others are right."""
    vit, m = ctx
    groups = len(edges) - 1
    good = [g for g in range(groups) if 0 <= edges[g] <= edges[g + 1] <= rows]
    dt = _dt(vit, dtype)
    gen = _gen(rows + k)
    x, dout = _normal(gen, rows, k, dtype=dtype), _normal(gen, rows, n, dtype=dtype)
    w = _normal(gen, groups, n, k, scale=k ** -0.5, dtype=dtype)
    off = torch.tensor(edges, dtype=torch.int32, device="cuda")
    p = vit.make_grouped_problem(groups, rows, k, n, off.data_ptr())
    out, dx = torch.full_like(dout, 77.0), torch.full_like(x, 77.0)
    dw, db = torch.full_like(w, 777.0), torch.full((groups, n), 777.0, device="cuda")
    size = vit.vit_linear_grouped_backward_weights_bytes(dt, p)
    ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
    for call in (lambda: vit.vit_op_linear_grouped(m.h, dt, p, x.data_ptr(), k, w.data_ptr(), 0, 0, 0, 0, out.data_ptr(), n, 0, 0),
                 lambda: vit.vit_op_linear_grouped_backward_input(m.h, dt, p, dout.data_ptr(), n, w.data_ptr(), 0, 0, dx.data_ptr(), k),
                 lambda: vit.vit_op_linear_grouped_backward_weights(m.h, dt, p, x.data_ptr(), k, dout.data_ptr(), n, dw.data_ptr(), db.data_ptr(),
                                                                    ws.data_ptr(), size)):
        call()
        with pytest.raises(vit.VitError) as e:
            m.check()
        assert e.value.status == vit.VIT_ERR_OFFSETS
    owners = torch.zeros(rows, dtype=torch.int32, device="cuda")
    for g in good:
        owners[edges[g]:edges[g + 1]] += 1
    assert (out[owners == 0] == 77).all() and (dx[owners == 0] == 77).all()
    for g in range(groups):
        b, e = edges[g], edges[g + 1]
        if g not in good:
            assert (dw[g] == 777).all() and (db[g] == 777).all()
            continue
        own = (owners[b:e] == 1)[:, None]
        xs, ds, wg = x[b:e].double(), dout[b:e].double(), w[g].double()
        for got, want, terms, length in ((out[b:e], xs @ wg.t(), xs.abs() @ wg.abs().t(), k), (dx[b:e], ds @ wg, ds.abs() @ wg.abs(), n)):
            assert (((got.double() - want).abs() <= HALF[dtype] * want.abs() + (_sum_error(length, dtype) + 8 * STEP) * terms) | ~own).all()
        want, terms = ds.t() @ xs, ds.abs().t() @ xs.abs()
        assert ((dw[g].double() - want).abs() <= HALF[dtype] * want.abs() + (_sum_error(e - b, dtype) + 8 * STEP) * terms).all()
        assert ((db[g].double() - ds.sum(0)).abs() <= ((e - b) / 16 + 32) * STEP * ds.abs().sum(0)).all()
