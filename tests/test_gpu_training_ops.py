"""Operators that training a layer needs (layer norm, linear layers by group, their gradients, gradient clipping) against
their definitions in 64 bits, called through the C boundary."""
import math

import pytest

import vitgen

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}      # half a step of the type, relative
STEP = 2.0 ** -24                                                  # one rounding in 32 bits
EPS = 1e-6
BOTH = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])


@pytest.fixture(scope="module")
def ctx():
    import paper_2110_14895_b200 as vit
    shape = vitgen.preset("tiny16").with_(layers=1)
    _, blob = vitgen.make_params(shape, seed=0)
    m = vit.VitModel(shape, blob, vit.VIT_BF16, 1)
    yield vit, m
    m.check()
    m.close()


def _dt(vit, dtype):
    return vit.VIT_BF16 if dtype == torch.bfloat16 else vit.VIT_FP32


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(gen, *shape, scale=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=gen, device="cuda") * scale).to(dtype)


def _refused(vit, call, status=None):
    with pytest.raises(vit.VitError) as e:
        call()
    assert e.value.status == (vit.VIT_ERR_INVALID_ARG if status is None else status)


# ------------------------------------------------------------------------------------ layer norm
NORM_SHAPES = [(1, 8), (3, 16), (197, 192), (7, 248), (33, 256), (50, 264), (197, 384), (1531, 768), (40, 776), (64, 1024), (257, 1280),
               (29, 1544), (130, 2048), (5, 2056), (31, 4096), (17, 4104), (9, 8192), (5000, 64), (2000, 1024)]


def _norm_rows(gen, rows, cols, ld, dtype):
    """Rows with sizes and offsets of their own in a wider buffer; what lies behind the columns is not a number."""
    x = torch.full((rows, ld), float("nan"), dtype=dtype, device="cuda")
    x[:, :cols] = (_normal(gen, rows, cols) * (0.1 + _normal(gen, rows, 1).abs()) + _normal(gen, rows, 1)).to(dtype)
    return x


def _forward(vit, m, x, cols, gain, shift, ldy, with_stats=True):
    rows = x.shape[0]
    y = torch.full((rows, ldy), 77.0, dtype=x.dtype, device="cuda")
    stats = torch.full((rows, 2), 77.0, device="cuda")
    vit.vit_op_layernorm_forward(m.h, _dt(vit, x.dtype), rows, cols, x.data_ptr(), x.stride(0), gain.data_ptr(), shift.data_ptr(), EPS,
                                 y.data_ptr(), ldy, stats.data_ptr() if with_stats else 0)
    m.check()
    return y, stats


@pytest.mark.parametrize("rows,cols", NORM_SHAPES)
@BOTH
def test_layernorm_forward(ctx, rows, cols, dtype):
    vit, m = ctx
    gen = _gen(rows + cols)
    x = _norm_rows(gen, rows, cols, cols + 8, dtype)
    gain, shift = 1 + _normal(gen, cols, scale=0.2), _normal(gen, cols, scale=0.2)
    y, stats = _forward(vit, m, x, cols, gain, shift, cols + 16)
    x64 = x[:, :cols].double()
    mean, var = x64.mean(1, keepdim=True), x64.var(1, unbiased=False, keepdim=True)
    rstd = 1 / (var + EPS).sqrt()
    z = (x64 - mean) * rstd
    want = z * gain.double() + shift.double()
    # a row's sums are chains of at most 64 values and 10 joins: 80 roundings of the mean size; the deviation from the
    # rounded mean counts twice in the variance, in second order
    off = 80 * STEP * x64.abs().mean(1, keepdim=True)
    rel = 48 * STEP + (off * rstd) ** 2
    assert ((stats[:, :1].double() - mean).abs() <= off + STEP * mean.abs()).all()
    assert ((stats[:, 1:].double() - rstd).abs() <= rel * rstd).all()
    tol = HALF[dtype] * want.abs() + ((off + 2 * STEP * x64.abs()) * rstd + (rel + 4 * STEP) * z.abs()) * gain.double().abs() + 2 * STEP * want.abs()
    assert ((y[:, :cols].double() - want).abs() <= tol).all()
    assert (y[:, cols:] == 77).all()
    # without statistics and in place: the same bits
    again, untouched = _forward(vit, m, x, cols, gain, shift, cols + 16, with_stats=False)
    assert torch.equal(again, y) and (untouched == 77).all()
    z = x.clone()
    vit.vit_op_layernorm_forward(m.h, _dt(vit, dtype), rows, cols, z.data_ptr(), cols + 8, gain.data_ptr(), shift.data_ptr(), EPS,
                                 z.data_ptr(), cols + 8, 0)
    m.check()
    assert torch.equal(z[:, :cols], y[:, :cols])


def _backward(vit, m, x, cols, gain, stats, dy, dres, lddx, into=None):
    rows = x.shape[0]
    dx = torch.full((rows, lddx), 77.0, dtype=x.dtype, device="cuda") if into is None else into
    grads = torch.full((2, cols), 77.0, device="cuda")
    n = vit.vit_layernorm_backward_bytes(rows, cols)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")                # not a number, if read before it is written
    vit.vit_op_layernorm_backward(m.h, _dt(vit, x.dtype), rows, cols, x.data_ptr(), x.stride(0), gain.data_ptr(), stats.data_ptr(),
                                  dy.data_ptr(), dy.stride(0), dres.data_ptr() if dres is not None else 0,
                                  dres.stride(0) if dres is not None else 0, dx.data_ptr(), dx.stride(0), grads[0].data_ptr(),
                                  grads[1].data_ptr(), ws.data_ptr(), n)
    m.check()
    return dx, grads


@pytest.mark.parametrize("rows,cols", NORM_SHAPES)
@pytest.mark.parametrize("residual", [False, True])
@BOTH
def test_layernorm_backward(ctx, rows, cols, residual, dtype):
    vit, m = ctx
    gen = _gen(rows * 3 + cols)
    x = _norm_rows(gen, rows, cols, cols + 8, dtype)
    gain, shift = 1 + _normal(gen, cols, scale=0.2), torch.zeros(cols, device="cuda")
    stats = _forward(vit, m, x, cols, gain, shift, cols)[1]
    dy, dres = _normal(gen, rows, cols + 24, scale=0.7, dtype=dtype), _normal(gen, rows, cols + 40, dtype=dtype) if residual else None
    dx, grads = _backward(vit, m, x, cols, gain, stats, dy, dres, cols + 16)
    x64, dy64, g64 = x[:, :cols].double(), dy[:, :cols].double(), gain.double()
    mean, rstd = stats[:, :1].double(), stats[:, 1:].double()                   # as given: their rounding is the forward's
    z, w = (x64 - mean) * rstd, dy64 * g64
    c1, c2 = w.mean(1, keepdim=True), (w * z).mean(1, keepdim=True)
    want = rstd * (w - c1 - z * c2) + (dres[:, :cols].double() if residual else 0)
    size = lambda t: t.abs().mean(1, keepdim=True)
    z_off = 2 * STEP * (x64.abs() + mean.abs()) * rstd
    c2_off = 84 * STEP * size(w * z) + (w.abs() * z_off).mean(1, keepdim=True)
    tol = HALF[dtype] * want.abs() + 2 * STEP * want.abs() + rstd * (
        4 * STEP * (w.abs() + c1.abs() + (z * c2).abs()) + 84 * STEP * size(w) + z_off * c2.abs() + z.abs() * c2_off)
    assert ((dx[:, :cols].double() - want).abs() <= tol).all()
    assert (dx[:, cols:] == 77).all()
    # chains over the rows of a block (at least 148 rows at a time, or all of them), its warps and the blocks
    chain = rows // 148 + 64
    for got, terms, more in ((grads[0], dy64 * z, (dy64.abs() * z_off).sum(0)), (grads[1], dy64, 0)):
        assert ((got.double() - terms.sum(0)).abs() <= chain * STEP * terms.abs().sum(0) + more).all()
    # in place of any of the three operands, and once more: the same bits
    for name, t in (("x", x), ("dy", dy), ("dres", dres)):
        if t is None:
            continue
        own = t.clone()
        again, more = _backward(vit, m, own if name == "x" else x, cols, gain, stats, own if name == "dy" else dy,
                                own if name == "dres" else dres, 0, into=own)
        assert torch.equal(again[:, :cols], dx[:, :cols]) and torch.equal(more, grads), name


def test_layernorm_gradients_against_differences(ctx):
    """The kernels' gradients against differences of the 64-bit forward pass."""
    vit, m = ctx
    gen = _gen(11)
    rows, cols = 5, 40
    x, gain, shift = _normal(gen, rows, cols), 1 + _normal(gen, cols, scale=0.2), _normal(gen, cols)
    dy = _normal(gen, rows, cols)
    stats = _forward(vit, m, x, cols, gain, shift, cols)[1]
    dx, grads = _backward(vit, m, x, cols, gain, stats, dy, None, cols)

    def loss(x, g, b):
        z = (x - x.mean(1, keepdim=True)) / (x.var(1, unbiased=False, keepdim=True) + EPS).sqrt()
        return ((z * g + b) * dy.double()).sum()

    operands = [x.double(), gain.double(), shift.double()]
    for i, got in enumerate((dx, grads[0], grads[1])):
        for at in range(0, operands[i].numel(), 7):
            sides = []
            for h in (1e-5, -1e-5):
                moved = [t.clone() for t in operands]
                moved[i].view(-1)[at] += h
                sides.append(loss(*moved))
            difference = ((sides[0] - sides[1]) / 2e-5).item()
            # differences: third derivatives times 1e-10, and 2^-52 of the loss over the step
            assert abs(got.reshape(-1)[at].item() - difference) <= 2e-5 * (1 + abs(difference))


def test_layernorm_without_rows(ctx):
    vit, m = ctx
    g = torch.ones(64, device="cuda")
    vit.vit_op_layernorm_forward(m.h, vit.VIT_BF16, 0, 64, 0, 64, g.data_ptr(), g.data_ptr(), EPS, 0, 64, 0)
    grads = torch.full((2, 64), 77.0, device="cuda")
    n = vit.vit_layernorm_backward_bytes(0, 64)
    ws = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
    vit.vit_op_layernorm_backward(m.h, vit.VIT_BF16, 0, 64, 0, 64, g.data_ptr(), 0, 0, 64, 0, 64, 0, 64, grads[0].data_ptr(),
                                  grads[1].data_ptr(), ws.data_ptr(), n)
    m.check()
    assert (grads == 0).all()


@BOTH
def test_layernorm_rows_do_not_mix(ctx, dtype):
    """A row of NaN, infinities or equal values changes no other row; equal values give the shift and finite gradients."""
    vit, m = ctx
    gen = _gen(4)
    rows, cols = 61, 320
    x = _normal(gen, rows, cols, dtype=dtype)
    gain, shift = 1 + _normal(gen, cols, scale=0.2), _normal(gen, cols)
    y, stats = _forward(vit, m, x, cols, gain, shift, cols)
    dy = _normal(gen, rows, cols, dtype=dtype)
    dx, _ = _backward(vit, m, x, cols, gain, stats, dy, None, cols)
    bad = x.clone()
    bad[3], bad[10, 5], bad[20] = float("nan"), float("inf"), 2.5
    y2, stats2 = _forward(vit, m, bad, cols, gain, shift, cols)
    dx2, grads2 = _backward(vit, m, bad, cols, gain, stats2, dy, None, cols)
    same = torch.ones(rows, dtype=torch.bool, device="cuda")
    same[[3, 10, 20]] = False
    assert torch.equal(y2[same], y[same]) and torch.equal(stats2[same], stats[same]) and torch.equal(dx2[same], dx[same])
    assert y2[3].isnan().all() and torch.equal(y2[20], shift.to(dtype)) and dx2[20].isfinite().all()
    assert grads2[0].isnan().all() and grads2[1].isfinite().all()


def test_layernorm_refusals(ctx):
    vit, m = ctx
    x, dy, dx, dres = (torch.zeros(8, 64, dtype=torch.bfloat16, device="cuda") for _ in range(4))
    gain, shift, dgain, dshift = (torch.ones(64, device="cuda") for _ in range(4))
    stats = torch.zeros(8, 2, device="cuda")
    n = vit.vit_layernorm_backward_bytes(8, 64)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    forward = dict(h=m.h, dtype=0, rows=8, cols=64, x=x.data_ptr(), ldx=64, gain=gain.data_ptr(), shift=shift.data_ptr(), eps=EPS,
                   y=dx.data_ptr(), ldy=64, stats=stats.data_ptr())
    backward = dict(h=m.h, dtype=0, rows=8, cols=64, x=x.data_ptr(), ldx=64, gain=gain.data_ptr(), stats=stats.data_ptr(),
                    dy=dy.data_ptr(), lddy=64, dres=dres.data_ptr(), lddres=64, dx=dx.data_ptr(), lddx=64, dgain=dgain.data_ptr(),
                    dshift=dshift.data_ptr(), ws=ws.data_ptr(), ws_bytes=n)
    before = m.launches
    for bad in (dict(h=None), dict(dtype=2), dict(rows=-1), dict(cols=0), dict(cols=60), dict(cols=8200), dict(x=0), dict(ldx=56), dict(ldx=68),
                dict(x=x.data_ptr() + 2), dict(gain=0), dict(gain=gain.data_ptr() + 4), dict(shift=0), dict(eps=-1.0), dict(eps=float("nan")),
                dict(y=0), dict(ldy=60), dict(y=x.data_ptr() + 128), dict(x=dx.data_ptr(), ldx=72), dict(stats=x.data_ptr()),
                dict(stats=gain.data_ptr()), dict(y=shift.data_ptr()), dict(stats=stats.data_ptr() + 8)):
        _refused(vit, lambda: vit.vit_op_layernorm_forward(**{**forward, **bad}))
    for bad in (dict(h=None), dict(dtype=2), dict(rows=-1), dict(cols=60), dict(x=0), dict(dy=0), dict(dx=0), dict(stats=0), dict(ws=0),
                dict(dgain=0), dict(dshift=0), dict(lddy=32), dict(lddres=60), dict(lddx=65), dict(dx=x.data_ptr() + 128),
                dict(dx=dres.data_ptr(), lddx=72), dict(dgain=dshift.data_ptr()), dict(dgain=gain.data_ptr()), dict(dgain=stats.data_ptr()),
                dict(ws=dy.data_ptr()), dict(ws=ws.data_ptr() + 8), dict(dshift=dx.data_ptr())):
        _refused(vit, lambda: vit.vit_op_layernorm_backward(**{**backward, **bad}))
    _refused(vit, lambda: vit.vit_op_layernorm_backward(**{**backward, "ws_bytes": n - 1}), vit.VIT_ERR_WORKSPACE)
    assert m.launches == before
    vit.vit_op_layernorm_forward(**forward)
    vit.vit_op_layernorm_backward(**backward)
    m.check()
    assert m.launches == before + 3


# ------------------------------------------------------------------------------------ gradient clipping
def _clip(vit, m, sources, bound, dsts="new", stream=0):
    """sources: tensors; dsts: "new", "same" or "none".  Returns the norm and the scaled tensors."""
    out = [torch.full_like(t, 77.0) for t in sources] if dsts == "new" else sources if dsts == "same" else [None] * len(sources)
    tensors = vit.make_tensors([(t.data_ptr(), o.data_ptr() if o is not None else 0, t.numel(), _dt(vit, t.dtype)) for t, o in zip(sources, out)])
    norm = torch.full((1,), 77.0, device="cuda")
    n = vit.vit_grad_clip_bytes(len(sources))
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    vit.vit_op_grad_clip(m.h, tensors, len(sources), bound, norm.data_ptr(), ws.data_ptr(), n, stream)
    m.check()
    return norm, out


def _check_clip(sources, bound, norm, out):
    want = math.sqrt(sum(t.double().square().sum().item() for t in sources))
    # 16 squares are added in 32 bits: 17 roundings, half of them in the root; the result and the factor are rounded too
    assert abs(norm.item() - want) <= 12 * STEP * want
    by = min(1.0, bound / want) if want > 0 else 1.0
    for t, o in zip(sources, out):
        if o is not None:
            assert ((o.double() - t.double() * by).abs() <= (HALF[t.dtype] + 12 * STEP) * (t.double() * by).abs() + 2.0 ** -134).all()


CLIP_LISTS = [[1], [8], [4096], [4097], [3], [0, 5, 0, 0, 12289, 0], [7, 100003, 64, 1], [1 << 22, 3, 1 << 20], list(range(1, 41)),
              [33] * 200, [130] * 500, [5, 4099] * 481, [17] * 2500]


@pytest.mark.parametrize("sizes", CLIP_LISTS, ids=lambda s: "%dx%d" % (len(s), max(s)))
@pytest.mark.parametrize("kind", ["bf16", "fp32", "mixed"])
def test_grad_clip(ctx, sizes, kind):
    vit, m = ctx
    gen = _gen(len(sizes))
    types = [torch.bfloat16 if kind == "bf16" or (kind == "mixed" and i % 3) else torch.float32 for i in range(len(sizes))]
    sources = [_normal(gen, n, scale=0.02, dtype=t) for n, t in zip(sizes, types)]
    kept = [t.clone() for t in sources]
    for bound in (0.01, 1e9):
        norm, out = _clip(vit, m, sources, bound)
        _check_clip(sources, bound, norm, out)
        if bound > 1:
            assert all(torch.equal(a, b) for a, b in zip(sources, out))
        again = _clip(vit, m, sources, bound)
        assert torch.equal(norm, again[0]) and all(torch.equal(a, b) for a, b in zip(out, again[1]))
        assert all(torch.equal(a, b) for a, b in zip(sources, kept))
    norm, out = _clip(vit, m, sources, 0.01)
    alone = _clip(vit, m, sources, 0.01, "none")[0]
    assert torch.equal(alone, norm) and all(torch.equal(a, b) for a, b in zip(sources, kept))
    _clip(vit, m, sources, 0.01, "same")
    assert all(torch.equal(a, b) for a, b in zip(sources, out))


@pytest.mark.parametrize("size", [1e-44, 1e-30, 1e-22, 1e15, 1e25, 3e37])
def test_grad_clip_of_values_whose_squares_leave_the_range(ctx, size):
    vit, m = ctx
    sources = [(_normal(_gen(1), n) * size) for n in (5000, 77)]
    sources.append(_normal(_gen(2), 300) * size)
    norm, out = _clip(vit, m, sources, 1e-3)
    want = math.sqrt(sum(t.double().square().sum().item() for t in sources))
    # at 3e37 the norm of 5377 values is 2e39: beyond the largest fp32 value, 2^128 (1 - 2^-24), and infinite in 32 bits
    assert abs(norm.item() - want) <= 12 * STEP * want + 2.0 ** -149 if want < 3.4e38 else norm.item() == math.inf
    by = min(1.0, 1e-3 / want)
    for t, o in zip(sources, out):
        assert ((o.double() - t.double() * by).abs() <= 16 * STEP * (t.double() * by).abs() + 2.0 ** -148 * max(1.0, size)).all()


def test_grad_clip_edges(ctx):
    vit, m = ctx
    # nothing, nothing but zeros, a bound of zero and of infinity
    norm, _ = _clip(vit, m, [], 1.0)
    assert norm.item() == 0
    zeros = [torch.zeros(5000, device="cuda"), torch.zeros(3, dtype=torch.bfloat16, device="cuda")]
    norm, out = _clip(vit, m, zeros, 0.0)
    assert norm.item() == 0 and all((t == 0).all() for t in out)
    some = [_normal(_gen(3), 6000), _normal(_gen(4), 11, dtype=torch.bfloat16)]
    norm, out = _clip(vit, m, some, 0.0)
    assert all((t == 0).all() for t in out)
    norm, out = _clip(vit, m, some, float("inf"))
    assert all(torch.equal(a, b) for a, b in zip(some, out))
    # an infinite norm: zeros, and no number in the infinite place; no number anywhere: no number everywhere
    wild = [t.clone() for t in some]
    wild[0][4999] = float("-inf")
    norm, out = _clip(vit, m, wild, 1.0)
    assert norm.item() == math.inf and out[0][4999].isnan() and (out[0].nan_to_num(0) == 0).all() and (out[1] == 0).all()
    wild[1][10] = float("nan")
    norm, out = _clip(vit, m, wild, 1.0)
    assert norm.isnan().all() and all(t.isnan().all() for t in out)
    # norm may be left out; a tensor without a dst only counts
    t = vit.make_tensors([(some[0].data_ptr(), 0, 6000, vit.VIT_FP32), (some[1].data_ptr(), out[1].data_ptr(), 11, vit.VIT_BF16)])
    n = vit.vit_grad_clip_bytes(2)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    vit.vit_op_grad_clip(m.h, t, 2, 1.0, 0, ws.data_ptr(), n)
    m.check()
    norm, both = _clip(vit, m, some, 1.0)
    assert torch.equal(out[1], both[1])


def test_grad_clip_refusals(ctx):
    vit, m = ctx
    a, b, c = (torch.zeros(64, device="cuda") for _ in range(3))
    norm = torch.zeros(4, device="cuda")
    n = vit.vit_grad_clip_bytes(2)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    A, B, C = a.data_ptr(), b.data_ptr(), c.data_ptr()

    def call(entries, count=None, bound=1.0, norm=norm.data_ptr(), ws=ws.data_ptr(), ws_bytes=n, h=m.h):
        vit.vit_op_grad_clip(h, vit.make_tensors(entries), len(entries) if count is None else count, bound, norm, ws, ws_bytes)

    good = [(A, A, 64, 1), (B, C, 64, 1)]
    before = m.launches
    for entries in ([(A, B, 64, 1), (B, C, 64, 1)], [(A, C, 64, 1), (B, C, 64, 1)], [(A, A, 64, 1), (A, A, 64, 1)], [(A, A + 16, 32, 1)],
                    [(A, A, 64, 1), (A, 0, 64, 1)], [(A, B, 64, 2)], [(A, B, -1, 1)], [(0, B, 64, 1)], [(A + 4, B, 8, 1)], [(A, B + 2, 8, 0)],
                    [(A, norm.data_ptr(), 4, 1)], [(A, ws.data_ptr(), 4, 1)], [(A, B, 2 ** 40 + 1, 1)]):
        _refused(vit, lambda: call(entries))
    for bad in (dict(h=None), dict(count=-1), dict(bound=-1.0), dict(bound=float("nan")), dict(norm=norm.data_ptr() + 4), dict(ws=0),
                dict(ws=ws.data_ptr() + 8), dict(norm=A), dict(ws=B)):
        _refused(vit, lambda: call(good, **bad))
    _refused(vit, lambda: call(good, ws_bytes=n - 1), vit.VIT_ERR_WORKSPACE)
    assert m.launches == before
    call(good)
    call([(A, 0, 64, 1), (A, 0, 64, 1)])                   # read twice, written nowhere
    m.check()
    assert m.launches == before + 4
