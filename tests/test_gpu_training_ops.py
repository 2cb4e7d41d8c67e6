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


# ------------------------------------------------------------------------------------ linear layers by group
LAYERS = [
    # lengths of the groups, rows before the first and behind the last, in, out
    ([1], 0, 0, 8, 8), ([5], 0, 0, 16, 24), ([130], 2, 3, 64, 64), ([0, 7, 0, 0, 1], 1, 9, 72, 40), ([127, 128, 129], 0, 1, 136, 264),
    ([256, 257, 31, 32, 33], 5, 5, 200, 328), ([64, 63, 65, 0, 15, 16, 17], 0, 0, 128, 256), ([1000], 0, 7, 192, 768), ([40] * 70, 3, 0, 48, 96),
    ([3000, 0, 500, 1], 0, 0, 256, 512), ([700, 900], 11, 0, 1024, 64), ([0, 0], 0, 4, 64, 64), ([1, 1, 1, 1], 0, 0, 640, 8),
    ([9000], 0, 0, 64, 128), ([2500, 2500, 2500], 1, 1, 512, 1288), ([6400], 0, 0, 1280, 1280),
    # long sums with few tiles, forwards or backwards
    ([1], 0, 0, 4096, 72), ([5, 0, 130, 1], 2, 3, 1544, 200), ([33], 0, 0, 64, 2056), ([1, 2, 300], 0, 1, 136, 1600), ([129], 0, 0, 1536, 1536),
]
LAYER_CASES = pytest.mark.parametrize("lengths,before,behind,k,n", LAYERS, ids=lambda v: "%dx%d" % (len(v), max(v)) if isinstance(v, list) else str(v))


class Layer:
    """Rows in groups with rows of nobody around them, which hold no numbers."""

    def __init__(self, vit, m, lengths, before, behind, k, n, dtype, seed=0):
        self.vit, self.m, self.k, self.n, self.dtype = vit, m, k, n, dtype
        self.gen = _gen(sum(lengths) + 31 * k + n + seed)
        self.rows, self.lengths, self.first = before + sum(lengths) + behind, lengths, before
        edges = [before]
        for length in lengths:
            edges.append(edges[-1] + length)
        self.spans = list(zip(edges, edges[1:]))
        self.offsets = torch.tensor(edges, dtype=torch.int32, device="cuda")
        self.covered = torch.zeros(self.rows, dtype=torch.bool, device="cuda")
        self.covered[before:edges[-1]] = True
        self.w = _normal(self.gen, len(lengths), n, k, scale=k ** -0.5, dtype=dtype)
        self.problem = vit.make_grouped_problem(len(lengths), self.rows, k, n, self.offsets.data_ptr())

    def some(self, width, ld, scale=1.0):
        t = torch.full((self.rows, ld), float("nan"), dtype=self.dtype, device="cuda")
        values = _normal(self.gen, self.rows, width, scale=scale, dtype=self.dtype)
        t[self.covered, :width] = values[self.covered]
        return t

    def blank(self, ld):
        return torch.full((self.rows, ld), 77.0, dtype=self.dtype, device="cuda")

    def forward(self, x, bias=None, epilogue=0, residual=None, out=None, pre=None, w=None):
        p = lambda t: t.data_ptr() if t is not None else 0
        ld = lambda t: t.stride(0) if t is not None else 0
        self.vit.vit_op_linear_grouped(self.m.h, _dt(self.vit, self.dtype), self.problem, p(x), x.stride(0), p(self.w if w is None else w), p(bias),
                                       epilogue, p(residual), ld(residual), p(out), out.stride(0), p(pre), ld(pre))
        self.m.check()
        return out

    def input_grad(self, dout, pre, dx):
        self.vit.vit_op_linear_grouped_backward_input(self.m.h, _dt(self.vit, self.dtype), self.problem, dout.data_ptr(), dout.stride(0),
                                                      self.w.data_ptr(), pre.data_ptr() if pre is not None else 0,
                                                      pre.stride(0) if pre is not None else 0, dx.data_ptr(), dx.stride(0))
        self.m.check()
        return dx

    def weight_grads(self, x, dout, bias=True, problem=None):
        problem = problem or self.problem
        dw = torch.full((len(self.lengths), self.n, self.k), 77.0, dtype=self.dtype, device="cuda")
        db = torch.full((len(self.lengths), self.n), 77.0, device="cuda") if bias else None
        size = self.vit.vit_linear_grouped_backward_weights_bytes(_dt(self.vit, self.dtype), problem)
        ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
        self.vit.vit_op_linear_grouped_backward_weights(self.m.h, _dt(self.vit, self.dtype), problem, x.data_ptr(), x.stride(0),
                                                        dout.data_ptr(), dout.stride(0), dw.data_ptr(), db.data_ptr() if bias else 0,
                                                        ws.data_ptr(), size)
        self.m.check()
        return dw, db

    def products(self, a, transposed):
        """Each row times its group's weights (or their transpose) in 64 bits, and the sums of the terms' sizes."""
        width = self.k if transposed else self.n
        out, size = (torch.full((self.rows, width), 77.0, dtype=torch.float64, device="cuda") for _ in range(2))
        for g, (b, e) in enumerate(self.spans):
            w = self.w[g].double() if transposed else self.w[g].double().t()
            out[b:e], size[b:e] = a[b:e].double() @ w, a[b:e].double().abs() @ w.abs()
        return out, size


# sums in 32 bits: in bf16 sixteen products and the sum before are added with two bits less than a rounding keeps, in fp32 a
# chain of as many roundings as products
def _sum_error(length, dtype):
    return ((length / 16 + 2) * 4 if dtype == torch.bfloat16 else length + 2) * STEP


def _gelu64(v):
    return 0.5 * v * torch.erfc(-v / math.sqrt(2))


def _slope64(v):
    return 0.5 * torch.erfc(-v / math.sqrt(2)) + v * torch.exp(-0.5 * v * v) / math.sqrt(2 * math.pi)


@LAYER_CASES
@BOTH
def test_linear_grouped(ctx, lengths, before, behind, k, n, dtype):
    vit, m = ctx
    l = Layer(vit, m, lengths, before, behind, k, n, dtype)
    x, residual = l.some(k, k + 8), l.some(n, n + 16)
    bias = _normal(l.gen, len(lengths), n, scale=0.3)
    want, size = l.products(x[:, :k], False)
    err = _sum_error(k, dtype) * size
    rows = l.covered
    biased = want.clone()
    for g, (b, e) in enumerate(l.spans):
        biased[b:e] += bias[g].double()
    err_b = err + STEP * (biased.abs() + size)

    def check(got, want, tol):
        assert ((got[rows][:, :n].double() - want[rows]).abs() <= (tol + HALF[dtype] * want.abs())[rows]).all()
        assert (got[~rows] == 77).all() and (got[:, n:] == 77).all()

    check(l.forward(x, out=l.blank(n + 24)), want, err)
    plain = l.forward(x, bias, out=l.blank(n + 8))
    check(plain, biased, err_b)
    # |slope of gelu| <= 1.13; the error function's approximation is good to 1.5e-7 and its parts to 2^-20
    tol = 1.13 * err_b + 1e-7 * biased.abs() + 2.5e-7
    pre = l.blank(n + 40)
    out = l.forward(x, bias, 1, out=l.blank(n + 8), pre=pre)
    check(out, _gelu64(biased), tol)
    assert torch.equal(pre[:, :n][rows], plain[:, :n][rows]) and (pre[~rows] == 77).all() and (pre[:, n:] == 77).all()
    again = l.forward(x, bias, 1, out=l.blank(n + 8))
    assert torch.equal(again, out)
    summed = l.forward(x, bias, 2, residual=residual, out=l.blank(n + 8))
    check(summed, biased + residual[:, :n].double().nan_to_num(0), err_b + STEP * (biased.abs() + residual[:, :n].double().abs().nan_to_num(0)))
    own = residual.clone()
    l.forward(x, bias, 2, residual=own, out=own)
    assert torch.equal(own[:, :n][rows], summed[:, :n][rows]) and torch.equal(own[:, n:].isnan(), residual[:, n:].isnan())


@LAYER_CASES
@BOTH
def test_linear_grouped_input_grad(ctx, lengths, before, behind, k, n, dtype):
    vit, m = ctx
    l = Layer(vit, m, lengths, before, behind, k, n, dtype)
    dout, pre = l.some(n, n + 8), l.some(k, k + 8, scale=1.5)
    want, size = l.products(dout[:, :n], True)
    err = _sum_error(n, dtype) * size
    rows = l.covered
    dx = l.input_grad(dout, None, l.blank(k + 16))
    assert ((dx[rows][:, :k].double() - want[rows]).abs() <= (err + HALF[dtype] * want.abs())[rows]).all()
    assert (dx[~rows] == 77).all() and (dx[:, k:] == 77).all()
    # the slope's two parts are good to 1e-6
    slope = _slope64(pre[:, :k].double())
    got = l.input_grad(dout, pre, l.blank(k + 24))
    tol = err * slope.abs() + (want.abs() + err) * 1.2e-6 + HALF[dtype] * (want * slope).abs()
    assert ((got[rows][:, :k].double() - (want * slope)[rows]).abs() <= tol[rows]).all()
    assert (got[~rows] == 77).all() and (got[:, k:] == 77).all()
    own = pre.clone()
    l.input_grad(dout, own, own)
    assert torch.equal(own[:, :k][rows], got[:, :k][rows])


@LAYER_CASES
@BOTH
def test_linear_grouped_weight_grads(ctx, lengths, before, behind, k, n, dtype):
    vit, m = ctx
    l = Layer(vit, m, lengths, before, behind, k, n, dtype)
    x, dout = l.some(k, k + 8), l.some(n, n + 16, scale=0.5)
    dw, db = l.weight_grads(x, dout)
    for g, (b, e) in enumerate(l.spans):
        d, v = dout[b:e, :n].double(), x[b:e, :k].double()
        want, size = d.t() @ v, d.abs().t() @ v.abs()
        parts = 150                                                             # a sum may be cut between all blocks
        assert ((dw[g].double() - want).abs() <= (_sum_error(e - b, dtype) + parts * STEP) * size + HALF[dtype] * want.abs()).all()
        # 16 values at a time, their sums one after the other, four lanes and the parts
        assert ((db[g].double() - d.sum(0)).abs() <= ((e - b) / 16 + 24 + parts) * STEP * d.abs().sum(0)).all()
    again, none = l.weight_grads(x, dout, bias=False)
    assert torch.equal(again, dw)
    assert torch.equal(l.weight_grads(x, dout)[1], db)


# one long sum of few tiles of 256 x 256 is shared by clusters: two and four pairs to a tile, tiles that hang over either edge, a
# last unit of rows that is not full, pairs without rows, and more tiles or units than clusters take
@pytest.mark.parametrize("length,before,behind,k,n", [
    (577, 0, 0, 264, 512), (1091, 3, 70, 776, 520), (520, 0, 130, 1000, 1000), (2000, 0, 0, 512, 1792), (2000, 0, 0, 1032, 1024),
    (64, 5, 900, 128, 1024), (1, 0, 600, 256, 512), (0, 300, 300, 256, 512), (6304, 1, 0, 1280, 1272), (1600, 0, 16, 2056, 1024),
    (12608, 0, 0, 192, 768)])
def test_weight_grads_of_one_group(ctx, length, before, behind, k, n):
    test_linear_grouped_weight_grads(ctx, [length], before, behind, k, n, torch.bfloat16)


# either tile of the fp32 products of rows, whole and with its sum in halves, quarters and eighths, in one round and in several
@pytest.mark.parametrize("lengths,before,behind,k,n", [
    ([577], 0, 0, 768, 768), ([2000], 0, 0, 768, 768), ([333, 333, 334], 0, 7, 1000, 1000), ([33] * 30, 2, 0, 768, 768), ([25] * 8, 0, 0, 384, 1536),
    ([481], 3, 9, 2952, 368), ([1325] * 4, 0, 0, 576, 520), ([1, 300, 0, 299], 0, 0, 136, 2056), ([4] * 16, 0, 0, 2048, 512), ([3152], 0, 0, 192, 192)],
    ids=lambda v: "%dx%d" % (len(v), max(v)) if isinstance(v, list) else str(v))
def test_linear_grouped_fp32_tiles(ctx, lengths, before, behind, k, n):
    test_linear_grouped(ctx, lengths, before, behind, k, n, torch.float32)
    test_linear_grouped_input_grad(ctx, lengths, before, behind, k, n, torch.float32)


@BOTH
def test_linear_without_offsets_is_one_group(ctx, dtype):
    vit, m = ctx
    l = Layer(vit, m, [333], 0, 0, 96, 136, dtype)
    x, dout, bias = l.some(96, 96), l.some(136, 136), _normal(l.gen, 1, 136)
    first = [l.forward(x, bias, out=l.blank(136)), l.input_grad(dout, None, l.blank(96)), *l.weight_grads(x, dout)]
    l.problem = vit.make_grouped_problem(1, 333, 96, 136, 0)
    second = [l.forward(x, bias, out=l.blank(136)), l.input_grad(dout, None, l.blank(96)), *l.weight_grads(x, dout)]
    assert all(torch.equal(a, b) for a, b in zip(first, second))
    # and an ordinary linear layer gives the same sums
    y = torch.empty(333, 136, dtype=dtype, device="cuda")
    vit.vit_op_linear(m.h, _dt(vit, dtype), 333, 136, 96, x.data_ptr(), l.w.data_ptr(), bias.data_ptr(), 0, 0, y.data_ptr())
    m.check()
    want, size = l.products(x, False)
    assert ((first[0].double() - y.double()).abs() <= 2 * (HALF[dtype] * want.abs() + (_sum_error(96, dtype) + 4 * STEP) * (size + 4)) + HALF[dtype] * 4).all()


@BOTH
def test_groups_do_not_mix(ctx, dtype):
    """What is not a number in one group, in its rows or its weights, stays there."""
    vit, m = ctx
    lengths = [70, 33, 200, 1]
    l = Layer(vit, m, lengths, 0, 0, 72, 88, dtype)
    x, dout, pre = l.some(72, 72), l.some(88, 88), l.some(72, 72)
    clean = [l.forward(x, out=l.blank(88)), l.input_grad(dout, pre, l.blank(72)), *l.weight_grads(x, dout)]
    b, e = l.spans[1]
    for t in (x, dout, pre):
        t[b:e] = float("nan")
    x[b], dout[e - 1] = float("inf"), float("-inf")
    l.w[1] = float("nan")
    wild = [l.forward(x, out=l.blank(88)), l.input_grad(dout, pre, l.blank(72)), *l.weight_grads(x, dout)]
    for i, (a, c) in enumerate(zip(clean, wild)):
        if i < 2:
            others = torch.ones(l.rows, dtype=torch.bool, device="cuda")
            others[b:e] = False
            assert torch.equal(a[others], c[others]) and c[b:e].isnan().all()
        else:
            assert torch.equal(a[[0, 2, 3]], c[[0, 2, 3]]) and c[1].isnan().all()


@BOTH
def test_gelu_and_its_slope_far_out(ctx, dtype):
    """Arguments of any size, infinite ones too."""
    vit, m = ctx
    k = 64
    values = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 0.5, -0.5, 3, -3, 5.5, -5.5, 9, -9, 13, -13, 30, -30, 1e4, -1e4, 1e30, -1e30, math.inf, -math.inf,
                           math.nan, 1.0], device="cuda").to(dtype)
    rows = len(values)
    l = Layer(vit, m, [rows], 0, 0, k, k, dtype)
    l.w[0] = torch.eye(k, device="cuda").to(dtype)
    x = torch.zeros(rows, k, dtype=dtype, device="cuda")
    x[:20, 0] = values[:20]
    out = l.forward(x, None, 1, out=l.blank(k))
    want = _gelu64(values[:20].double())
    assert ((out[:20, 0].double() - want).abs() <= HALF[dtype] * want.abs() + 2.5e-7 * values[:20].double().abs().clamp(max=24)).all()
    pre = values[:, None].expand(rows, k).contiguous()
    ones = torch.ones(rows, k, dtype=dtype, device="cuda")
    dx = l.input_grad(ones, pre, l.blank(k))[:, 0].double()
    want = _slope64(values.double())
    want[20:22] = torch.tensor([1.0, 0.0], device="cuda")                       # the limits
    want[18:20] = torch.tensor([1.0, 0.0], device="cuda")                       # (not a number in 64 bits: infinity times zero)
    assert dx[22].isnan()
    keep = torch.arange(rows, device="cuda") != 22
    assert ((dx - want)[keep].abs() <= (HALF[dtype] * want.abs() + 1.2e-6)[keep]).all()
    bias = torch.zeros(1, k, device="cuda")
    bias[0, :3] = torch.tensor([math.inf, -math.inf, math.nan], device="cuda")
    out = l.forward(torch.zeros_like(x), bias, 1, out=l.blank(k))
    assert (out[:, 0] == math.inf).all() and (out[:, 1] == 0).all() and out[:, 2].isnan().all() and (out[:, 3:] == 0).all()


@pytest.mark.parametrize("edges", [[0, 40, 30, 90], [0, -1, 50, 90], [10, 20, 200, 90], [0, 2 ** 31 - 1, 60, 90], [50, 0, 60, 91]])
@BOTH
def test_groups_with_bad_offsets_are_skipped_and_reported(ctx, edges, dtype):
    vit, m = ctx
    l = Layer(vit, m, [90, 0, 0], 0, 0, 64, 72, dtype)
    x, dout = l.some(64, 64), l.some(72, 72)
    l.offsets.copy_(torch.tensor(edges, dtype=torch.int32))
    good = [g for g, (b, e) in enumerate(zip(edges, edges[1:])) if 0 <= b <= e <= 90]
    dt = _dt(vit, dtype)

    def reported(call):
        call()
        with pytest.raises(vit.VitError) as e:
            m.check()
        assert e.value.status == vit.VIT_ERR_OFFSETS
        m.check()

    out, dx = l.blank(72), l.blank(64)
    dw, db = torch.full((3, 72, 64), 77.0, dtype=dtype, device="cuda"), torch.full((3, 72), 77.0, device="cuda")
    n = vit.vit_linear_grouped_backward_weights_bytes(dt, l.problem)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    reported(lambda: vit.vit_op_linear_grouped(m.h, dt, l.problem, x.data_ptr(), 64, l.w.data_ptr(), 0, 0, 0, 0, out.data_ptr(), 72, 0, 0))
    reported(lambda: vit.vit_op_linear_grouped_backward_input(m.h, dt, l.problem, dout.data_ptr(), 72, l.w.data_ptr(), 0, 0, dx.data_ptr(), 64))
    reported(lambda: vit.vit_op_linear_grouped_backward_weights(m.h, dt, l.problem, x.data_ptr(), 64, dout.data_ptr(), 72, dw.data_ptr(),
                                                                db.data_ptr(), ws.data_ptr(), n))
    owners = torch.zeros(90, dtype=torch.int32, device="cuda")
    for g in good:
        owners[edges[g]:edges[g + 1]] += 1
    touched = owners > 0
    for g in range(3):
        b, e = edges[g], edges[g + 1]
        if g not in good:
            assert (dw[g] == 77).all() and (db[g] == 77).all()
            continue
        xs, ds, w = x[b:e].double(), dout[b:e].double(), l.w[g].double()
        for got, want, size, length in ((out[b:e], xs @ w.t(), xs.abs() @ w.abs().t(), 64), (dx[b:e], ds @ w, ds.abs() @ w.abs(), 72),
                                        (dw[g], ds.t() @ xs, ds.abs().t() @ xs.abs(), e - b)):
            fine = (got.double() - want).abs() <= HALF[dtype] * want.abs() + (_sum_error(length, dtype) + 8 * STEP) * size
            if got.shape[0] == e - b and got.data_ptr() != dw[g].data_ptr():
                fine = fine[owners[b:e] == 1]               # rows that two groups share are undefined
            assert fine.all()
    assert (out[~touched] == 77).all() and (dx[~touched] == 77).all()
    # without rows every group that is not empty is a bad one
    none = vit.make_grouped_problem(3, 0, 64, 72, l.offsets.data_ptr())
    reported(lambda: vit.vit_op_linear_grouped(m.h, dt, none, 0, 64, l.w.data_ptr(), 0, 0, 0, 0, 0, 72, 0, 0))
    l.offsets.zero_()
    vit.vit_op_linear_grouped(m.h, dt, none, 0, 64, l.w.data_ptr(), 0, 0, 0, 0, 0, 72, 0, 0)
    vit.vit_op_linear_grouped_backward_input(m.h, dt, none, 0, 72, l.w.data_ptr(), 0, 0, 0, 64)
    vit.vit_op_linear_grouped_backward_weights(m.h, dt, none, 0, 64, 0, 72, dw.data_ptr(), db.data_ptr(), ws.data_ptr(), n)
    m.check()
    assert (dw == 0).all() and (db == 0).all()


def test_grouped_refusals(ctx):
    vit, m = ctx
    rows, k, n, groups = 24, 64, 72, 3
    z = lambda *shape, t=torch.bfloat16: torch.zeros(*shape, dtype=t, device="cuda")
    x, out, res, pre, dx, w, dw = z(rows, k), z(rows, n), z(rows, n), z(rows, n), z(rows, k), z(groups, n, k), z(groups, n, k)
    prek, bias, db = z(rows, k), z(groups, n, t=torch.float32), z(groups, n, t=torch.float32)
    off = torch.tensor([0, 8, 8, 24], dtype=torch.int32, device="cuda")
    P = lambda t: t.data_ptr()
    shape = dict(groups=groups, rows=rows, in_features=k, out_features=n, offsets=P(off))
    size = vit.vit_linear_grouped_backward_weights_bytes(0, vit.make_grouped_problem(**shape))
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    forward = dict(h=m.h, dtype=0, x=P(x), ldx=k, w=P(w), bias=P(bias), epilogue=1, residual=0, ldr=0, out=P(out), ldo=n, pre=P(pre), ldp=n)
    inputs = dict(h=m.h, dtype=0, dout=P(out), lddout=n, w=P(w), pre=P(prek), ldp=k, dx=P(dx), lddx=k)
    weights = dict(h=m.h, dtype=0, x=P(x), ldx=k, dout=P(out), lddout=n, dw=P(dw), dbias=P(db), ws=P(ws), ws_bytes=size)
    calls = ((vit.vit_op_linear_grouped, forward), (vit.vit_op_linear_grouped_backward_input, inputs), (vit.vit_op_linear_grouped_backward_weights, weights))

    def call(f, arguments, problem={}, **changed):
        f(**{**arguments, **changed, "problem": vit.make_grouped_problem(**{**shape, **problem})})

    before = m.launches
    for f, arguments in calls:
        for problem in (dict(groups=0), dict(groups=-1), dict(rows=-1), dict(in_features=0), dict(in_features=60), dict(out_features=4),
                        dict(out_features=76), dict(offsets=0), dict(offsets=P(off) + 2)):
            _refused(vit, lambda: call(f, arguments, problem))
        for problem in (dict(rows=2 ** 31 - 1000), dict(groups=2 ** 30, in_features=2 ** 20, out_features=2 ** 20), dict(groups=2 ** 30)):
            _refused(vit, lambda: call(f, arguments, problem), vit.VIT_ERR_TOO_LARGE)
        for bad in (dict(h=None), dict(dtype=2)):
            _refused(vit, lambda: call(f, arguments, **bad))
        _refused(vit, lambda: f(**{**arguments, "problem": None}))
    for bad in (dict(x=0), dict(w=0), dict(out=0), dict(ldx=56), dict(ldo=76), dict(ldp=64), dict(epilogue=3), dict(epilogue=-1), dict(x=P(x) + 2),
                dict(w=P(w) + 8), dict(bias=P(bias) + 4), dict(out=P(x)), dict(out=P(w)), dict(out=P(bias)), dict(out=P(off)), dict(pre=P(out)),
                dict(pre=P(x)), dict(pre=P(out) + 16), dict(epilogue=2, pre=0), dict(epilogue=2, pre=0, residual=P(res), ldr=40),
                dict(epilogue=2, pre=0, residual=P(out), ldr=80)):
        _refused(vit, lambda: call(vit.vit_op_linear_grouped, forward, **bad))
    for bad in (dict(dout=0), dict(w=0), dict(dx=0), dict(lddout=64), dict(lddx=60), dict(ldp=8), dict(dx=P(out)), dict(dx=P(w)), dict(dx=P(off)),
                dict(dx=P(prek), lddx=72), dict(dx=P(prek) + 128), dict(dout=P(out) + 4)):
        _refused(vit, lambda: call(vit.vit_op_linear_grouped_backward_input, inputs, **bad))
    for bad in (dict(x=0), dict(dout=0), dict(dw=0), dict(ws=0), dict(ldx=8), dict(lddout=8), dict(dw=P(x)), dict(dw=P(out)), dict(dw=P(off)),
                dict(dbias=P(dw)), dict(dbias=P(out)), dict(dbias=P(db) + 4), dict(ws=P(x)), dict(ws=P(dw)), dict(ws=P(ws) + 8), dict(ws=P(db))):
        _refused(vit, lambda: call(vit.vit_op_linear_grouped_backward_weights, weights, **bad))
    _refused(vit, lambda: call(vit.vit_op_linear_grouped_backward_weights, weights, ws_bytes=size - 1), vit.VIT_ERR_WORKSPACE)
    assert m.launches == before
    for f, arguments in calls:
        call(f, arguments)
    # what is not looked at may be anything
    call(vit.vit_op_linear_grouped, forward, epilogue=0, residual=3, ldr=1, pre=5, ldp=1)
    call(vit.vit_op_linear_grouped, forward, epilogue=2, residual=P(res), ldr=n, pre=7, ldp=3)
    m.check()
    assert m.launches == before + 5


# ------------------------------------------------------------------------------------ as they are used
class Mlp:
    """The MLP half of a layer with experts, rows sorted by expert: x + fc2(gelu(fc1(norm(x)))), its gradients, clipped."""

    NAMES = ("w1", "b1", "w2", "b2", "gain", "shift")

    def __init__(self, vit, m, dtype, lengths, hidden, mlp, seed=0):
        self.vit, self.m, self.dtype, self.lengths, self.h, self.f = vit, m, dtype, lengths, hidden, mlp
        gen = _gen(seed)
        groups, rows = len(lengths), sum(lengths)
        self.rows, self.dt = rows, _dt(vit, dtype)
        self.off = torch.tensor([0] + lengths, device="cuda").cumsum(0).to(torch.int32)
        self.p1 = vit.make_grouped_problem(groups, rows, hidden, mlp, self.off.data_ptr())
        self.p2 = vit.make_grouped_problem(groups, rows, mlp, hidden, self.off.data_ptr())
        self.weights = dict(w1=_normal(gen, groups, mlp, hidden, scale=hidden ** -0.5, dtype=dtype), b1=_normal(gen, groups, mlp, scale=0.1),
                            w2=_normal(gen, groups, hidden, mlp, scale=mlp ** -0.5, dtype=dtype), b2=_normal(gen, groups, hidden, scale=0.1),
                            gain=1 + _normal(gen, hidden, scale=0.1), shift=_normal(gen, hidden, scale=0.1))
        self.x, self.dy = _normal(gen, rows, hidden, dtype=dtype), _normal(gen, rows, hidden, scale=0.1, dtype=dtype)
        e = lambda *shape, t=dtype: torch.empty(*shape, dtype=t, device="cuda")
        self.norm, self.pre, self.hid, self.y, self.dpre, self.dnorm, self.dx = (e(rows, d) for d in (hidden, mlp, mlp, hidden, mlp, hidden, hidden))
        self.stats, self.total = e(rows, 2, t=torch.float32), e(1, t=torch.float32)
        self.grads = {k: torch.empty_like(v) for k, v in self.weights.items()}
        self.clipped = {k: torch.empty_like(v) for k, v in self.weights.items()}
        self.tensors = vit.make_tensors([(self.grads[k].data_ptr(), self.clipped[k].data_ptr(), self.grads[k].numel(), _dt(vit, self.grads[k].dtype))
                                         for k in self.NAMES])
        self.size = max(vit.vit_layernorm_backward_bytes(rows, hidden), vit.vit_grad_clip_bytes(len(self.NAMES)),
                        *(vit.vit_linear_grouped_backward_weights_bytes(self.dt, p) for p in (self.p1, self.p2)))
        self.ws = torch.empty(self.size, dtype=torch.uint8, device="cuda")

    def step(self, bound, stream=0):
        vit, h, dt, rows, H, F, w, g = self.vit, self.m.h, self.dt, self.rows, self.h, self.f, self.weights, self.grads
        P = lambda t: t.data_ptr()
        ws = (P(self.ws), self.size)
        vit.vit_op_layernorm_forward(h, dt, rows, H, P(self.x), H, P(w["gain"]), P(w["shift"]), EPS, P(self.norm), H, P(self.stats), stream)
        vit.vit_op_linear_grouped(h, dt, self.p1, P(self.norm), H, P(w["w1"]), P(w["b1"]), 1, 0, 0, P(self.hid), F, P(self.pre), F, stream)
        vit.vit_op_linear_grouped(h, dt, self.p2, P(self.hid), F, P(w["w2"]), P(w["b2"]), 2, P(self.x), H, P(self.y), H, 0, 0, stream)
        vit.vit_op_linear_grouped_backward_weights(h, dt, self.p2, P(self.hid), F, P(self.dy), H, P(g["w2"]), P(g["b2"]), *ws, stream)
        vit.vit_op_linear_grouped_backward_input(h, dt, self.p2, P(self.dy), H, P(w["w2"]), P(self.pre), F, P(self.dpre), F, stream)
        vit.vit_op_linear_grouped_backward_weights(h, dt, self.p1, P(self.norm), H, P(self.dpre), F, P(g["w1"]), P(g["b1"]), *ws, stream)
        vit.vit_op_linear_grouped_backward_input(h, dt, self.p1, P(self.dpre), F, P(w["w1"]), 0, 0, P(self.dnorm), H, stream)
        vit.vit_op_layernorm_backward(h, dt, rows, H, P(self.x), H, P(w["gain"]), P(self.stats), P(self.dnorm), H, P(self.dy), H, P(self.dx), H,
                                      P(g["gain"]), P(g["shift"]), *ws, stream)
        vit.vit_op_grad_clip(h, self.tensors, len(self.NAMES), bound, P(self.total), *ws, stream)

    def results(self):
        return [self.y, self.dx, self.total, *self.grads.values(), *self.clipped.values()]

    def loss(self, x, w):
        """In 64 bits; x and the weights as tensors that may ask for gradients."""
        z = (x - x.mean(1, keepdim=True)) / (x.var(1, unbiased=False, keepdim=True) + EPS).sqrt() * w["gain"] + w["shift"]
        ys = []
        for g, rows in enumerate(z.split(self.lengths)):
            ys.append(_gelu64(rows @ w["w1"][g].t() + w["b1"][g]) @ w["w2"][g].t() + w["b2"][g])
        return x + torch.cat(ys)


@BOTH
def test_training_step_of_an_mlp_with_experts(ctx, dtype):
    vit, m = ctx
    mlp = Mlp(vit, m, dtype, [130, 0, 57, 300, 1], 192, 384)
    mlp.step(0.5)
    m.check()
    x = mlp.x.double().requires_grad_()
    w = {k: v.double().requires_grad_() for k, v in mlp.weights.items()}
    y = mlp.loss(x, w)
    want = dict(zip(("x",) + mlp.NAMES, torch.autograd.grad((y * mlp.dy.double()).sum(), [x] + [w[k] for k in mlp.NAMES])))
    # Every tensor on the way is rounded once, by at most HALF of each value and so of its norm; products with matrices of random
    # numbers carry such a part of the norm on as it is, give or take a few percent.  On the longest way (x, norm, argument, GELU,
    # gradient of the argument, of the norm, result) there are six roundings; the sums in 32 bits add a few hundred steps.
    part = lambda a, b: ((a.double() - b).norm() / b.norm()).item()
    most = 6 * 1.1 * HALF[dtype] + 500 * STEP
    assert part(mlp.y, y.detach()) <= most
    assert part(mlp.dx, want["x"]) <= most
    for k in mlp.NAMES:
        assert part(mlp.grads[k], want[k]) <= most, k
    _check_clip(list(mlp.grads.values()), 0.5, mlp.total, list(mlp.clipped.values()))
    assert mlp.total.item() > 0.5                                                # the bound is at work
    # along a direction, against differences of the 64-bit forward pass
    gen = _gen(9)
    by = {k: _normal(gen, *v.shape).double() * v.double().abs().mean() for k, v in [("x", mlp.x)] + list(mlp.weights.items())}
    at = lambda e: (mlp.loss(mlp.x.double() + e * by["x"], {k: v.double() + e * by[k] for k, v in mlp.weights.items()}) * mlp.dy.double()).sum().item()
    difference = (at(1e-5) - at(-1e-5)) / 2e-5
    got = {**mlp.grads, "x": mlp.dx}
    inner = sum((got[k].double() * by[k]).sum().item() for k in by)
    size = math.sqrt(sum(got[k].double().norm().item() ** 2 for k in by)) * math.sqrt(sum(by[k].norm().item() ** 2 for k in by))
    assert abs(inner - difference) <= most * size + 1e-6 * abs(difference)


@BOTH
def test_training_step_on_streams_and_in_graphs(ctx, dtype):
    """Two loops at once, each with scratch of its own, eagerly on two streams and as graphs replayed with other inputs."""
    vit, m = ctx
    loops = [Mlp(vit, m, dtype, [200, 31, 0, 400], 128, 320, seed=1), Mlp(vit, m, dtype, [1500], 256, 512, seed=2)]
    want = []
    for loop in loops:
        loop.step(0.3)
        m.check()
        want.append([t.clone() for t in loop.results()])
    streams = [torch.cuda.Stream() for _ in loops]
    torch.cuda.synchronize()
    for _ in range(5):
        for loop, stream in zip(loops, streams):
            loop.step(0.3, stream.cuda_stream)
    torch.cuda.synchronize()
    m.check()
    for loop, w in zip(loops, want):
        assert all(torch.equal(a, b) for a, b in zip(loop.results(), w))
    graphs = [torch.cuda.CUDAGraph() for _ in loops]
    for loop, stream, graph in zip(loops, streams, graphs):
        with torch.cuda.graph(graph, stream=stream):
            loop.step(0.3, stream.cuda_stream)
    for loop in loops:
        for t in loop.results():
            t.fill_(55.0)
        loop.dy.mul_(2)
        loop.x.neg_()
    torch.cuda.synchronize()
    for _ in range(3):
        for stream, graph in zip(streams, graphs):
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    m.check()
    replayed = [[t.clone() for t in loop.results()] for loop in loops]
    for loop, r in zip(loops, replayed):
        loop.step(0.3)
        m.check()
        assert all(torch.equal(a, b) for a, b in zip(loop.results(), r))


def test_rows_beyond_two_to_the_31_elements(ctx):
    """The last rows of buffers whose offsets need more than 32 bits."""
    vit, m = ctx
    rows, ld, k, n, last = 70000, 32768, 64, 72, 300
    a, b = (torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda").view(rows, ld) for _ in range(2))
    gen = _gen(8)
    a[-last:, :k] = _normal(gen, last, k, dtype=torch.bfloat16)
    off = torch.tensor([0, 0, rows - last, rows], dtype=torch.int32, device="cuda")
    off[1] = off[2]                                        # the first group has all other rows; the second none
    l = Layer(vit, m, [1], 0, 0, k, n, torch.bfloat16)
    small = a[-last:, :k].contiguous()
    w = _normal(gen, 3, n, k, dtype=torch.bfloat16)
    p = vit.make_grouped_problem(3, rows, k, n, off.data_ptr())
    one = vit.make_grouped_problem(1, last, k, n, 0)
    vit.vit_op_linear_grouped(m.h, 0, p, a.data_ptr(), ld, w.data_ptr(), 0, 0, 0, 0, b.data_ptr(), ld, 0, 0)
    want = torch.empty(last, n, dtype=torch.bfloat16, device="cuda")
    vit.vit_op_linear_grouped(m.h, 0, one, small.data_ptr(), k, w[2].data_ptr(), 0, 0, 0, 0, want.data_ptr(), n, 0, 0)
    m.check()
    assert torch.equal(b[-last:, :n], want)
    dx = torch.empty(last, k, dtype=torch.bfloat16, device="cuda")
    vit.vit_op_linear_grouped_backward_input(m.h, 0, one, want.data_ptr(), n, w[2].data_ptr(), 0, 0, dx.data_ptr(), k)
    g, s = torch.ones(k, device="cuda"), torch.zeros(k, device="cuda")
    size = vit.vit_linear_grouped_backward_weights_bytes(0, p)
    ws, dw, dw1 = torch.empty(size, dtype=torch.uint8, device="cuda"), torch.empty_like(w), torch.empty_like(w[:1])
    a[:last, :k] = a[-last:, :k]
    b[:last, :n] = b[-last:, :n]
    off.copy_(torch.tensor([0, last, last, last], dtype=torch.int32))
    vit.vit_op_linear_grouped_backward_weights(m.h, 0, p, a.data_ptr(), ld, b.data_ptr(), ld, dw.data_ptr(), 0, ws.data_ptr(), size)
    off.copy_(torch.tensor([rows - last, rows, rows, rows], dtype=torch.int32))
    dw2 = torch.empty_like(w)
    vit.vit_op_linear_grouped_backward_weights(m.h, 0, p, a.data_ptr(), ld, b.data_ptr(), ld, dw2.data_ptr(), 0, ws.data_ptr(), size)
    assert torch.equal(dw, dw2) and dw[0].abs().sum() > 0 and (dw[1:] == 0).all()
    off.copy_(torch.tensor([rows, rows, rows - last, rows], dtype=torch.int32))       # (the second one is a bad one)
    vit.vit_op_linear_grouped_backward_input(m.h, 0, p, b.data_ptr(), ld, w.data_ptr(), 0, 0, a.data_ptr(), ld)
    with pytest.raises(vit.VitError):
        m.check()
    assert torch.equal(a[-last:, :k], dx)
    stats, stats1 = torch.empty(rows, 2, device="cuda"), torch.empty(last, 2, device="cuda")
    y1 = torch.empty(last, k, dtype=torch.bfloat16, device="cuda")
    vit.vit_op_layernorm_forward(m.h, 0, last, k, a[-last:].data_ptr(), ld, g.data_ptr(), s.data_ptr(), EPS, y1.data_ptr(), k, stats1.data_ptr())
    vit.vit_op_layernorm_forward(m.h, 0, rows, k, a.data_ptr(), ld, g.data_ptr(), s.data_ptr(), EPS, b.data_ptr(), ld, stats.data_ptr())
    assert torch.equal(b[-last:, :k], y1) and torch.equal(stats[-last:], stats1)
    m.check()
    # and one tensor as long
    a.fill_(0.5)
    norm, out = _clip(vit, m, [a.view(-1)], 1.0, "same")
    assert norm.item() == pytest.approx(0.5 * math.sqrt(rows * ld), rel=1e-6)
    by = 1 / norm.item()
    assert (a == torch.tensor(0.5 * by).to(torch.bfloat16).item()).all()
