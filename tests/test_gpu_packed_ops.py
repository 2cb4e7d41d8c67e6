"""Operators of a layer over packed images (rotation, query/key norm, attention and their gradients)
against their definitions in 64 bits, called through the C boundary."""
import math
from fractions import Fraction

import numpy as np
import pytest

import vitgen

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}      # half a step of the type, relative
EPS = 1e-6


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


# ------------------------------------------------------------------------------- rotation and norm
def _turn64(x, pairs, freqs, positions, interleaved, inverse=False):
    """x [rows, heads, d] in 64 bits; the rotation as a product of complex numbers."""
    n, parts, first = sum(pairs), [], 0
    for axis, count in enumerate(pairs):
        angle = positions[axis].double()[:, None] * freqs[first:first + count].double()[None]
        parts.append(torch.polar(torch.ones_like(angle), -angle if inverse else angle))
        first += count
    unit = torch.cat(parts, 1)[:, None]
    if interleaved:
        z = torch.complex(x[..., 0:2 * n:2], x[..., 1:2 * n:2]) * unit
        head = torch.stack([z.real, z.imag], -1).flatten(-2)
    else:
        z = torch.complex(x[..., :n], x[..., n:2 * n]) * unit
        head = torch.cat([z.real, z.imag], -1)
    return torch.cat([head, x[..., 2 * n:]], -1)


def _rope_inputs(gen, rows, pairs, far):
    freqs = torch.cat([100.0 ** (-torch.arange(k, device="cuda", dtype=torch.float64) / max(1, k)) for k in pairs]).float()
    positions = torch.randint(-far, far + 1, (len(pairs), rows), generator=gen, device="cuda").to(torch.int32)
    return freqs, positions


ROPE_CASES = [
    # rows, heads, d, pairs per axis, far
    (1, 1, 16, (8,), 3), (1, 3, 64, (16, 16), 14), (197, 6, 64, (16, 16), 14), (33, 5, 80, (20, 20), 1000),
    (7, 2, 128, (16, 24, 24), 2 ** 31 - 1), (300, 3, 96, (9, 11, 5, 3), 10 ** 6), (65, 1, 48, (11,), 100), (129, 17, 112, (30, 0, 26), 77),
    (5, 40, 32, (16,), 9), (2000, 3, 16, (3, 2), 50),
]


@pytest.mark.parametrize("rows,heads,d,pairs,far", ROPE_CASES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rope_axes(ctx, rows, heads, d, pairs, far, interleaved, dtype):
    vit, m = ctx
    gen = _gen(rows * 7 + d)
    freqs, positions = _rope_inputs(gen, rows, pairs, far)
    ldx, ldy = heads * d + 24, heads * d + 8
    x = _normal(gen, rows, ldx, dtype=dtype)
    rope = vit.make_rope(pairs, freqs.data_ptr(), positions.data_ptr(), interleaved)
    for inverse in (False, True):
        y = torch.full((rows, ldy), 77.0, dtype=dtype, device="cuda")
        vit.vit_op_rope_axes(m.h, _dt(vit, dtype), rows, heads, d, rope, inverse, x.data_ptr(), ldx, y.data_ptr(), ldy)
        m.check()
        x64 = x[:, :heads * d].double().unflatten(1, (heads, d))
        want = _turn64(x64, pairs, freqs, positions, interleaved, inverse).flatten(1)
        # rounding of the result; cosine and sine are off by at most a few 2^-24 (angle reduced in 64
        # bits, one rounding of the remaining turn, 2 ulp of the function), products and sum by 3 more
        n = sum(pairs)
        size = torch.zeros_like(x64)
        if interleaved:
            r = torch.hypot(x64[..., 0:2 * n:2], x64[..., 1:2 * n:2])
            size[..., 0:2 * n:2] = size[..., 1:2 * n:2] = r
        else:
            size[..., :n] = size[..., n:2 * n] = torch.hypot(x64[..., :n], x64[..., n:2 * n])
        tol = HALF[dtype] * want.abs() + 16 * 2.0 ** -24 * size.flatten(1)
        assert ((y[:, :heads * d].double() - want).abs() <= tol).all()
        assert (y[:, heads * d:] == 77).all()                                        # behind the heads: as it was
        # channels that do not turn come through bit for bit
        assert torch.equal(y[:, :heads * d].unflatten(1, (heads, d))[..., 2 * n:], x[:, :heads * d].unflatten(1, (heads, d))[..., 2 * n:])
    # in place gives the same bits
    z = x.clone()
    vit.vit_op_rope_axes(m.h, _dt(vit, dtype), rows, heads, d, rope, True, z.data_ptr(), ldx, z.data_ptr(), ldx)
    m.check()
    assert torch.equal(z[:, :heads * d], y[:, :heads * d]) and torch.equal(z[:, heads * d:], x[:, heads * d:])


def test_rope_axes_does_not_mix_in_what_a_still_channel_holds(ctx):
    """NaN and infinity in channels that do not turn stay there."""
    vit, m = ctx
    for interleaved in (False, True):
        gen = _gen(5)
        freqs, positions = _rope_inputs(gen, 9, (5,), 4)
        x = _normal(gen, 9, 32, dtype=torch.bfloat16)
        x[:, 10:] = float("nan")
        x[:, 20] = float("inf")
        y = torch.zeros_like(x)
        rope = vit.make_rope((5,), freqs.data_ptr(), positions.data_ptr(), interleaved)
        vit.vit_op_rope_axes(m.h, vit.VIT_BF16, 9, 1, 32, rope, False, x.data_ptr(), 32, y.data_ptr(), 32)
        m.check()
        assert torch.isfinite(y[:, :10]).all()
        assert torch.isnan(y[:, 11:20]).all() and torch.isinf(y[:, 20]).all()


NORM_CASES = [
    # rows, q heads, k heads, d, pairs
    (1, 1, 1, 16, (8,)), (197, 12, 12, 64, (16, 16)), (33, 9, 3, 48, (8, 7, 8)), (257, 16, 16, 80, (20, 20)),
    (10, 4, 1, 128, (16, 24, 24)), (515, 0, 5, 96, (13, 9)), (64, 3, 0, 112, ()), (3001, 2, 2, 32, (4, 4, 4, 4)),
    # many rows: they come through the rings in shared memory, of four, three and two rows; or are too long for them
    (5003, 3, 2, 64, (16, 16)), (4737, 2, 2, 128, (16, 24, 24)), (4990, 12, 12, 64, (16, 16)), (4750, 20, 20, 112, (28, 28)),
    (5001, 5, 5, 80, (11, 9)),
]


def _norm_rope64(x, gains, heads, pairs, freqs, positions, interleaved):
    parts = []
    for part, gain in zip(x.split(heads, 1), gains):
        y = part / ((part * part).mean(-1, keepdim=True) + EPS).sqrt() * gain
        parts.append(_turn64(y, pairs, freqs, positions, interleaved) if pairs else y)
    return torch.cat(parts, 1)


@pytest.mark.parametrize("rows,hq,hk,d,pairs", NORM_CASES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_qk_norm_rope_and_gradients(ctx, rows, hq, hk, d, pairs, interleaved, dtype):
    vit, m = ctx
    gen = _gen(rows + 3 * d)
    heads, width = hq + hk, (hq + hk) * d
    ld = width + 16
    x = _normal(gen, rows, ld, scale=1.7, dtype=dtype)
    x[rows // 2, :d] = 0                                                # a head of zeros: eps keeps it finite
    dy = _normal(gen, rows, ld, scale=0.5, dtype=dtype)
    gains = 1 + _normal(gen, 2, d, scale=0.2)
    rope = None
    freqs = positions = None
    if pairs:
        freqs, positions = _rope_inputs(gen, rows, pairs, 5000)
        rope = vit.make_rope(pairs, freqs.data_ptr(), positions.data_ptr(), interleaved)
    y = torch.full((rows, ld), 55.0, dtype=dtype, device="cuda")
    args = (m.h, _dt(vit, dtype), rows, hq, hk, d, gains[0].data_ptr(), gains[1].data_ptr(), EPS, rope)
    vit.vit_op_qk_norm_rope(*args, x.data_ptr(), ld, y.data_ptr(), ld)
    m.check()
    x64 = x[:, :width].double().unflatten(1, (heads, d)).requires_grad_()
    g64 = [g.double().requires_grad_() for g in gains]
    want = _norm_rope64(x64, g64, [hq, hk], pairs, freqs, positions, interleaved)
    # the norm is a sum of d squares in fp32 (relative d 2^-24 at most), a division and a root; the
    # rotation mixes the two channels of a pair: their size is at most the head's largest
    size = _norm_rope64(x64, g64, [hq, hk], (), None, None, False).detach().abs().amax(-1, keepdim=True) * math.sqrt(2)
    rel32 = (d + 24) * 2.0 ** -24
    tol = HALF[dtype] * want.detach().abs() + rel32 * size
    assert ((y[:, :width].double().unflatten(1, (heads, d)) - want.detach()).abs() <= tol).all()
    assert (y[:, width:] == 55).all()
    inplace = x.clone()
    vit.vit_op_qk_norm_rope(*args, inplace.data_ptr(), ld, inplace.data_ptr(), ld)
    m.check()
    assert torch.equal(inplace[:, :width], y[:, :width]) and torch.equal(inplace[:, width:], x[:, width:])

    # gradients against those of the definition
    n = vit.vit_qk_norm_rope_backward_bytes(rows, hq, hk, d)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")       # NaN: nothing of it may be read before it is written
    dg = torch.full((2, d), float("nan"), device="cuda")
    dx = torch.full((rows, ld), 55.0, dtype=dtype, device="cuda")
    vit.vit_op_qk_norm_rope_backward(*args, x.data_ptr(), ld, dy.data_ptr(), ld, dx.data_ptr(), ld, dg[0].data_ptr(), dg[1].data_ptr(),
                                     ws.data_ptr(), n)
    m.check()
    dy64 = dy[:, :width].double().unflatten(1, (heads, d))
    wx, *wg = torch.autograd.grad(want, [x64] + g64, dy64, allow_unused=True)
    rstd = 1 / ((x64 * x64).mean(-1, keepdim=True) + EPS).sqrt().detach()
    xh = (x64.detach() * rstd).abs()
    gain_max = gains.abs().max().double()
    u = dy64.abs().amax(-1, keepdim=True) * math.sqrt(2)                # bound of a channel of the turned-back gradient
    inner = gain_max * u * xh.mean(-1, keepdim=True)                    # bound of mean(w xh)
    tol = HALF[dtype] * wx.abs() + 4 * rel32 * rstd * (gain_max * u + xh * inner)
    assert ((dx[:, :width].double().unflatten(1, (heads, d)) - wx).abs() <= tol).all()
    assert (dx[:, width:] == 55).all()
    parts = (u * xh).split([hq, hk], 1)
    for got, exact, part, count in zip(dg, wg, parts, (hq, hk)):
        exact = torch.zeros(d, device="cuda", dtype=torch.float64) if exact is None else exact
        # fp32 sums over rows * heads in parts: at most the number of additions of one partial sum and of their join
        tol = (rel32 * 4 + 2.0 ** -24 * min(rows * max(1, count), 4096)) * part.sum((0, 1)) + 1e-30
        assert ((got.double() - exact).abs() <= tol).all()
    # in place over dy, and over x: the same bits
    for over in (x, dy):
        both = over.clone()
        xs, ds = (both, dy) if over is x else (x, both)
        dg2 = torch.empty_like(dg)
        vit.vit_op_qk_norm_rope_backward(*args, xs.data_ptr(), ld, ds.data_ptr(), ld, both.data_ptr(), ld, dg2[0].data_ptr(),
                                         dg2[1].data_ptr(), ws.data_ptr(), n)
        m.check()
        assert torch.equal(both[:, :width], dx[:, :width]) and torch.equal(dg2, dg)


def test_qk_norm_rope_of_no_rows(ctx):
    vit, m = ctx
    g = torch.ones(64, device="cuda")
    dg = torch.full((2, 64), float("nan"), device="cuda")
    n = vit.vit_qk_norm_rope_backward_bytes(0, 2, 2, 64)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    vit.vit_op_qk_norm_rope(m.h, vit.VIT_BF16, 0, 2, 2, 64, g.data_ptr(), g.data_ptr(), EPS, None, 0, 256, 0, 256)
    vit.vit_op_qk_norm_rope_backward(m.h, vit.VIT_BF16, 0, 2, 2, 64, g.data_ptr(), g.data_ptr(), EPS, None, 0, 256, 0, 256, 0, 256,
                                     dg[0].data_ptr(), dg[1].data_ptr(), ws.data_ptr(), n)
    m.check()
    assert (dg == 0).all()


# ------------------------------------------------------------------------------- attention
class Packed:
    """One problem with its operands in the column blocks of wider buffers, and its exact results."""

    def __init__(self, vit, ql, kl, heads, kv, d, dtype, seed=0, lead=0, trail=0, spread=1.2, cross=None):
        self.vit, self.ql, self.kl, self.heads, self.kv, self.d, self.dtype = vit, ql, kl, heads, kv, d, dtype
        gen = _gen(seed + d * 31 + sum(ql))
        self.q_rows, self.k_rows = lead + sum(ql) + trail, lead + sum(kl) + trail
        self.q_off = torch.tensor(np.cumsum([lead] + ql), dtype=torch.int32, device="cuda")
        self.k_off = torch.tensor(np.cumsum([lead] + kl), dtype=torch.int32, device="cuda")
        self.covered_q = slice(lead, lead + sum(ql))
        self.covered_k = slice(lead, lead + sum(kl))
        self.ldq, self.ldkv = heads * d + 16, (2 * kv + 1) * d
        self.qbuf = _normal(gen, self.q_rows, self.ldq, scale=spread, dtype=dtype)
        self.kvbuf = _normal(gen, self.k_rows, self.ldkv, scale=spread, dtype=dtype)
        self.q, self.k, self.v = self.qbuf[:, :heads * d], self.kvbuf[:, :kv * d], self.kvbuf[:, kv * d:2 * kv * d]
        self.dout = _normal(gen, self.q_rows, heads * d, scale=0.3, dtype=dtype)
        self.scale = 1 / math.sqrt(d)
        self.problem = vit.make_attention_problem(len(ql), heads, kv, d, self.q_rows, max(ql), self.q_off.data_ptr(), self.k_rows,
                                                  max(kl), self.k_off.data_ptr(), self.scale)

    def forward(self, m, stream=0):
        vit = self.vit
        dt = _dt(vit, self.dtype)
        out = torch.full((self.q_rows, self.heads * self.d + 8), 33.0, dtype=self.dtype, device="cuda")
        lse = torch.full((self.heads, self.q_rows), 33.0, device="cuda")
        n = vit.vit_attention_packed_bytes(dt, self.problem, False)
        ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        vit.vit_op_attention_packed(m.h, dt, self.problem, self.q.data_ptr(), self.ldq, self.k.data_ptr(), self.ldkv, self.v.data_ptr(),
                                    self.ldkv, out.data_ptr(), out.stride(0), lse.data_ptr(), ws.data_ptr(), n, stream)
        self._keep = ws
        return out, lse

    def backward(self, m, out, lse, stream=0):
        vit = self.vit
        dt = _dt(vit, self.dtype)
        dq = torch.full_like(self.qbuf, 33.0)
        dkv = torch.full_like(self.kvbuf, 33.0)
        n = vit.vit_attention_packed_bytes(dt, self.problem, True)
        ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        kw = self.kv * self.d
        vit.vit_op_attention_packed_backward(
            m.h, dt, self.problem, self.q.data_ptr(), self.ldq, self.k.data_ptr(), self.ldkv, self.v.data_ptr(), self.ldkv,
            out.data_ptr(), out.stride(0), lse.data_ptr(), self.dout.data_ptr(), self.dout.stride(0), dq.data_ptr(), self.ldq,
            dkv.data_ptr(), self.ldkv, dkv[:, kw:].data_ptr() if self.k_rows else 0, self.ldkv, ws.data_ptr(), n, stream)
        self._keep = ws
        return dq, dkv

    def sequences(self):
        q0, k0 = int(self.q_off[0]), int(self.k_off[0])
        for a, b in zip(self.ql, self.kl):
            yield slice(q0, q0 + a), slice(k0, k0 + b)
            q0, k0 = q0 + a, k0 + b

    def check_forward(self, out, lse):
        d, half, group = self.d, HALF[self.dtype], self.heads // self.kv
        for qs, ks in self.sequences():
            a, b = qs.stop - qs.start, ks.stop - ks.start
            if a == 0:
                continue
            for h in range(self.heads):
                got = out[qs, h * d:(h + 1) * d].double()
                if b == 0:
                    assert (got == 0).all() and (lse[h, qs] == -math.inf).all()
                    continue
                q, k, v = self.q[qs, h * d:(h + 1) * d].double(), *(t[ks, (h // group) * d:(h // group + 1) * d].double()
                                                                     for t in (self.k, self.v))
                s = self.scale * q @ k.t()
                # a score is a sum of d products in fp32; its error is a relative one of the probability
                e = (d + 8) * 2.0 ** -24 * (self.scale * q.abs() @ k.abs().t()).max() + 2.0 ** -20
                w = torch.logsumexp(s, 1)
                p = torch.softmax(s, 1)
                # probabilities rounded to the operands' type before the product with v (bf16), their sum and the
                # product accumulated in fp32, the result rounded once
                tol = half * (p @ v).abs() + (half * 1.01 + 2 * e + (b + 16) * 2.0 ** -24) * (p @ v.abs())
                assert ((got - p @ v).abs() <= tol).all(), (a, b, h, float(((got - p @ v).abs() - tol).max()))
                assert ((lse[h, qs].double() - w).abs() <= e + (b + 16) * 2.0 ** -24 + 2.0 ** -22 * w.abs()).all()
        rest = torch.ones(self.q_rows, dtype=torch.bool, device="cuda")
        rest[self.covered_q] = False
        assert (out[rest] == 33).all() and (lse[:, rest] == 33).all() and (out[:, self.heads * d:] == 33).all()

    def check_backward(self, out, lse, dq, dkv):
        d, half, group, kw = self.d, HALF[self.dtype], self.heads // self.kv, self.kv * self.d
        for qs, ks in self.sequences():
            a, b = qs.stop - qs.start, ks.stop - ks.start
            for g in range(self.kv):
                k, v = (t[ks, g * d:(g + 1) * d].double() for t in (self.k, self.v))
                wk, wv, tk, tv = (torch.zeros(b, d, dtype=torch.float64, device="cuda") for _ in range(4))
                for h in range(g * group, (g + 1) * group):
                    if a == 0:
                        continue
                    got = dq[qs, h * d:(h + 1) * d].double()
                    if b == 0:
                        assert (got == 0).all()
                        continue
                    q, o, do = (t[qs, h * d:(h + 1) * d].double() for t in (self.q, out, self.dout))
                    s = self.scale * q @ k.t()
                    e = (d + 8) * 2.0 ** -24 * (self.scale * q.abs() @ k.abs().t()).max() + 2.0 ** -20
                    p = torch.exp(s - lse[h, qs, None].double())
                    dp, delta = do @ v.t(), (do * o).sum(1, keepdim=True)
                    ds = p * (dp - delta)
                    # dp and delta are sums of d products in fp32 and their difference is rounded; ds is rounded to
                    # the operands' type (bf16) before its two products
                    dds = ds.abs() * (half * 1.01 + 2 * e) + p * (d + 8) * 2.0 ** -24 * (do.abs() @ v.abs().t() + (do * o).abs().sum(1, keepdim=True))
                    acc = (max(a, b) * group + 16) * 2.0 ** -24
                    want = self.scale * ds @ k
                    tol = half * want.abs() + self.scale * (dds + acc * ds.abs()) @ k.abs()
                    assert ((got - want).abs() <= tol).all(), (a, b, h, float(((got - want).abs() - tol).max()))
                    wk += self.scale * ds.t() @ q
                    tk += self.scale * (dds + acc * ds.abs()).t() @ q.abs()
                    wv += p.t() @ do
                    tv += ((half * 1.01 + 2 * e + acc) * p).t() @ do.abs()
                if b:
                    gk, gv = dkv[ks, g * d:(g + 1) * d].double(), dkv[ks, kw + g * d:kw + (g + 1) * d].double()
                    assert ((gk - wk).abs() <= tk + half * wk.abs()).all(), (a, b, g, float((gk - wk).abs().max()))
                    assert ((gv - wv).abs() <= tv + half * wv.abs()).all(), (a, b, g, float((gv - wv).abs().max()))
        for t, covered, width in ((dq, self.covered_q, self.heads * d), (dkv, self.covered_k, 2 * kw)):
            rest = torch.ones(t.shape[0], dtype=torch.bool, device="cuda")
            rest[covered] = False
            assert (t[rest] == 33).all() and (t[:, width:] == 33).all()


ATTENTION_CASES = [
    # query lengths, key lengths (None: the same), heads, kv heads, d
    ([1], None, 1, 1, 16), ([1], [5], 2, 1, 64), ([197, 197], None, 3, 3, 64), ([257], None, 2, 2, 80), ([64, 128, 192], None, 2, 1, 64),
    ([5, 0, 63, 65, 1, 127, 129], None, 2, 2, 48), ([300, 17], None, 4, 2, 128), ([33, 260, 1], None, 3, 1, 96), ([130], None, 2, 2, 112),
    ([100, 3, 40], [7, 0, 300], 2, 2, 32), ([0, 70, 20], [50, 0, 129], 4, 1, 64), ([1, 1, 1, 1], [577, 1, 0, 1030], 4, 4, 64),
    ([2, 3, 1], [1025, 64, 2000], 6, 2, 80), ([700, 385], None, 2, 2, 64), ([1, 1], [3000, 129], 3, 1, 128), ([513], [1], 2, 2, 128),
    ([1100], None, 1, 1, 80), ([256, 255, 384], None, 1, 1, 16),
    # few and long: the work on a tile of keys (or queries) is shared out, also for the short sequences beside them
    ([1300, 20, 0, 530], None, 8, 2, 64), ([2100, 70], None, 4, 1, 128), ([30, 700], [2000, 1], 2, 2, 48),
    ([1500, 3], None, 2, 1, 96), ([900, 1030], None, 2, 2, 112),
    # as many queries as the kernel for few of them takes (four rows in bf16, eight in fp32), and one more
    ([1, 1, 0], [1030, 5, 3], 8, 1, 64), ([2, 1], [300, 0], 4, 2, 128), ([4, 3], [700, 70], 2, 2, 112), ([8, 2], [333, 65], 2, 2, 48),
    ([9, 5], [333, 65], 1, 1, 16),
    # shares in which a short sequence counts for more tiles than it has
    ([3000, 1, 0, 70], None, 8, 2, 64), ([2600, 3, 0, 129], None, 8, 2, 128),
]


@pytest.mark.parametrize("ql,kl,heads,kv,d", ATTENTION_CASES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_packed_attention_and_gradients(ctx, ql, kl, heads, kv, d, dtype):
    vit, m = ctx
    p = Packed(vit, ql, kl or ql, heads, kv, d, dtype, lead=3, trail=5)
    out, lse = p.forward(m)
    m.check()
    p.check_forward(out, lse)
    dq, dkv = p.backward(m, out, lse)
    m.check()
    p.check_backward(out, lse, dq, dkv)
    # the same call gives the same bits
    out2, lse2 = p.forward(m)
    dq2, dkv2 = p.backward(m, out, lse)
    m.check()
    for x, y in ((out, out2), (lse, lse2), (dq, dq2), (dkv, dkv2)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("spread", [0.02, 6.0])
def test_packed_attention_flat_and_peaked(ctx, dtype, spread):
    """Near-uniform attention, and scores so far apart that one key takes everything."""
    vit, m = ctx
    p = Packed(vit, [197, 70], [197, 70], 2, 2, 64, dtype, spread=spread, seed=9)
    out, lse = p.forward(m)
    m.check()
    p.check_forward(out, lse)
    dq, dkv = p.backward(m, out, lse)
    m.check()
    p.check_backward(out, lse, dq, dkv)


@pytest.mark.parametrize("rising", [False, True])
def test_packed_attention_scores_that_keep_rising(ctx, rising):
    """The row maximum moves in every tile of keys (or never after the first)."""
    vit, m = ctx
    p = Packed(vit, [130], [900], 1, 1, 64, torch.bfloat16, seed=4)
    ramp = torch.linspace(0, 30, 900, device="cuda")
    p.q[:, 0] = 8.0
    p.k[:, 0] = (ramp if rising else ramp.flip(0)).to(torch.bfloat16)
    out, lse = p.forward(m)
    m.check()
    p.check_forward(out, lse)
    dq, dkv = p.backward(m, out, lse)
    m.check()
    p.check_backward(out, lse, dq, dkv)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("ql,kl", [([70, 61, 200], None), ([1, 1, 1], [70, 61, 200])])
def test_packed_attention_neighbours_stay_out(ctx, dtype, ql, kl):
    """A sequence full of NaN, and infinities in the rows before and behind all of them, reach no other sequence."""
    vit, m = ctx
    p = Packed(vit, ql, kl or ql, 2, 2, 80, dtype, lead=2, trail=9)
    clean = p.forward(m)
    clean_grads = p.backward(m, *clean)
    m.check()
    poison = list(p.sequences())[1]
    for t, at, covered in ((p.qbuf, poison[0], p.covered_q), (p.kvbuf, poison[1], p.covered_k), (p.dout, poison[0], p.covered_q)):
        t[at] = float("nan")
        t[:covered.start] = float("inf")
        t[covered.stop:] = float("-inf")
    out, lse = p.forward(m)
    out_b, lse_b = clean[0].clone(), clean[1].clone()
    out_b[poison[0]] = float("nan")
    lse_b[:, poison[0]] = float("nan")
    dq, dkv = p.backward(m, out_b, lse_b)
    m.check()
    for i in (0, 2):
        qs, ks = list(p.sequences())[i]
        assert torch.equal(out[qs], clean[0][qs]) and torch.equal(lse[:, qs], clean[1][:, qs])
        assert torch.equal(dq[qs], clean_grads[0][qs]) and torch.equal(dkv[ks], clean_grads[1][ks])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_packed_attention_without_any_key(ctx, dtype):
    vit, m = ctx
    p = Packed(vit, [5, 130], [0, 0], 2, 1, 64, dtype)
    out, lse = p.forward(m)
    m.check()
    assert (out[:, :128] == 0).all() and (lse == -math.inf).all()
    dq, _ = p.backward(m, out, lse)
    m.check()
    assert (dq[:, :128] == 0).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("bad", ["decreasing", "negative", "behind", "too long", "keys behind"])
def test_packed_attention_bad_offsets_are_reported(ctx, dtype, bad):
    """The sequence is skipped, the others are computed, and the status word says so once."""
    vit, m = ctx
    p = Packed(vit, [40, 50, 60], [40, 50, 60], 2, 2, 64, dtype, trail=30)
    good = p.forward(m)
    good_grads = p.backward(m, *good)
    m.check()
    q_off, k_off = p.q_off.clone(), p.k_off.clone()
    keep = 1
    if bad == "decreasing":
        p.q_off[2] = 30                     # sequence 1 runs backwards (and 2 starts inside it: 120 long)
    elif bad == "negative":
        p.q_off[0] = -7
        keep = 2
    elif bad == "behind":
        p.q_off[3] = p.q_rows + 1
        keep = 0
    elif bad == "too long":
        p.q_off[3] = p.q_rows               # inside the buffer, but longer than max_q
        keep = 0
    else:
        p.k_off[3] = p.k_rows + 100
        keep = 0
    if bad == "decreasing":
        keep = 0
    qs, ks = [(slice(int(a), int(b)), slice(int(c), int(e))) for a, b, c, e in zip(q_off, q_off[1:], k_off, k_off[1:])][keep]
    out, lse = p.forward(m)
    with pytest.raises(vit.VitError) as e:
        m.check()
    assert e.value.status == vit.VIT_ERR_OFFSETS
    m.check()
    assert torch.equal(out[qs], good[0][qs]) and torch.equal(lse[:, qs], good[1][:, qs])
    dq, dkv = p.backward(m, *good)
    with pytest.raises(vit.VitError) as e:
        m.check()
    assert e.value.status == vit.VIT_ERR_OFFSETS
    assert torch.equal(dq[qs], good_grads[0][qs]) and torch.equal(dkv[ks], good_grads[1][ks])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("ql,kl,heads,kv,d", [([1, 1, 1], [1, 1, 1], 3, 1, 96), ([40, 513, 3, 70], [1, 1, 0, 65], 2, 2, 64),
                                             ([2600, 2600], [1, 1], 8, 1, 128)])
def test_packed_attention_of_one_key_passes_no_gradient_to_its_score(ctx, dtype, ql, kl, heads, kv, d):
    """The softmax of one number is 1: dq and dk are zero, and not a rounding; what is not a number stays so."""
    vit, m = ctx
    p = Packed(vit, ql, kl, heads, kv, d, dtype, seed=6)
    out, lse = p.forward(m)
    dq, dkv = p.backward(m, out, lse)
    m.check()
    p.check_backward(out, lse, dq, dkv)
    for (qs, ks), b in zip(p.sequences(), kl):
        if b == 1:
            assert (dq[qs, :heads * d] == 0).all() and (dkv[ks, :kv * d] == 0).all() and (dkv[ks, kv * d:2 * kv * d] != 0).any()
    qs, ks = next(p.sequences())
    p.v[ks] = float("nan")
    out, lse = p.forward(m)
    dq, dkv = p.backward(m, out, lse)
    m.check()
    assert torch.isnan(dq[qs, :heads * d]).all() and torch.isnan(dkv[ks, :kv * d]).all()


def test_packed_attention_gradients_against_differences(ctx):
    """Directional derivatives of the library's own forward pass in fp32."""
    vit, m = ctx
    p = Packed(vit, [37, 70], [37, 70], 2, 1, 48, torch.float32, seed=3, spread=0.7)
    out, lse = p.forward(m)
    dq, dkv = p.backward(m, out, lse)
    m.check()
    gen = _gen(17)
    for buf, grad, cols in ((p.qbuf, dq, slice(0, 96)), (p.kvbuf, dkv, slice(0, 48)), (p.kvbuf, dkv, slice(48, 96))):
        direction = _normal(gen, buf.shape[0], cols.stop - cols.start)
        kept = buf[:, cols].clone()

        def loss(step):
            buf[:, cols] = kept + step * direction
            o, _ = p.forward(m)
            m.check()
            buf[:, cols] = kept
            return float((o[:, :96].double() * p.dout.double()).sum())

        h = 2.0 ** -7
        near, far = (loss(h) - loss(-h)) / (2 * h), (loss(2 * h) - loss(-2 * h)) / (4 * h)
        want = float((grad[:, cols].double() * direction.double()).sum())
        # the error of a central difference goes with h^2: the two steps differ by three times the nearer one's;
        # the loss is a sum of about 1e4 terms of 0.1, each rounded to 2^-22 or so: 1e-6 over 2 h
        assert abs(near - want) <= abs(far - near) + 1e-3 * max(1.0, abs(want)) * 0.1 + 4e-4, (near, far, want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_packed_attention_bad_offsets_where_long_walks_are_shared(ctx, dtype):
    vit, m = ctx
    p = Packed(vit, [1300, 600, 530], [1300, 600, 530], 8, 2, 64, dtype, trail=8)
    good = p.forward(m)
    m.check()
    p.k_off[3] = p.k_rows + 1
    out, lse = p.forward(m)
    dq, dkv = p.backward(m, *good)
    with pytest.raises(vit.VitError) as e:
        m.check()
    assert e.value.status == vit.VIT_ERR_OFFSETS
    assert torch.equal(out[:1900], good[0][:1900]) and torch.equal(lse[:, :1900], good[1][:, :1900])
    assert (out[1900:] == 33).all() and (lse[:, 1900:] == 33).all()
    # how the walks are cut into shares follows the lengths: the others' gradients are the definition's, and those of
    # this sequence are left alone
    p.ql, p.kl, p.covered_q, p.covered_k = p.ql[:2], p.kl[:2], slice(0, 1900), slice(0, 1900)
    p.check_backward(*good, dq, dkv)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("sequences,n", [(9700, 5), (513, 9), (700, 1)])
def test_packed_attention_of_many_short_sequences(ctx, dtype, sequences, n):
    """More sequences than a block looks up at a time, and more pieces than its table holds."""
    vit, m = ctx
    heads, d = 2, 32
    p = Packed(vit, [n] * sequences, [n] * sequences, heads, heads, d, dtype, trail=3)
    out, lse = p.forward(m)
    dq, dkv = p.backward(m, out, lse)
    m.check()
    half, width, rows = HALF[dtype], heads * d, sequences * n
    cut = lambda t: t[:rows].double().reshape(sequences, n, heads, d).transpose(1, 2)
    q, k, v, o, do = (cut(t) for t in (p.q, p.k, p.v, out[:, :width], p.dout))
    s = p.scale * q @ k.transpose(-1, -2)
    e = (d + 8) * 2.0 ** -24 * (p.scale * q.abs() @ k.abs().transpose(-1, -2)).max() + 2.0 ** -20
    w, want = torch.logsumexp(s, -1), torch.softmax(s, -1) @ v
    got_lse = lse[:, :rows].double().reshape(heads, sequences, n).transpose(0, 1)
    tol = half * want.abs() + (half * 1.01 + 2 * e + (n + 16) * 2.0 ** -24) * (torch.softmax(s, -1) @ v.abs())
    assert ((o - want).abs() <= tol).all()
    assert ((got_lse - w).abs() <= e + (n + 16) * 2.0 ** -24 + 2.0 ** -22 * w.abs()).all()
    prob = torch.exp(s - got_lse[..., None])
    ds = prob * (do @ v.transpose(-1, -2) - (do * o).sum(-1, keepdim=True))
    dds = ds.abs() * (half * 1.01 + 2 * e) + prob * (d + 8) * 2.0 ** -24 * (do.abs() @ v.abs().transpose(-1, -2) +
                                                                         (do * o).abs().sum(-1, keepdim=True))
    acc = (n + 16) * 2.0 ** -24
    spread = p.scale * (dds + acc * ds.abs())
    for got, exact, tol in ((cut(dq[:, :width]), p.scale * ds @ k, spread @ k.abs()),
                            (cut(dkv[:, :width]), p.scale * ds.transpose(-1, -2) @ q, spread.transpose(-1, -2) @ q.abs()),
                            (cut(dkv[:, width:2 * width]), prob.transpose(-1, -2) @ do,
                             ((half * 1.01 + 2 * e + acc) * prob).transpose(-1, -2) @ do.abs())):
        assert ((got - exact).abs() <= half * exact.abs() + tol).all()
    assert (out[rows:] == 33).all() and (dq[rows:] == 33).all() and (dkv[rows:] == 33).all()


def test_packed_attention_shares_over_many_sequences(ctx):
    """More sequences than are looked at together, where the blocks share the tiles of the gradients."""
    vit, m = ctx
    rng = np.random.default_rng(8)
    ql = [1000 if i % 50 == 7 else int(n) for i, n in enumerate(rng.integers(0, 41, 600))]
    kl = [128 if i % 50 == 7 else int(n) for i, n in enumerate(rng.integers(0, 129, 600))]
    p = Packed(vit, ql, kl, 1, 1, 64, torch.bfloat16, lead=2, trail=4)
    out, lse = p.forward(m)
    m.check()
    p.check_forward(out, lse)
    dq, dkv = p.backward(m, out, lse)
    m.check()
    p.check_backward(out, lse, dq, dkv)
    dq2, dkv2 = p.backward(m, out, lse)
    m.check()
    assert torch.equal(dq, dq2) and torch.equal(dkv, dkv2)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_far_apart(ctx, dtype):
    """Strides that put the rows behind 2^31 elements: the bits of the dense call."""
    vit, m = ctx
    ld, rows, heads, d = 2 ** 24 + 8, 150, 2, 64
    dt, width = _dt(vit, dtype), 2 * 64
    assert (rows - 20) * ld > 2 ** 31
    far = torch.empty(rows * ld, dtype=dtype, device="cuda").view(rows, ld)     # columns: q, k, v, out, dout, dq, dk, dv
    assert width * 8 <= ld
    block = lambda i: far[:, i * width:(i + 1) * width]
    gen = _gen(31)
    dense = [_normal(gen, rows, width, dtype=dtype) for _ in range(3)] + [torch.empty(rows, width, dtype=dtype, device="cuda")]
    dense += [_normal(gen, rows, width, dtype=dtype)] + [torch.empty_like(dense[0]) for _ in range(3)]
    for i, t in enumerate(dense):
        block(i).copy_(t)
    q_off = torch.tensor([0, 20, 150], dtype=torch.int32, device="cuda")
    one = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    lse = torch.empty(heads, rows, device="cuda")
    for off, q_rows, max_q in ((q_off, rows, 130), (one, 2, 1)):               # and with one query to a sequence
        problem = vit.make_attention_problem(2, heads, heads, d, q_rows, max_q, off.data_ptr(), rows, 130, q_off.data_ptr(), 0.125)
        n = vit.vit_attention_packed_bytes(dt, problem, True)
        ws = torch.empty(n, dtype=torch.uint8, device="cuda")
        for get, step in ((lambda i: dense[i], width), (block, ld)):
            q, k, v, o, do, dq, dk, dv = (get(i).data_ptr() for i in range(8))
            vit.vit_op_attention_packed(m.h, dt, problem, q, step, k, step, v, step, o, step, lse.data_ptr(), 0, 0)
            vit.vit_op_attention_packed_backward(m.h, dt, problem, q, step, k, step, v, step, o, step, lse.data_ptr(), do, step, dq, step,
                                                 dk, step, dv, step, ws.data_ptr(), n)
            m.check()
        for i in (3, 5):
            assert torch.equal(block(i)[:q_rows], dense[i][:q_rows])
        for i in (6, 7):
            assert torch.equal(block(i), dense[i])
    gains = 1 + _normal(gen, 2, d, scale=0.1)
    freqs, positions = _rope_inputs(gen, rows, (16, 16), 50)
    rope = vit.make_rope((16, 16), freqs.data_ptr(), positions.data_ptr())
    n = vit.vit_qk_norm_rope_backward_bytes(rows, 1, 1, d)
    ws, dg = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.empty(2, 2, d, device="cuda")
    for j, (get, step) in enumerate(((lambda i: dense[i], width), (block, ld))):
        x, y, z, dy, dx = (get(i).data_ptr() for i in (0, 1, 2, 4, 5))
        vit.vit_op_rope_axes(m.h, dt, rows, heads, d, rope, False, x, step, y, step)
        vit.vit_op_qk_norm_rope(m.h, dt, rows, 1, 1, d, gains[0].data_ptr(), gains[1].data_ptr(), EPS, rope, x, step, z, step)
        vit.vit_op_qk_norm_rope_backward(m.h, dt, rows, 1, 1, d, gains[0].data_ptr(), gains[1].data_ptr(), EPS, rope, x, step, dy, step,
                                         dx, step, dg[j, 0].data_ptr(), dg[j, 1].data_ptr(), ws.data_ptr(), n)
        m.check()
    for i in (1, 2, 5):
        assert torch.equal(block(i), dense[i])
    assert torch.equal(dg[0], dg[1])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_two_streams_at_once(ctx, dtype):
    """Calls on two streams, each with a workspace of its own, give the bits of calls one after the other."""
    vit, m = ctx
    problems = [Packed(vit, [700, 385], [700, 385], 4, 2, 80, dtype, seed=1), Packed(vit, [1, 1, 1], [577, 40, 1030], 4, 4, 64, dtype, seed=2),
                Packed(vit, [2100], [2100], 4, 1, 64, dtype, seed=3)]
    alone = []
    for p in problems:
        out, lse = p.forward(m)
        alone.append((out, lse, *p.backward(m, out, lse)))
        m.check()
    dt = _dt(vit, dtype)
    streams = [torch.cuda.Stream() for _ in problems]
    results, keep = [], []
    for p in problems:
        out, lse = torch.full_like(alone[len(results)][0], 33.0), torch.full_like(alone[len(results)][1], 33.0)
        results.append((out, lse, torch.full_like(p.qbuf, 33.0), torch.full_like(p.kvbuf, 33.0)))
        keep.append(torch.empty(vit.vit_attention_packed_bytes(dt, p.problem, True), dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    for _ in range(3):
        for p, s, (out, lse, dq, dkv), ws in zip(problems, streams, results, keep):
            kw, s = p.kv * p.d, s.cuda_stream
            ops = (p.q.data_ptr(), p.ldq, p.k.data_ptr(), p.ldkv, p.v.data_ptr(), p.ldkv)
            vit.vit_op_attention_packed(m.h, dt, p.problem, *ops, out.data_ptr(), out.stride(0), lse.data_ptr(), 0, 0, s)
            vit.vit_op_attention_packed_backward(m.h, dt, p.problem, *ops, out.data_ptr(), out.stride(0), lse.data_ptr(), p.dout.data_ptr(),
                                                 p.dout.stride(0), dq.data_ptr(), p.ldq, dkv.data_ptr(), p.ldkv, dkv[:, kw:].data_ptr(),
                                                 p.ldkv, ws.data_ptr(), ws.numel(), s)
    torch.cuda.synchronize()
    m.check()
    for a, b in zip(alone, results):
        for x, y in zip(a, b):
            assert torch.equal(x, y)


# ------------------------------------------------------------------------------- the layer, as it is used
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_layer_of_packed_images(ctx, dtype):
    """QKV buffer -> norm and rotation -> attention -> gradients back to the QKV buffer and the gains, on a stream."""
    vit, m = ctx
    gen = _gen(77)
    grids = [(14, 14), (9, 5), (1, 1), (20, 11)]
    lens = [a * b for a, b in grids]
    heads, kv, d, pairs = 4, 2, 64, (16, 16)
    rows, width = sum(lens), (heads + 2 * kv) * d
    positions = torch.cat([torch.stack(torch.meshgrid(torch.arange(a), torch.arange(b), indexing="ij")).flatten(1) for a, b in grids], 1)
    positions = positions.to(torch.int32).cuda().contiguous()
    freqs = torch.cat([100.0 ** (-torch.arange(16, device="cuda") / 16)] * 2).float()
    off = torch.tensor(np.cumsum([0] + lens), dtype=torch.int32, device="cuda")
    qkv = _normal(gen, rows, width, scale=1.5, dtype=dtype)
    dout = _normal(gen, rows, heads * d, scale=0.3, dtype=dtype)
    gains = 1 + _normal(gen, 2, d, scale=0.1)
    dt, nqk = _dt(vit, dtype), (heads + kv) * d
    rope = vit.make_rope(pairs, freqs.data_ptr(), positions.data_ptr())
    problem = vit.make_attention_problem(len(lens), heads, kv, d, rows, max(lens), off.data_ptr(), rows, max(lens), off.data_ptr(),
                                         1 / math.sqrt(d))
    qk, dqkv, out = torch.empty(rows, nqk, dtype=dtype, device="cuda"), torch.empty_like(qkv), torch.empty_like(dout)
    lse, dg = torch.empty(heads, rows, device="cuda"), torch.empty(2, d, device="cuda")
    nf, nb = (vit.vit_attention_packed_bytes(dt, problem, b) for b in (False, True))
    nn = vit.vit_qk_norm_rope_backward_bytes(rows, heads, kv, d)
    ws = torch.empty(max(nf, nb, nn), dtype=torch.uint8, device="cuda")
    es = qkv.element_size()

    def layer(s):
        vit.vit_op_qk_norm_rope(m.h, dt, rows, heads, kv, d, gains[0].data_ptr(), gains[1].data_ptr(), EPS, rope, qkv.data_ptr(), width,
                                qk.data_ptr(), nqk, s)
        v = qkv.data_ptr() + nqk * es
        q, k = qk.data_ptr(), qk.data_ptr() + heads * d * es
        vit.vit_op_attention_packed(m.h, dt, problem, q, nqk, k, nqk, v, width, out.data_ptr(), heads * d, lse.data_ptr(), ws.data_ptr(),
                                    ws.numel(), s)
        # gradients of the turned queries and keys and of the values land in the column blocks of one buffer
        vit.vit_op_attention_packed_backward(m.h, dt, problem, q, nqk, k, nqk, v, width, out.data_ptr(), heads * d, lse.data_ptr(),
                                             dout.data_ptr(), heads * d, dqkv.data_ptr(), width, dqkv.data_ptr() + heads * d * es, width,
                                             dqkv.data_ptr() + nqk * es, width, ws.data_ptr(), ws.numel(), s)
        vit.vit_op_qk_norm_rope_backward(m.h, dt, rows, heads, kv, d, gains[0].data_ptr(), gains[1].data_ptr(), EPS, rope, qkv.data_ptr(),
                                         width, dqkv.data_ptr(), width, dqkv.data_ptr(), width, dg[0].data_ptr(), dg[1].data_ptr(),
                                         ws.data_ptr(), ws.numel(), s)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    layer(side.cuda_stream)
    m.check(side)
    first = [t.clone() for t in (out, lse, dqkv, dg)]

    x = qkv.double().requires_grad_()
    g = [t.double().requires_grad_() for t in gains]
    qk64 = _norm_rope64(x[:, :nqk].unflatten(1, (heads + kv, d)), g, [heads, kv], pairs, freqs, positions, False)
    if dtype == torch.bfloat16:                    # the layer hands its queries and keys on in bf16
        qk64 = qk64 + (qk64.detach().to(dtype).double() - qk64.detach())
    want, begin = [], 0
    for n in lens:
        at = slice(begin, begin + n)
        for h in range(heads):
            s = qk64[at, h] @ qk64[at, heads + h // 2].t() / math.sqrt(d)
            want.append(torch.softmax(s, 1) @ x[at, nqk + h // 2 * d:nqk + (h // 2 + 1) * d])
        begin += n
    parts, i = [], 0
    for n in lens:
        parts.append(torch.cat(want[i:i + heads], 1))
        i += heads
    want = torch.cat(parts)
    grads = torch.autograd.grad(want, [x] + g, dout.double())
    # norms of the differences: every intermediate in bf16 (queries, keys, probabilities, score gradients, out, the
    # gradients handed from one operator to the next) adds a relative 2^-8 at most, and there are six of them
    bound = 6 * 2.0 ** -8 if dtype == torch.bfloat16 else 1e-5
    for got, exact in ((out, want.detach()), (dqkv, grads[0]), (dg[0], grads[1]), (dg[1], grads[2])):
        assert float((got.double() - exact).norm() / exact.norm()) <= bound

    # captured and replayed on new inputs: what a direct call gives on them
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        layer(torch.cuda.current_stream().cuda_stream)
    qkv.copy_(_normal(gen, rows, width, scale=1.5, dtype=dtype))
    graph.replay()
    m.check()
    replayed = [t.clone() for t in (out, lse, dqkv, dg)]
    layer(0)
    m.check()
    for a, b, c in zip(replayed, (out, lse, dqkv, dg), first):
        assert torch.equal(a, b) and not torch.equal(a, c)


# ------------------------------------------------------------------------------- refusals
def test_packed_ops_refuse(ctx):
    vit, m = ctx
    x = torch.zeros(64, 256, dtype=torch.bfloat16, device="cuda")
    y = torch.zeros(64, 256, dtype=torch.bfloat16, device="cuda")
    f = torch.zeros(256, device="cuda")
    pos = torch.zeros(2, 64, dtype=torch.int32, device="cuda")
    off = torch.tensor([0, 64], dtype=torch.int32, device="cuda")
    xp, yp, fp, pp = x.data_ptr(), y.data_ptr(), f.data_ptr(), pos.data_ptr()
    before = m.launches

    def refused(status, call, *args):
        with pytest.raises(vit.VitError) as e:
            call(*args)
        assert e.value.status == status

    bad = vit.VIT_ERR_INVALID_ARG
    good = vit.make_rope((8, 8), fp, pp)
    for args in [(5, 64, 2, 64, good, 0, xp, 256, yp, 256), (0, -1, 2, 64, good, 0, xp, 256, yp, 256), (0, 64, 0, 64, good, 0, xp, 256, yp, 256),
                 (0, 64, 2, 24, good, 0, xp, 256, yp, 256), (0, 64, 1, 144, good, 0, xp, 256, yp, 256), (0, 64, 2, 64, None, 0, xp, 256, yp, 256),
                 (0, 64, 2, 64, vit.make_rope((30, 8), fp, pp), 0, xp, 256, yp, 256), (0, 64, 2, 64, vit.make_rope((-1, 8), fp, pp), 0, xp, 256, yp, 256),
                 (0, 64, 2, 64, vit.make_rope((8, 8), 0, pp), 0, xp, 256, yp, 256), (0, 64, 2, 64, good, 0, xp, 120, yp, 256),
                 (0, 64, 2, 64, good, 0, xp, 132, yp, 256), (0, 64, 2, 64, good, 0, xp + 2, 256, yp, 256), (0, 64, 2, 64, good, 0, 0, 256, yp, 256),
                 (0, 32, 2, 64, good, 0, xp, 256, xp + 128, 256), (0, 32, 2, 64, good, 0, xp, 256, xp + 512, 256),
                 (0, 1, 2, 64, good, 0, xp, 256, pp, 256), (0, 1, 2, 64, good, 0, xp, 256, fp, 256),
                 (0, 1, 2 ** 28, 64, good, 0, xp, 2 ** 34, yp, 2 ** 34)]:
        refused(bad, vit.vit_op_rope_axes, m.h, *args)
    norm = (0, 64, 1, 1, 64, fp, fp, EPS, good)
    for i, v in [(1, -1), (2, -1), (4, 40), (5, 0), (6, fp + 4), (7, -1.0), (7, float("nan"))]:
        args = list(norm)
        args[i] = v
        refused(bad, vit.vit_op_qk_norm_rope, m.h, *args, xp, 256, yp, 256)
    refused(bad, vit.vit_op_qk_norm_rope, m.h, 0, 1, *norm[2:], xp, 256, fp, 256)
    n = vit.vit_qk_norm_rope_backward_bytes(64, 1, 1, 64)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    dg = torch.empty(2, 64, device="cuda")
    dx = torch.zeros_like(x)
    tail = [xp, 256, yp, 256, dx.data_ptr(), 256, dg[0].data_ptr(), dg[1].data_ptr(), ws.data_ptr(), n]
    refused(vit.VIT_ERR_WORKSPACE, vit.vit_op_qk_norm_rope_backward, m.h, *norm, *tail[:-1], n - 1)
    for i, v in [(6, 0), (7, dg[0].data_ptr()), (8, 0), (4, xp + 16), (6, dx.data_ptr()), (8, dx.data_ptr()), (6, fp),
                 (7, pp)]:
        args = list(tail)
        args[i] = v
        refused(bad, vit.vit_op_qk_norm_rope_backward, m.h, *norm, *args)

    o, lse = torch.zeros_like(x), torch.zeros(4, 64, device="cuda")
    base = [1, 4, 2, 64, 64, 64, off.data_ptr(), 64, 64, off.data_ptr(), 0.125]
    kv = torch.zeros(64, 256, dtype=torch.bfloat16, device="cuda")

    def forward(problem, dtype=0, q=xp, ldq=256, out=o.data_ptr(), l=lse.data_ptr()):
        vit.vit_op_attention_packed(m.h, dtype, problem, q, ldq, kv.data_ptr(), 256, kv[:, 128:].data_ptr(), 256, out, 256, l, ws.data_ptr(),
                                    ws.numel())

    for i, v in [(0, -1), (1, 0), (2, 3), (2, 0), (3, 40), (3, 144), (4, -1), (5, -1), (6, 0), (9, off.data_ptr() + 2), (10, 0.0), (10, -1.0),
                 (10, float("inf")), (10, float("nan"))]:
        args = list(base)
        args[i] = v
        refused(bad, forward, vit.make_attention_problem(*args))
    ok = vit.make_attention_problem(*base)
    refused(bad, forward, ok, 7)
    for kw in (dict(q=xp + 2), dict(q=0), dict(ldq=252), dict(ldq=248), dict(out=xp), dict(out=kv.data_ptr()), dict(l=0), dict(l=o.data_ptr()),
               dict(l=off.data_ptr())):
        refused(bad, lambda: forward(ok, **kw))
    huge = vit.make_attention_problem(2 ** 30, *base[1:])
    refused(vit.VIT_ERR_TOO_LARGE, forward, huge)
    nb = vit.vit_attention_packed_bytes(0, ok, True)
    big = torch.empty(nb, dtype=torch.uint8, device="cuda")
    dq, dkv = torch.zeros_like(x), torch.zeros_like(kv)
    rest = [xp, 256, kv.data_ptr(), 256, kv[:, 128:].data_ptr(), 256, o.data_ptr(), 256, lse.data_ptr(), yp, 256, dq.data_ptr(), 256,
            dkv.data_ptr(), 256, dkv[:, 128:].data_ptr(), 256, big.data_ptr(), nb]
    refused(vit.VIT_ERR_WORKSPACE, vit.vit_op_attention_packed_backward, m.h, 0, ok, *rest[:-1], nb - 1)
    for i, v in [(0, 0), (8, 0), (9, yp + 2), (11, xp), (13, dkv.data_ptr() + 64), (15, dq.data_ptr()), (17, 0), (17, dq.data_ptr()),
                 (17, off.data_ptr())]:
        args = list(rest)
        args[i] = v
        refused(bad, vit.vit_op_attention_packed_backward, m.h, 0, ok, *args)
    assert m.launches == before


def test_packed_ops_of_nothing(ctx):
    vit, m = ctx
    off = torch.zeros(1, dtype=torch.int32, device="cuda")
    p = vit.make_attention_problem(0, 2, 2, 64, 0, 0, off.data_ptr(), 0, 0, off.data_ptr(), 0.125)
    vit.vit_op_attention_packed(m.h, 0, p, 0, 128, 0, 128, 0, 128, 0, 128, 0, 0, 0)
    vit.vit_op_attention_packed_backward(m.h, 0, p, 0, 128, 0, 128, 0, 128, 0, 128, 0, 0, 128, 0, 128, 0, 128, 0, 128, 0, 0)
    m.check()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("last", [30, -1, -2 ** 31])
def test_packed_attention_bad_last_offset_leaves_the_others_alone(ctx, dtype, last):
    """Whatever the last offset says, the gradients of the sequences before the last one are those of the good call."""
    vit, m = ctx
    p = Packed(vit, [40, 50, 60], [40, 50, 60], 4, 2, 64, dtype, trail=30)
    good = p.forward(m)
    good_grads = p.backward(m, *good)
    m.check()
    for off in (p.q_off, p.k_off):
        off[3] = last
    out, lse = p.forward(m)
    dq, dkv = p.backward(m, *good)              # (its scratch holds NaN)
    with pytest.raises(vit.VitError) as e:
        m.check()
    assert e.value.status == vit.VIT_ERR_OFFSETS
    assert torch.equal(out[:90], good[0][:90]) and torch.equal(lse[:, :90], good[1][:, :90])
    assert torch.equal(dq[:90], good_grads[0][:90]) and torch.equal(dkv[:90], good_grads[1][:90])
    for t in (out, dq, dkv):
        assert (t[90:] == 33).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_packed_attention_sequence_behind_the_last_offset(ctx, dtype):
    """After a step backwards the last offset is not the largest: what lies behind it is still a sequence's."""
    vit, m = ctx
    p = Packed(vit, [60, 40], [60, 40], 4, 2, 64, dtype, lead=50)
    parts = torch.tensor([90, 150, 50, 90], dtype=torch.int32, device="cuda")      # rows 90 ... 149, none, rows 50 ... 89
    p.q_off, p.k_off = parts, parts.clone()
    p.problem = vit.make_attention_problem(3, 4, 2, 64, 150, 60, p.q_off.data_ptr(), 150, 60, p.k_off.data_ptr(), p.scale)
    p.sequences = lambda: [(slice(90, 150),) * 2, (slice(50, 90),) * 2]
    p.covered_q = p.covered_k = slice(50, 150)
    out, lse = p.forward(m)
    dq, dkv = p.backward(m, out, lse)
    with pytest.raises(vit.VitError) as e:
        m.check()
    assert e.value.status == vit.VIT_ERR_OFFSETS
    p.check_forward(out, lse)
    p.check_backward(out, lse, dq, dkv)


@pytest.mark.parametrize("rows,hq,hk,d,pairs", [
    # heads that leave places of a warp empty: rotation of a part, none, and of all channels
    (33, 16, 4, 80, (11, 9)), (40, 3, 1, 112, ()), (21, 6, 3, 64, (9, 8)), (300, 5, 2, 48, (8, 8)), (33, 16, 4, 80, (20, 20)), (5000, 3, 2, 64, (16, 16)),
])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_qk_norm_rope_with_eps_of_zero(ctx, rows, hq, hk, d, pairs, interleaved, dtype):
    """Without eps the norm of every head that is not zero is finite, and so are all gradients."""
    vit, m = ctx
    gen = _gen(rows + d)
    heads, width = hq + hk, (hq + hk) * d
    x, dy = _normal(gen, rows, width, scale=1.3, dtype=dtype), _normal(gen, rows, width, scale=0.5, dtype=dtype)
    gains = 1 + _normal(gen, 2, d, scale=0.2)
    rope = freqs = positions = None
    if pairs:
        freqs, positions = _rope_inputs(gen, rows, pairs, 50)
        rope = vit.make_rope(pairs, freqs.data_ptr(), positions.data_ptr(), interleaved)
    n = vit.vit_qk_norm_rope_backward_bytes(rows, hq, hk, d)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
    y, dx, dg = torch.empty_like(x), torch.empty_like(x), torch.empty(2, d, device="cuda")
    args = (m.h, _dt(vit, dtype), rows, hq, hk, d, gains[0].data_ptr(), gains[1].data_ptr(), 0.0, rope)
    vit.vit_op_qk_norm_rope(*args, x.data_ptr(), width, y.data_ptr(), width)
    vit.vit_op_qk_norm_rope_backward(*args, x.data_ptr(), width, dy.data_ptr(), width, dx.data_ptr(), width, dg[0].data_ptr(),
                                     dg[1].data_ptr(), ws.data_ptr(), n)
    m.check()
    x64, dy64 = (t.double().unflatten(1, (heads, d)) for t in (x, dy))
    x64.requires_grad_()
    g64 = [g.double().requires_grad_() for g in gains]
    rstd = 1 / (x64 * x64).mean(-1, keepdim=True).sqrt()
    scaled = torch.cat([part * g for part, g in zip((x64 * rstd).split([hq, hk], 1), g64)], 1)
    want = _turn64(scaled, pairs, freqs, positions, interleaved) if pairs else scaled
    wx, *wg = torch.autograd.grad(want, [x64] + g64, dy64)
    want, rstd, scaled = want.detach(), rstd.detach(), scaled.detach()
    # the bounds of the test with eps: a sum of d squares, a root, a division; the rotation mixes two channels of a head
    rel32 = (d + 24) * 2.0 ** -24
    tol = HALF[dtype] * want.abs() + rel32 * scaled.abs().amax(-1, keepdim=True) * math.sqrt(2)
    assert ((y.double().unflatten(1, (heads, d)) - want).abs() <= tol).all()
    xh, gain_max = (x64.detach() * rstd).abs(), gains.abs().max().double()
    u = dy64.abs().amax(-1, keepdim=True) * math.sqrt(2)
    tol = HALF[dtype] * wx.abs() + 4 * rel32 * rstd * (gain_max * u + xh * gain_max * u * xh.mean(-1, keepdim=True))
    assert ((dx.double().unflatten(1, (heads, d)) - wx).abs() <= tol).all()
    for got, exact, part, count in zip(dg, wg, (u * xh).split([hq, hk], 1), (hq, hk)):
        tol = (rel32 * 4 + 2.0 ** -24 * min(rows * count, 4096)) * part.sum((0, 1))
        assert ((got.double() - exact).abs() <= tol).all()


@pytest.mark.parametrize("ql,kl,heads,kv", [([197, 70], None, 2, 1), ([1300, 20], None, 8, 2), ([1, 1], [577, 40], 2, 2), ([130], None, 1, 1)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_packed_attention_without_a_bound_of_the_lengths(ctx, ql, kl, heads, kv, dtype):
    """max_q and max_k may be anything that is long enough, the largest number among them."""
    vit, m = ctx
    p = Packed(vit, ql, kl or ql, heads, kv, 64, dtype, lead=2, trail=6)
    for max_q, max_k in ((2 ** 31 - 1, 2 ** 31 - 1), (2 ** 31 - 40, 2 ** 31 - 1), (p.q_rows, 2 ** 31 - 33)):
        p.problem.max_q, p.problem.max_k = max_q, max_k
        out, lse = p.forward(m)
        dq, dkv = p.backward(m, out, lse)
        m.check()
        p.check_forward(out, lse)
        p.check_backward(out, lse, dq, dkv)


def test_packed_attention_refuses_rows_that_it_cannot_count(ctx):
    vit, m = ctx
    x = torch.zeros(64, 64, dtype=torch.bfloat16, device="cuda")
    off = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    a, o, before = x.data_ptr(), off.data_ptr(), m.launches
    for q_rows, k_rows in ((2 ** 31 - 1, 1), (1, 2 ** 31 - 1), (2 ** 31 - 1024, 1)):
        p = vit.make_attention_problem(1, 1, 1, 64, q_rows, 1, o, k_rows, 1, o, 0.125)
        for call in (lambda: vit.vit_op_attention_packed(m.h, 0, p, a, 64, a, 64, a, 64, a, 64, a, 0, 0),
                     lambda: vit.vit_op_attention_packed_backward(m.h, 0, p, a, 64, a, 64, a, 64, a, 64, a, a, 64, a, 64, a, 64, a, 64, 0, 0)):
            with pytest.raises(vit.VitError) as e:
                call()
            assert e.value.status == vit.VIT_ERR_TOO_LARGE
    assert m.launches == before


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_packed_attention_bad_offsets_are_reported_where_nothing_is_computed(ctx, dtype):
    """No rows, or a bound of zero, but offsets that say otherwise; nothing is said where they fit."""
    vit, m = ctx
    dt, d = _dt(vit, dtype), 64
    x, lse = torch.full((20, d), 33.0, dtype=dtype, device="cuda"), torch.full((1, 20), 33.0, device="cuda")
    grads = torch.full((3, 20, d), 33.0, dtype=dtype, device="cuda")
    empty, some = (torch.tensor(o, dtype=torch.int32, device="cuda") for o in ([0, 0, 0], [0, 5, 5]))
    low = torch.tensor([-1, -1, -1], dtype=torch.int32, device="cuda")
    for q_off, k_off, q_rows, max_q, k_rows, max_k, ok in [
            (empty, empty, 20, 0, 20, 0, True), (empty, empty, 0, 0, 0, 0, True), (some, empty, 20, 0, 20, 0, False), (some, empty, 0, 5, 0, 0, False),
            (empty, some, 20, 0, 20, 0, False), (empty, low, 0, 0, 0, 0, False), (low, empty, 20, 0, 20, 0, False), (some, some, 20, 0, 20, 5, False)]:
        problem = vit.make_attention_problem(2, 1, 1, d, q_rows, max_q, q_off.data_ptr(), k_rows, max_k, k_off.data_ptr(), 0.125)
        n = vit.vit_attention_packed_bytes(dt, problem, True)
        ws = torch.empty(n + 16, dtype=torch.uint8, device="cuda")
        q, out = x.data_ptr(), grads[0].data_ptr()

        def forward():
            vit.vit_op_attention_packed(m.h, dt, problem, q, d, q, d, q, d, out, d, lse.data_ptr(), 0, 0)

        def backward():
            vit.vit_op_attention_packed_backward(m.h, dt, problem, q, d, q, d, q, d, q, d, lse.data_ptr(), q, d, grads[0].data_ptr(), d,
                                                 grads[1].data_ptr(), d, grads[2].data_ptr(), d, ws.data_ptr(), n)

        for call in (forward, backward):
            call()
            if ok:
                m.check()
                continue
            with pytest.raises(vit.VitError) as e:
                m.check()
            assert e.value.status == vit.VIT_ERR_OFFSETS
            m.check()
        assert (lse == 33).all() and (grads == 33).all()


def _unit_turns(positions, freqs):
    """cos and sin of position * freq, the angle reduced in exact fractions."""
    two_pi = 2 * Fraction(3141592653589793238462643383279502884197169399375105820974944, 10 ** 60)
    unit = np.empty((len(positions), len(freqs), 2))
    for i, position in enumerate(positions):
        for j, freq in enumerate(freqs):
            angle = Fraction(position) * Fraction(freq)
            angle -= two_pi * round(angle / two_pi)
            unit[i, j] = math.cos(angle), math.sin(angle)
    return torch.tensor(unit, device="cuda")


@pytest.mark.parametrize("d", [16, 32])                # all channels turn, or half of them
def test_rope_axes_at_the_ends_of_the_range(ctx, d):
    """The whole range of positions, with frequencies from far below 1 to far above, keeps its angle."""
    vit, m = ctx
    rng = np.random.default_rng(3)
    far = [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 2, -2 ** 31 + 1, 2 ** 29 + 1, -2 ** 30 - 1, 0, 1]
    positions = far + [int(s) * (2 ** 31 - 1 - int(n)) for s, n in zip(rng.choice([-1, 1], 248), rng.integers(0, 2 ** 20, 248))]
    freqs = torch.tensor([1.0, 0.9, 0.77, 1e-4, 3.3, 31.4, 100.0, 1e6], device="cuda")
    where = torch.tensor([positions], dtype=torch.int32, device="cuda")
    rows = len(positions)
    x, y = torch.zeros(rows, d, device="cuda"), torch.empty(rows, d, device="cuda")
    x[:, :8] = 1                                       # pair i is (1, 0): its turn is (cos, sin)
    want = _unit_turns(positions, [float(f) for f in freqs])
    rope = vit.make_rope((8,), freqs.data_ptr(), where.data_ptr())
    for inverse in (False, True):
        vit.vit_op_rope_axes(m.h, vit.VIT_FP32, rows, 1, d, rope, inverse, x.data_ptr(), d, y.data_ptr(), d)
        m.check()
        # the remaining half turns, at most 1, are rounded once (pi 2^-25 as an angle); 2 ulp of the functions
        tol = (math.pi / 2 + 2) * 2.0 ** -24
        assert ((y[:, :8].double() - want[..., 0]).abs() <= tol).all()
        assert ((y[:, 8:16].double() - (-1 if inverse else 1) * want[..., 1]).abs() <= tol).all()


def test_rope_of_no_rows_or_no_pairs(ctx):
    """Empty positions and frequencies have no address; nothing of them is read."""
    vit, m = ctx
    g, dg = torch.ones(32, device="cuda"), torch.full((2, 32), float("nan"), device="cuda")
    freqs = torch.ones(16, device="cuda")
    ws = torch.empty(vit.vit_qk_norm_rope_backward_bytes(3, 1, 1, 32), dtype=torch.uint8, device="cuda")
    for rows, rope in ((0, vit.make_rope((8, 8), freqs.data_ptr(), 0)), (0, vit.make_rope((0, 0), 0, 0)), (3, vit.make_rope((0,), 0, 0))):
        x = _normal(_gen(2), rows, 64)
        y, z, dx = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
        args = (m.h, vit.VIT_FP32, rows, 1, 1, 32, g.data_ptr(), g.data_ptr(), EPS)
        vit.vit_op_rope_axes(m.h, vit.VIT_FP32, rows, 2, 32, rope, False, x.data_ptr(), 64, y.data_ptr(), 64)
        vit.vit_op_qk_norm_rope(*args, rope, x.data_ptr(), 64, y.data_ptr(), 64)
        vit.vit_op_qk_norm_rope_backward(*args, rope, x.data_ptr(), 64, x.data_ptr(), 64, dx.data_ptr(), 64, dg[0].data_ptr(), dg[1].data_ptr(),
                                         ws.data_ptr(), ws.numel())
        vit.vit_op_qk_norm_rope(*args, None, x.data_ptr(), 64, z.data_ptr(), 64)
        m.check()
        assert torch.equal(y, z) and torch.isfinite(dg).all() and ((dg == 0).all() if rows == 0 else torch.isfinite(dx).all())
        vit.vit_op_rope_axes(m.h, vit.VIT_FP32, rows, 2, 32, rope, False, x.data_ptr(), 64, y.data_ptr(), 64)
        m.check()
        assert torch.equal(y, x)
    for rope in (vit.make_rope((8, 8), freqs.data_ptr(), 0), vit.make_rope((8, 8), 0, freqs.data_ptr())):
        with pytest.raises(vit.VitError) as e:
            vit.vit_op_rope_axes(m.h, vit.VIT_FP32, 3, 2, 32, rope, False, x.data_ptr(), 64, y.data_ptr(), 64)
        assert e.value.status == vit.VIT_ERR_INVALID_ARG
