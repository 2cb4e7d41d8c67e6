"""The operators of an attention layer over packed images, measured one call at a time.

A batch of images of different sizes is one row-major buffer of tokens, image after image, with an
array of offsets; a token has a position on each of one to four axes (row and column of its patch,
frame of a video).  The cases are the calls that such a layer makes:

  rope_axes              rotation of channel pairs by the token's positions, or back
  qk_norm_rope           root-mean-square norm of every query and key head, gain, rotation
  qk_norm_rope_backward  its gradients (of the projections and of the two gains)
  attention              softmax attention of each image's queries over its keys, and the rows' log-sum-exp
  attention_backward     its gradients, from the saved output and log-sum-exp

`run` computes the plain form in torch where `own` is false and calls the library where it is true.
"""
import functools
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
HEAD_SIZES = (16, 32, 48, 64, 80, 96, 112, 128)
EPS = 1e-6


# ------------------------------------------------------------------------------------ the cases
def listed():
    return [
        # one 224 x 224 image of the tiny model: the smallest call, all latency
        dict(name="rope one image", op="rope_axes", dtype="bf16", rows=197, heads=6, d=64, pairs="16,16", interleaved=False,
             inverse=True, far=14),
        # queries and keys of four clips of 16 frames of 24 x 24 patches, far into a long video
        dict(name="rope video", op="rope_axes", dtype="bf16", rows=36864, heads=24, d=128, pairs="16,24,24", interleaved=True,
             inverse=False, far=1000000),
        # a layer of ViT-H/14 on 128 images
        dict(name="norm+rope huge14", op="qk_norm_rope", dtype="bf16", rows=32896, q_heads=16, k_heads=16, d=80, pairs="20,20",
             interleaved=False, far=16),
        # one 384 x 384 image at patch 16 in the fp32 mode, shared key heads, part of the head turned
        dict(name="norm+rope fp32 one image", op="qk_norm_rope", dtype="fp32", rows=577, q_heads=12, k_heads=3, d=64, pairs="11,12",
             interleaved=True, far=24),
        # fine-tuning ViT-L/16 on 64 images
        dict(name="norm+rope backward large16", op="qk_norm_rope_backward", dtype="bf16", rows=12608, q_heads=16, k_heads=16, d=64,
             pairs="16,16", interleaved=False, far=14),
        # fine-tuning in fp32 on a few odd-sized images
        dict(name="norm+rope backward fp32", op="qk_norm_rope_backward", dtype="fp32", rows=1531, q_heads=9, k_heads=3, d=48,
             pairs="8,7,8", interleaved=True, far=100),
        # a layer of ViT-B/16 on 64 images of one size
        dict(name="attention base16", op="attention", dtype="bf16", sequences=64, heads=12, kv_heads=12, d=64, q_len=197, k_len=197,
             cross=False, ragged=False),
        # a dozen images at their native resolution, up to 672 x 672 at patch 14, ViT-H head size
        dict(name="attention native sizes", op="attention", dtype="bf16", sequences=12, heads=16, kv_heads=16, d=80, q_len=2305,
             k_len=2305, cross=False, ragged=True),
        # attention pooling of two images when served: one learned query over each image's tokens
        dict(name="attention pooling", op="attention", dtype="bf16", sequences=2, heads=16, kv_heads=16, d=64, q_len=1, k_len=1025,
             cross=True, ragged=False),
        # fine-tuning ViT-L/16 on 64 images
        dict(name="attention backward large16", op="attention_backward", dtype="bf16", sequences=64, heads=16, kv_heads=16, d=64,
             q_len=197, k_len=197, cross=False, ragged=False),
        # fine-tuning on a few very large images with shared key heads
        dict(name="attention backward long", op="attention_backward", dtype="bf16", sequences=4, heads=8, kv_heads=2, d=128,
             q_len=4097, k_len=4097, cross=False, ragged=True),
        # a gradient check of a small layer in the fp32 mode
        dict(name="attention backward fp32", op="attention_backward", dtype="fp32", sequences=5, heads=4, kv_heads=4, d=80, q_len=257,
             k_len=257, cross=False, ragged=True),
    ]


def _log_uniform(rng, low, high):
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 1))) - 0.5))))


def draw(rng):
    op = rng.choice(["rope_axes", "qk_norm_rope", "qk_norm_rope_backward", "attention", "attention", "attention_backward",
                     "attention_backward"])
    d = rng.choice(HEAD_SIZES)
    dtype = "bf16" if rng.random() < 0.75 else "fp32"
    if op.startswith("attention"):
        kv_heads = rng.randint(1, 16)
        heads = kv_heads * (1 if rng.random() < 0.6 else rng.randint(2, 4))
        cross = rng.random() < 0.3
        q_len = _log_uniform(rng, 1, 4097)
        k_len = _log_uniform(rng, 1, 4097) if cross else q_len
        if cross and rng.random() < 0.3:
            q_len = 1
        sequences = _log_uniform(rng, 1, 96)
        most = 1.6e8 if dtype == "bf16" else 2.5e7       # scores of one pass
        sequences = max(1, min(sequences, int(most / (heads * q_len * k_len))))
        while heads * q_len * k_len > most and heads > kv_heads:
            heads -= kv_heads
        while heads * q_len * k_len > most:
            q_len, k_len = max(1, q_len * 2 // 3), max(1, k_len * 2 // 3)
        case = dict(op=op, dtype=dtype, sequences=sequences, heads=heads, kv_heads=kv_heads, d=d, q_len=q_len, k_len=k_len,
                    cross=cross, ragged=rng.random() < 0.6)
        while work(case)["bytes"] > 4e8:
            case["sequences"] = case["sequences"] * 2 // 3
        return case
    axes = rng.randint(1, 4)
    turned = rng.randint(axes, d // 2) if rng.random() < 0.5 else d // 2
    cuts = sorted(rng.sample(range(1, turned), axes - 1))
    pairs = ",".join(str(b - a) for a, b in zip([0] + cuts, cuts + [turned]))
    case = dict(op=op, dtype=dtype, rows=_log_uniform(rng, 1, 30000), d=d, pairs=pairs, interleaved=rng.random() < 0.5,
                far=_log_uniform(rng, 1, 1000000))
    if op == "rope_axes":
        case.update(heads=rng.randint(1, 24), inverse=rng.random() < 0.5)
    else:
        k_heads = rng.randint(1, 12)
        case.update(q_heads=k_heads * rng.randint(1, 2), k_heads=k_heads)
    while work(case)["bytes"] > 4e8:
        case["rows"] = case["rows"] * 2 // 3
    return case


def _lengths(case):
    """Query and key lengths of the sequences: the case's own, whatever the seed."""
    n = case["sequences"]
    if not case["ragged"]:
        return [case["q_len"]] * n, [case["k_len"]] * n
    rng = random.Random("%d %d %d" % (n, case["q_len"], case["k_len"]))

    def some(most):
        lengths = [most] + [rng.randint((most + 3) // 4, most) for _ in range(n - 1)]
        if n >= 4:
            lengths[rng.randint(1, n - 1)] = 0           # an image that a filter left empty
        return lengths

    if case["cross"]:
        return [case["q_len"]] * n, some(case["k_len"])
    lengths = some(case["q_len"])
    return lengths, lengths


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"].startswith("attention"):
        ql, kl = _lengths(case)
        q = sum(ql) * case["heads"] * case["d"] * size
        k = sum(kl) * case["kv_heads"] * case["d"] * size
        lse = sum(ql) * case["heads"] * 4
        product = 2 * case["d"] * case["heads"] * sum(a * b for a, b in zip(ql, kl))
        if case["op"] == "attention":
            return {"bytes": 2 * q + 2 * k + lse, "flops": 2 * product}
        return {"bytes": 4 * q + 4 * k + lse, "flops": 5 * product}
    heads = case["heads"] if case["op"] == "rope_axes" else case["q_heads"] + case["k_heads"]
    pairs = [int(p) for p in case["pairs"].split(",")]
    values = case["rows"] * heads * case["d"]
    tables = len(pairs) * case["rows"] * 4 + sum(pairs) * 4
    if case["op"] == "rope_axes":
        return {"bytes": 2 * values * size + tables, "flops": 6 * case["rows"] * heads * sum(pairs)}
    if case["op"] == "qk_norm_rope":
        return {"bytes": 2 * values * size + tables + 2 * case["d"] * 4, "flops": 7 * values}
    return {"bytes": 3 * values * size + tables + 4 * case["d"] * 4, "flops": 14 * values}


# ------------------------------------------------------------------------------------ the inputs
def _positions(case, gen):
    """Positions of the tokens on each axis: a raster scan from a random start up to `far`."""
    axes = len(case["pairs"].split(","))
    at = torch.arange(case["rows"], device="cuda")
    per = max(2, int(round(case["rows"] ** (1 / axes))))
    start = torch.randint(0, case["far"] + 1, (axes, 1), device="cuda", generator=gen)
    steps = torch.stack([(at // per ** (axes - 1 - a)) % per if a else at // per ** (axes - 1) for a in range(axes)])
    return (start + steps).to(torch.int32).contiguous()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = DTYPES[case["dtype"]]

    def normal(*shape, scale=1.0):
        return torch.randn(*shape, device="cuda", generator=gen) * scale

    if not case["op"].startswith("attention"):
        d, rows = case["d"], case["rows"]
        pairs = [int(p) for p in case["pairs"].split(",")]
        # each axis has its own range of frequencies, from one radian per step down
        freqs = torch.cat([100.0 ** (-torch.arange(n, device="cuda", dtype=torch.float64) / n) for n in pairs]).float()
        axis = torch.tensor([a for a, n in enumerate(pairs) for _ in range(n)], device="cuda")     # of each pair
        state = dict(case=case, pairs=pairs, axis=axis, freqs=freqs, positions=_positions(case, gen))
        if case["op"] == "rope_axes":
            # queries and keys as the QKV product leaves them: rows wider than the heads in use
            packed = normal(rows, (case["heads"] + case["heads"] // 2 + 1) * d).to(dtype)
            return dict(state, x=packed)
        heads = case["q_heads"] + case["k_heads"]
        packed = normal(rows, (heads + case["k_heads"]) * d, scale=1.7).to(dtype)
        gains = 1 + normal(2, d, scale=0.1)
        state.update(x=packed, q_gain=gains[0].contiguous(), k_gain=gains[1].contiguous())
        if case["op"] == "qk_norm_rope_backward":
            state["dy"] = normal(rows, heads * d, scale=0.5).to(dtype)
        return state

    d, heads, kv = case["d"], case["heads"], case["kv_heads"]
    ql, kl = _lengths(case)
    q_off = torch.tensor([0] + ql, device="cuda").cumsum(0).to(torch.int32)
    k_off = torch.tensor([0] + kl, device="cuda").cumsum(0).to(torch.int32) if case["cross"] else q_off
    q_rows, k_rows = sum(ql), sum(kl)
    if case["cross"]:
        q = normal(q_rows, heads * d, scale=1.2).to(dtype)
        packed = normal(k_rows, 2 * kv * d).to(dtype)
        k, v = packed[:, :kv * d], packed[:, kv * d:]
    else:                                                  # one buffer, as the QKV product leaves it
        packed = normal(q_rows, (heads + 2 * kv) * d, scale=1.1).to(dtype)
        q, k, v = packed[:, :heads * d], packed[:, heads * d:(heads + kv) * d], packed[:, (heads + kv) * d:]
    state = dict(case=case, q=q, k=k, v=v, q_off=q_off, k_off=k_off, max_q=max(ql), max_k=max(kl), scale=1 / math.sqrt(d))
    if case["op"] == "attention_backward":
        state["out"], state["lse"] = _attention(state)
        state["dout"] = normal(q_rows, heads * d, scale=0.3).to(dtype)
    return state


# ------------------------------------------------------------------------------------ the plain forms
def _turn(x, state, inverse):
    """x [rows, heads, d] in 32 bits, its pairs turned by the angles of the rows' positions."""
    n = sum(state["pairs"])
    angle = state["positions"].double()[state["axis"]].t() * state["freqs"].double()      # far positions need 64 bits
    c, s = angle.cos().float()[:, None], angle.sin().float()[:, None]
    if inverse:
        s = -s
    y = x.clone()
    a, b = (x[..., 0:2 * n:2], x[..., 1:2 * n:2]) if state["case"]["interleaved"] else (x[..., :n], x[..., n:2 * n])
    first, second = a * c - b * s, a * s + b * c
    if state["case"]["interleaved"]:
        y[..., 0:2 * n:2], y[..., 1:2 * n:2] = first, second
    else:
        y[..., :n], y[..., n:2 * n] = first, second
    return y


def _gains(state):
    case = state["case"]
    return torch.cat([state["q_gain"].expand(case["q_heads"], -1), state["k_gain"].expand(case["k_heads"], -1)])


def _norm_rope(state):
    case = state["case"]
    heads, d = case["q_heads"] + case["k_heads"], case["d"]
    x = state["x"][:, :heads * d].float().view(-1, heads, d)
    y = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * _gains(state)
    return _turn(y, state, False).view(-1, heads * d).to(state["x"].dtype)


def _norm_rope_backward(state):
    case = state["case"]
    heads, d, hq = case["q_heads"] + case["k_heads"], case["d"], case["q_heads"]
    x = state["x"][:, :heads * d].float().view(-1, heads, d)
    dy = _turn(state["dy"].float().view(-1, heads, d), state, True)
    rstd = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    xhat = x * rstd
    dgain = (dy * xhat).double().sum(0)                                          # a long sum
    dy = dy * _gains(state)
    dx = rstd * (dy - xhat * (dy * xhat).mean(-1, keepdim=True))
    return dx.view(-1, heads * d).to(state["x"].dtype), dgain[:hq].sum(0).float(), dgain[hq:].sum(0).float()


def _padded(state):
    """Row numbers [sequences, longest] of queries and keys, and which of them are there."""
    q_off, k_off = state["q_off"].long(), state["k_off"].long()
    qr = q_off[:-1, None] + torch.arange(state["max_q"], device="cuda")
    kr = k_off[:-1, None] + torch.arange(state["max_k"], device="cuda")
    return qr, qr < q_off[1:, None], kr, kr < k_off[1:, None]


def _spread(x, rows, heads):
    """x [total, heads * d] as [sequences, heads, longest, d] in 32 bits."""
    return x[rows.clamp(max=max(0, x.shape[0] - 1))].float().unflatten(-1, (heads, -1)).transpose(1, 2)


def _gather(x, rows, valid, total):
    """[sequences, heads, longest, ...] back to [total, heads, ...]."""
    y = x.new_empty((total + 1, x.shape[1]) + x.shape[3:])
    y[torch.where(valid, rows, total).flatten()] = x.transpose(1, 2).flatten(0, 1)
    return y[:total]


def _operands(state):
    case = state["case"]
    group = case["heads"] // case["kv_heads"]
    qr, q_there, kr, k_there = _padded(state)
    q = _spread(state["q"], qr, case["heads"])
    k = _spread(state["k"], kr, case["kv_heads"]).repeat_interleave(group, 1)
    v = (_spread(state["v"], kr, case["kv_heads"]) * k_there[:, None, :, None]).repeat_interleave(group, 1)
    there = q_there[:, None, :, None] & k_there[:, None, None, :]
    return q, k, v, there, qr, q_there, kr, k_there


def _attention(state):
    q, k, v, there, qr, q_there, _, _ = _operands(state)
    s = (q @ k.transpose(-1, -2)).mul_(state["scale"]).masked_fill_(~there, -math.inf)
    top = s.amax(-1, keepdim=True).clamp_(min=torch.finfo(torch.float32).min)
    p = s.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = (p @ v) / total.clamp(min=torch.finfo(torch.float32).tiny)              # no keys: zero
    lse = (top + total.log())[..., 0]
    rows = state["q"].shape[0]
    return (_gather(out, qr, q_there, rows).flatten(1).to(state["q"].dtype),
            _gather(lse, qr, q_there, rows).t().contiguous())


def _attention_backward(state):
    case = state["case"]
    q, k, v, there, qr, q_there, kr, k_there = _operands(state)
    rows, group = state["q"].shape[0], case["heads"] // case["kv_heads"]
    dout = _spread(state["dout"], qr, case["heads"]) * q_there[:, None, :, None]
    delta = (dout * _spread(state["out"], qr, case["heads"])).sum(-1, keepdim=True)
    lse = state["lse"].t()[qr.clamp(max=max(0, rows - 1))].transpose(1, 2)[..., None]
    p = (q @ k.transpose(-1, -2)).mul_(state["scale"]).sub_(lse).exp_().masked_fill_(~there, 0.0)
    dv = p.transpose(-1, -2) @ dout
    ds = (dout @ v.transpose(-1, -2)).sub_(delta).mul_(p).mul_(state["scale"])
    dq = ds @ k
    dk = ds.transpose(-1, -2) @ q
    k_rows, dtype = state["k"].shape[0], state["q"].dtype
    dk, dv = (t.unflatten(1, (-1, group)).sum(2) for t in (dk, dv))
    return (_gather(dq, qr, q_there, rows).flatten(1).to(dtype), _gather(dk, kr, k_there, k_rows).flatten(1).to(dtype),
            _gather(dv, kr, k_there, k_rows).flatten(1).to(dtype))


# ------------------------------------------------------------------------------------ the library's calls
@functools.lru_cache(None)
def _handle():
    """A handle of a model of the smallest kind: the single operations need no weights of it."""
    import numpy as np
    import paper_2110_14895_b200 as vit

    class shape:
        image_size, patch_size, channels, hidden, layers, heads, mlp_dim, num_classes, ln_eps = 32, 16, 3, 64, 1, 1, 64, 8, 1e-6

    cfg = vit.make_config(shape, vit.VIT_BF16, 1)
    return vit, vit.vit_create(cfg, np.zeros(vit.vit_param_count(cfg), dtype=np.float32))


def _run_own(state):
    vit, h = _handle()
    case = state["case"]
    stream = torch.cuda.current_stream().cuda_stream
    dt = vit.VIT_BF16 if case["dtype"] == "bf16" else vit.VIT_FP32
    d = case["d"]
    if not case["op"].startswith("attention"):
        x, rows = state["x"], case["rows"]
        rope = vit.make_rope(state["pairs"], state["freqs"].data_ptr(), state["positions"].data_ptr(), case["interleaved"])
        if case["op"] == "rope_axes":
            width = case["heads"] * d
            y = torch.empty((rows, width), dtype=x.dtype, device=x.device)
            vit.vit_op_rope_axes(h, dt, rows, case["heads"], d, rope, case["inverse"], x.data_ptr(), x.stride(0), y.data_ptr(), width,
                                 stream)
            return y
        hq, hk = case["q_heads"], case["k_heads"]
        width = (hq + hk) * d
        y = torch.empty((rows, width), dtype=x.dtype, device=x.device)
        if case["op"] == "qk_norm_rope":
            vit.vit_op_qk_norm_rope(h, dt, rows, hq, hk, d, state["q_gain"].data_ptr(), state["k_gain"].data_ptr(), EPS, rope,
                                    x.data_ptr(), x.stride(0), y.data_ptr(), width, stream)
            return y
        grads = torch.empty((2, d), dtype=torch.float32, device=x.device)
        n = vit.vit_qk_norm_rope_backward_bytes(rows, hq, hk, d)
        ws = torch.empty(n, dtype=torch.uint8, device=x.device)
        vit.vit_op_qk_norm_rope_backward(h, dt, rows, hq, hk, d, state["q_gain"].data_ptr(), state["k_gain"].data_ptr(), EPS, rope,
                                         x.data_ptr(), x.stride(0), state["dy"].data_ptr(), width, y.data_ptr(), width,
                                         grads[0].data_ptr(), grads[1].data_ptr(), ws.data_ptr(), n, stream)
        return y, grads[0], grads[1]
    q, k, v = state["q"], state["k"], state["v"]
    heads, kv = case["heads"], case["kv_heads"]
    problem = vit.make_attention_problem(case["sequences"], heads, kv, d, q.shape[0], state["max_q"], state["q_off"].data_ptr(),
                                         k.shape[0], state["max_k"], state["k_off"].data_ptr(), state["scale"])
    backward = case["op"] == "attention_backward"
    n = vit.vit_attention_packed_bytes(dt, problem, backward)
    ws = torch.empty(n, dtype=torch.uint8, device=q.device)
    if not backward:
        out = torch.empty((q.shape[0], heads * d), dtype=q.dtype, device=q.device)
        lse = torch.empty((heads, q.shape[0]), dtype=torch.float32, device=q.device)
        vit.vit_op_attention_packed(h, dt, problem, q.data_ptr(), q.stride(0), k.data_ptr(), k.stride(0), v.data_ptr(), v.stride(0),
                                    out.data_ptr(), heads * d, lse.data_ptr(), ws.data_ptr(), n, stream)
        return out, lse
    dq = torch.empty((q.shape[0], heads * d), dtype=q.dtype, device=q.device)
    dk, dv = (torch.empty((k.shape[0], kv * d), dtype=q.dtype, device=q.device) for _ in range(2))
    vit.vit_op_attention_packed_backward(h, dt, problem, q.data_ptr(), q.stride(0), k.data_ptr(), k.stride(0), v.data_ptr(),
                                         v.stride(0), state["out"].data_ptr(), heads * d, state["lse"].data_ptr(),
                                         state["dout"].data_ptr(), heads * d, dq.data_ptr(), heads * d, dk.data_ptr(), kv * d,
                                         dv.data_ptr(), kv * d, ws.data_ptr(), n, stream)
    return dq, dk, dv


def run(state):
    if own:
        return _run_own(state)
    op = state["case"]["op"]
    if op == "rope_axes":
        case = state["case"]
        x = state["x"][:, :case["heads"] * case["d"]].float().view(-1, case["heads"], case["d"])
        return _turn(x, state, case["inverse"]).flatten(1).to(state["x"].dtype)
    if op == "qk_norm_rope":
        return _norm_rope(state)
    if op == "qk_norm_rope_backward":
        return _norm_rope_backward(state)
    return _attention(state) if op == "attention" else _attention_backward(state)


# ------------------------------------------------------------------------------------ 64 bits, from the definition
def _turned_exactly(x, case, freqs, positions, inverse=False):
    """The rotation as a product of complex numbers: channel pairs times exp(i position frequency)."""
    pairs = [int(p) for p in case["pairs"].split(",")]
    n, parts = sum(pairs), []
    first = 0
    for axis, count in enumerate(pairs):
        angle = positions[axis].double()[:, None] * freqs[first:first + count].double()[None]
        parts.append(torch.polar(torch.ones_like(angle), -angle if inverse else angle))
        first += count
    unit = torch.cat(parts, 1)[:, None]
    head = x[..., :2 * n]
    if case["interleaved"]:
        z = torch.view_as_complex(head.unflatten(-1, (n, 2)).contiguous())
        turned = torch.view_as_real(z * unit).flatten(-2)
    else:
        z = torch.complex(head[..., :n].contiguous(), head[..., n:].contiguous()) * unit
        turned = torch.cat([z.real, z.imag], -1)
    return torch.cat([turned, x[..., 2 * n:]], -1)


def exact(case, seed):
    state = prepare(case, seed)
    d = case["d"]
    if case["op"] == "rope_axes":
        x = state["x"][:, :case["heads"] * d].double().unflatten(1, (-1, d))
        return _turned_exactly(x, case, state["freqs"], state["positions"], case["inverse"]).flatten(1)
    if case["op"].startswith("qk_norm"):
        heads = case["q_heads"] + case["k_heads"]
        x = state["x"][:, :heads * d].double().unflatten(1, (-1, d)).requires_grad_()
        gains = [state["q_gain"].double().requires_grad_(), state["k_gain"].double().requires_grad_()]
        y = []
        for part, gain in zip(x.split([case["q_heads"], case["k_heads"]], 1), gains):
            size = ((part * part).sum(-1, keepdim=True) / d + EPS).sqrt()
            y.append(_turned_exactly(part / size * gain, case, state["freqs"], state["positions"]))
        y = torch.cat(y, 1).flatten(1)
        if case["op"] == "qk_norm_rope":
            return y.detach()
        dx, dq, dk = torch.autograd.grad(y, [x] + gains, state["dy"].double())
        return dx.flatten(1), dq, dk
    ql, kl = _lengths(case)
    heads, group = case["heads"], case["heads"] // case["kv_heads"]
    q, k, v = (state[name].double().unflatten(1, (-1, d)) for name in "qkv")
    outs = [torch.zeros_like(q)] + ([q.new_full((heads, q.shape[0]), -math.inf)] if case["op"] == "attention" else
                                    [torch.zeros_like(k), torch.zeros_like(v)])
    q0 = k0 = 0
    for a, b in zip(ql, kl):
        for h in range(heads) if a and b else ():
            qs, ks = slice(q0, q0 + a), slice(k0, k0 + b)
            score = state["scale"] * torch.mm(q[qs, h], k[ks, h // group].t())
            if case["op"] == "attention":
                outs[1][h, qs] = torch.logsumexp(score, 1)
                outs[0][qs, h] = torch.softmax(score, 1).mm(v[ks, h // group])
                continue
            do = state["dout"][qs, h * d:(h + 1) * d].double()
            weight = torch.exp(score - state["lse"][h, qs, None].double())
            inner = torch.einsum("qc,qc->q", do, state["out"][qs, h * d:(h + 1) * d].double())
            slope = weight * (do.mm(v[ks, h // group].t()) - inner[:, None])
            outs[0][qs, h] = state["scale"] * slope.mm(k[ks, h // group])
            outs[1][ks, h // group] += state["scale"] * slope.t().mm(q[qs, h])
            outs[2][ks, h // group] += weight.t().mm(do)
        q0, k0 = q0 + a, k0 + b
    if case["op"] == "attention":
        return outs[0].flatten(1), outs[1]
    return tuple(t.flatten(1) for t in outs)
