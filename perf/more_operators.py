"""The operators that training an encoder layer needs beside its attention, measured one call at a time.

A layer's rows (the tokens of a batch of images, or their copies sorted by expert) pass a layer norm, a
linear layer of one or several weight matrices, and on the way back their gradients; at the end of a step
the gradients of all weights are clipped by their common norm.  The cases are the calls of such a step:

  layernorm              layer norm of every row, and the rows' statistics for the way back
  layernorm_backward     its gradients (of the rows, joined with the residual path's, of gain and shift)
  linear                 rows times the weights of their group, bias, and GELU or a residual added
  linear_input_grad      gradient of its rows, times the slope of the GELU before them where there is one
  linear_weight_grad     gradients of its weights and biases, group by group
  grad_clip              norm of all gradients together, and the gradients scaled down to a bound

`run` computes the plain form in torch where `own` is false and calls the library where it is true.
"""
import functools
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
EPS = 1e-6


# ------------------------------------------------------------------------------------ the cases
def listed():
    return [
        # one 224 x 224 image of the tiny model: the smallest call, all latency
        dict(name="norm one image", op="layernorm", dtype="bf16", rows=197, cols=192, wider=0),
        # a layer of ViT-H/14 on 128 images
        dict(name="norm huge14", op="layernorm", dtype="bf16", rows=32896, cols=1280, wider=0),
        # fine-tuning ViT-L/16 on 64 images; the residual path's gradient joins here
        dict(name="norm backward large16", op="layernorm_backward", dtype="bf16", rows=12608, cols=1024, wider=0, residual=True),
        # fine-tuning in fp32 on a few odd-sized images
        dict(name="norm backward fp32", op="layernorm_backward", dtype="fp32", rows=1531, cols=768, wider=24, residual=False),
        # one image of the small model, every token at one of eight experts: a few rows each
        dict(name="experts one image", op="linear", dtype="bf16", rows=197, groups=8, k=384, n=1536, ragged=True, epilogue=1, bias=True,
             pre=False),
        # the first product of ViT-L/16's MLP as sixteen experts, 64 images, every token at two of them, training
        dict(name="experts fc1 large16", op="linear", dtype="bf16", rows=25216, groups=16, k=1024, n=4096, ragged=True, epilogue=1,
             bias=True, pre=True),
        # the way back through the second product and the GELU before it
        dict(name="experts input gradient large16", op="linear_input_grad", dtype="bf16", rows=25216, groups=16, k=4096, n=1024,
             ragged=True, pre=True),
        # a gradient check of four small experts in the fp32 mode
        dict(name="experts input gradient fp32", op="linear_input_grad", dtype="fp32", rows=577, groups=4, k=192, n=768, ragged=True,
             pre=False),
        # the weights of the first product
        dict(name="experts weight gradient large16", op="linear_weight_grad", dtype="bf16", rows=25216, groups=16, k=1024, n=4096,
             ragged=True, bias=True),
        # the output projection of ViT-H/14, an ordinary linear layer: one group, 32 images, few tiles and a long sum
        dict(name="projection weight gradient huge14", op="linear_weight_grad", dtype="bf16", rows=8224, groups=1, k=1280, n=1280,
             ragged=False, bias=True),
        # all gradients of the tiny model in the fp32 mode
        dict(name="clip tiny16", op="grad_clip", dtype="fp32", hidden=192, layers=12, mlp=768, patch=768, tokens=197, classes=1000,
             bound=0.5),
        # all gradients of ViT-H/14: matrices in bf16, vectors in fp32
        dict(name="clip huge14", op="grad_clip", dtype="bf16", hidden=1280, layers=32, mlp=5120, patch=588, tokens=257, classes=1000,
             bound=1.0),
    ]


def _log_uniform(rng, low, high):
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 1))) - 0.5))))


def draw(rng):
    op = rng.choice(["layernorm", "layernorm_backward", "linear", "linear", "linear_input_grad", "linear_input_grad",
                     "linear_weight_grad", "linear_weight_grad", "grad_clip"])
    dtype = "bf16" if rng.random() < 0.75 else "fp32"
    if op.startswith("layernorm"):
        case = dict(op=op, dtype=dtype, rows=_log_uniform(rng, 1, 33000), cols=8 * _log_uniform(rng, 1, 400),
                    wider=rng.choice([0, 0, 8, 64]))
        if op == "layernorm_backward":
            case["residual"] = rng.random() < 0.5
        while work(case)["bytes"] > 2.5e8:
            case["rows"] = case["rows"] * 2 // 3
        return case
    if op == "grad_clip":
        hidden = 8 * _log_uniform(rng, 4, 160)
        case = dict(op=op, dtype=dtype, hidden=hidden, layers=_log_uniform(rng, 1, 32), mlp=hidden * rng.randint(1, 4),
                    patch=_log_uniform(rng, 12, 800), tokens=_log_uniform(rng, 5, 600), classes=_log_uniform(rng, 2, 3000),
                    bound=rng.choice([0.1, 1.0, 1e9]))
        while work(case)["bytes"] > 1.2e9:
            case["layers"] = max(1, case["layers"] // 2)
        return case
    groups = 1 if rng.random() < 0.3 else _log_uniform(rng, 2, 64)
    case = dict(op=op, dtype=dtype, rows=_log_uniform(rng, 1, 33000), groups=groups, k=8 * _log_uniform(rng, 2, 640),
                n=8 * _log_uniform(rng, 2, 640), ragged=groups > 1 and rng.random() < 0.8)
    if op == "linear":
        epilogue = rng.randint(0, 2)
        case.update(epilogue=epilogue, bias=rng.random() < 0.7, pre=epilogue == 1 and rng.random() < 0.5)
    elif op == "linear_input_grad":
        case["pre"] = rng.random() < 0.5
    else:
        case["bias"] = rng.random() < 0.7
    while work(case)["flops"] > (2e11 if dtype == "bf16" else 1.5e10):
        case["rows"] = case["rows"] * 2 // 3
    while work(case)["bytes"] > 8e8:
        case["groups"] = max(1, case["groups"] // 2)
        case["rows"] = case["rows"] * 2 // 3 + 1
    return case


def _group_lengths(case):
    """Rows of every group: the case's own, whatever the seed.  A router's favourites get several times the mean."""
    rows, groups = case["rows"], case["groups"]
    if not case["ragged"]:
        return [rows * (g + 1) // groups - rows * g // groups for g in range(groups)]
    rng = random.Random("%d %d %d %d" % (rows, groups, case["k"], case["n"]))
    weight = [math.exp(0.7 * rng.gauss(0, 1)) for _ in range(groups)]
    if groups >= 4:
        weight[rng.randrange(groups)] = 0.0                # an expert that nobody chose
    total, edge, edges = sum(weight), 0.0, [0]
    for w in weight:
        edge += w
        edges.append(int(rows * edge / total + 0.5))
    edges[-1] = rows
    return [b - a for a, b in zip(edges, edges[1:])]


def _shapes(case):
    """The weight tensors of a vision transformer, and which of them are vectors (32 bits always)."""
    h, f, c = case["hidden"], case["mlp"], case["classes"]
    matrices, vectors = [(h, case["patch"]), (case["tokens"], h), (c, h)], [(h,), (h,), (h,), (h,), (c,)]
    for _ in range(case["layers"]):
        matrices += [(3 * h, h), (h, h), (f, h), (h, f)]
        vectors += [(h,), (h,), (3 * h,), (h,), (h,), (h,), (f,), (h,)]
    return [(s, False) for s in matrices] + [(s, True) for s in vectors]


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"].startswith("layernorm"):
        values = case["rows"] * case["cols"]
        if case["op"] == "layernorm":
            return {"bytes": 2 * values * size + 8 * case["rows"] + 8 * case["cols"], "flops": 8 * values}
        return {"bytes": (4 if case["residual"] else 3) * values * size + 8 * case["rows"] + 12 * case["cols"], "flops": 14 * values}
    if case["op"] == "grad_clip":
        count = sum(math.prod(s) * (4 if vector else size) for s, vector in _shapes(case))
        return {"bytes": 2 * count, "flops": 3 * sum(math.prod(s) for s, _ in _shapes(case))}
    lengths = _group_lengths(case)
    used = sum(1 for n in lengths if n)
    rows, k, n = case["rows"], case["k"], case["n"]
    flops = 2 * rows * k * n
    if case["op"] == "linear":
        out = rows * n * size * (1 + (case["epilogue"] == 2) + case["pre"])
        return {"bytes": rows * k * size + used * k * n * size + out + (4 * used * n if case["bias"] else 0), "flops": flops}
    if case["op"] == "linear_input_grad":
        return {"bytes": rows * n * size + used * k * n * size + rows * k * size * (1 + case["pre"]), "flops": flops}
    groups = case["groups"]
    return {"bytes": rows * (n + k) * size + groups * k * n * size + (4 * groups * n if case["bias"] else 0), "flops": flops}


# ------------------------------------------------------------------------------------ the inputs
def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = DTYPES[case["dtype"]]

    def normal(*shape, scale=1.0):
        return torch.randn(*shape, device="cuda", generator=gen) * scale

    if case["op"].startswith("layernorm"):
        rows, cols = case["rows"], case["cols"]
        # a residual stream: rows have a mean and a size of their own
        x = normal(rows, cols + case["wider"]) * (1 + normal(rows, 1).abs()) + normal(rows, 1, scale=0.5)
        state = dict(case=case, x=x.to(dtype)[:, :cols], gain=1 + normal(cols, scale=0.1), shift=normal(cols, scale=0.1))
        if case["op"] == "layernorm_backward":
            state["dy"] = normal(rows, cols, scale=0.3).to(dtype)
            if case["residual"]:
                state["dres"] = normal(rows, cols, scale=0.3).to(dtype)
            state["stats"] = _row_stats(state["x"])
        return state
    if case["op"] == "grad_clip":
        # as optimizers keep them: all matrices in one buffer and all vectors in another, every tensor at a multiple of 16 bytes
        flat, flat_clipped, grads, clipped = [], [], [], []
        for t, some in ((dtype, [s for s, vector in _shapes(case) if not vector]), (torch.float32, [s for s, vector in _shapes(case) if vector])):
            first = [0]
            for s in some:
                first.append(first[-1] + (math.prod(s) + 7) // 8 * 8)
            flat.append(torch.zeros(first[-1], dtype=t, device="cuda"))
            flat_clipped.append(torch.zeros_like(flat[-1]))
            for s, at in zip(some, first):
                flat[-1][at:at + math.prod(s)] = normal(math.prod(s), scale=1e-3)
                for views, buffer in ((grads, flat[-1]), (clipped, flat_clipped[-1])):
                    views.append(buffer[at:at + math.prod(s)].view(s))
        state = dict(case=case, flat=flat, flat_clipped=flat_clipped, grads=grads, clipped=clipped)
        if own:                                            # a training loop lists its gradients once
            vit, _ = _handle()
            types = {torch.bfloat16: vit.VIT_BF16, torch.float32: vit.VIT_FP32}
            state["tensors"] = vit.make_tensors([(g.data_ptr(), c.data_ptr(), g.numel(), types[g.dtype])
                                                 for g, c in zip(grads, state["clipped"])])
        return state
    rows, groups, k, n = case["rows"], case["groups"], case["k"], case["n"]
    offsets = torch.tensor([0] + _group_lengths(case), device="cuda").cumsum(0).to(torch.int32)
    state = dict(case=case, offsets=offsets)
    if case["op"] != "linear_weight_grad":
        state["w"] = normal(groups, n, k, scale=k ** -0.5).to(dtype)
    if case["op"] != "linear_input_grad":
        state["x"] = normal(rows, k).to(dtype)
    if case["op"] == "linear":
        state["bias"] = normal(groups, n, scale=0.1) if case["bias"] else None
        state["residual"] = normal(rows, n).to(dtype) if case["epilogue"] == 2 else None
    else:
        state["dout"] = normal(rows, n, scale=0.3).to(dtype)
    if case["op"] == "linear_input_grad":
        state["pre"] = normal(rows, k, scale=1.3).to(dtype) if case["pre"] else None
    return state


def _row_stats(x):
    x = x.float()
    mean = x.mean(-1, keepdim=True)
    return torch.cat([mean, torch.rsqrt((x - mean).square().mean(-1, keepdim=True) + EPS)], -1)


# ------------------------------------------------------------------------------------ the plain forms
def _layernorm(state):
    stats = _row_stats(state["x"])
    y = (state["x"].float() - stats[:, :1]) * stats[:, 1:] * state["gain"] + state["shift"]
    return y.to(state["x"].dtype), stats


def _layernorm_backward(state):
    dy, rstd = state["dy"].float(), state["stats"][:, 1:]
    xhat = (state["x"].float() - state["stats"][:, :1]) * rstd
    w = dy * state["gain"]
    dx = rstd * (w - w.mean(-1, keepdim=True) - xhat * (w * xhat).mean(-1, keepdim=True))
    if "dres" in state:
        dx = dx + state["dres"].float()
    # long sums
    return dx.to(state["x"].dtype), (dy * xhat).double().sum(0).float(), dy.double().sum(0).float()


def _blocks(state):
    edges = [0]
    for length in _group_lengths(state["case"]):
        edges.append(edges[-1] + length)
    return list(zip(edges, edges[1:]))


def _gelu(v):
    return 0.5 * v * (1 + torch.erf(v * math.sqrt(0.5)))


def _gelu_slope(v):
    return 0.5 * (1 + torch.erf(v * math.sqrt(0.5))) + v * torch.exp(-0.5 * v * v) / math.sqrt(2 * math.pi)


def _linear(state):
    case, x, w = state["case"], state["x"], state["w"]
    pre = torch.empty(case["rows"], case["n"], device=x.device)
    for g, (a, b) in enumerate(_blocks(state)):
        if b > a:
            pre[a:b] = x[a:b].float() @ w[g].float().t()
            if case["bias"]:
                pre[a:b] += state["bias"][g]
    if case["epilogue"] == 0:
        return pre.to(x.dtype)
    if case["epilogue"] == 2:
        return (pre + state["residual"].float()).to(x.dtype)
    out = _gelu(pre).to(x.dtype)
    return (out, pre.to(x.dtype)) if case["pre"] else out


def _linear_input_grad(state):
    case, dout, w = state["case"], state["dout"], state["w"]
    dx = torch.empty(case["rows"], case["k"], device=dout.device)
    for g, (a, b) in enumerate(_blocks(state)):
        if b > a:
            dx[a:b] = dout[a:b].float() @ w[g].float()
    if case["pre"]:
        dx *= _gelu_slope(state["pre"].float())
    return dx.to(dout.dtype)


def _linear_weight_grad(state):
    case, x, dout = state["case"], state["x"], state["dout"]
    dw = torch.zeros(case["groups"], case["n"], case["k"], device=x.device)
    db = torch.zeros(case["groups"], case["n"], device=x.device)
    for g, (a, b) in enumerate(_blocks(state)):
        if b > a:
            dw[g] = dout[a:b].float().t() @ x[a:b].float()
            if case["bias"]:
                db[g] = dout[a:b].double().sum(0).float()
    dw = dw.to(x.dtype)
    return (dw, db) if case["bias"] else dw


def _grad_clip(state):
    total = sum(g.float().square().sum(dtype=torch.float64) for g in state["grads"])
    norm = total.sqrt()
    factor = torch.where(norm > state["case"]["bound"], state["case"]["bound"] / norm, 1.0).float()
    for g, to in zip(state["grads"], state["clipped"]):
        to.copy_(g.float() * factor)
    return [norm.float().view(1)] + state["flat_clipped"]


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


def _ptr(t):
    return t.data_ptr() if t is not None else 0


def _run_own(state):
    vit, h = _handle()
    case = state["case"]
    stream = torch.cuda.current_stream().cuda_stream
    dt = vit.VIT_BF16 if case["dtype"] == "bf16" else vit.VIT_FP32
    op = case["op"]
    if op == "layernorm":
        x, rows, cols = state["x"], case["rows"], case["cols"]
        y = torch.empty((rows, cols), dtype=x.dtype, device=x.device)
        stats = torch.empty((rows, 2), dtype=torch.float32, device=x.device)
        vit.vit_op_layernorm_forward(h, dt, rows, cols, x.data_ptr(), x.stride(0), state["gain"].data_ptr(), state["shift"].data_ptr(),
                                     EPS, y.data_ptr(), cols, stats.data_ptr(), stream)
        return y, stats
    if op == "layernorm_backward":
        x, rows, cols = state["x"], case["rows"], case["cols"]
        dx = torch.empty((rows, cols), dtype=x.dtype, device=x.device)
        grads = torch.empty((2, cols), dtype=torch.float32, device=x.device)
        size = vit.vit_layernorm_backward_bytes(rows, cols)
        ws = torch.empty(size, dtype=torch.uint8, device=x.device)
        vit.vit_op_layernorm_backward(h, dt, rows, cols, x.data_ptr(), x.stride(0), state["gain"].data_ptr(), state["stats"].data_ptr(),
                                      state["dy"].data_ptr(), cols, _ptr(state.get("dres")), cols, dx.data_ptr(), cols,
                                      grads[0].data_ptr(), grads[1].data_ptr(), ws.data_ptr(), size, stream)
        return dx, grads[0], grads[1]
    if op == "grad_clip":
        device = state["grads"][0].device
        norm = torch.empty(1, dtype=torch.float32, device=device)
        size = vit.vit_grad_clip_bytes(len(state["grads"]))
        ws = torch.empty(size, dtype=torch.uint8, device=device)
        vit.vit_op_grad_clip(h, state["tensors"], len(state["grads"]), case["bound"], norm.data_ptr(), ws.data_ptr(), size, stream)
        return [norm] + state["flat_clipped"]
    rows, k, n = case["rows"], case["k"], case["n"]
    problem = vit.make_grouped_problem(case["groups"], rows, k, n, state["offsets"].data_ptr())
    if op == "linear":
        x = state["x"]
        out = torch.empty((rows, n), dtype=x.dtype, device=x.device)
        pre = torch.empty_like(out) if case["pre"] else None
        vit.vit_op_linear_grouped(h, dt, problem, x.data_ptr(), k, state["w"].data_ptr(), _ptr(state["bias"]), case["epilogue"],
                                  _ptr(state["residual"]), n, out.data_ptr(), n, _ptr(pre), n, stream)
        return (out, pre) if case["pre"] else out
    dout = state["dout"]
    if op == "linear_input_grad":
        dx = torch.empty((rows, k), dtype=dout.dtype, device=dout.device)
        vit.vit_op_linear_grouped_backward_input(h, dt, problem, dout.data_ptr(), n, state["w"].data_ptr(), _ptr(state["pre"]), k,
                                                 dx.data_ptr(), k, stream)
        return dx
    dw = torch.empty((case["groups"], n, k), dtype=dout.dtype, device=dout.device)
    db = torch.empty((case["groups"], n), dtype=torch.float32, device=dout.device) if case["bias"] else None
    size = vit.vit_linear_grouped_backward_weights_bytes(dt, problem)
    ws = torch.empty(size, dtype=torch.uint8, device=dout.device)
    vit.vit_op_linear_grouped_backward_weights(h, dt, problem, state["x"].data_ptr(), k, dout.data_ptr(), n, dw.data_ptr(), _ptr(db),
                                               ws.data_ptr(), size, stream)
    return (dw, db) if case["bias"] else dw


def run(state):
    if own:
        return _run_own(state)
    return {"layernorm": _layernorm, "layernorm_backward": _layernorm_backward, "linear": _linear,
            "linear_input_grad": _linear_input_grad, "linear_weight_grad": _linear_weight_grad,
            "grad_clip": _grad_clip}[state["case"]["op"]](state)


# ------------------------------------------------------------------------------------ 64 bits, from the definition
def _normal_cdf(v):
    return 0.5 * torch.erfc(-v / math.sqrt(2.0))


def exact(case, seed):
    state = prepare(case, seed)
    op = case["op"]
    if op.startswith("layernorm"):
        x, gain, shift = (state[name].double() for name in ("x", "gain", "shift"))
        if op == "layernorm":
            var, mean = torch.var_mean(x, dim=1, unbiased=False)
            rstd = 1.0 / torch.sqrt(var + EPS)
            return torch.addcmul(shift, (x - mean[:, None]) * rstd[:, None], gain), torch.stack([mean, rstd], 1)
        # the statistics are inputs, as the forward pass left them
        mean, rstd = state["stats"].double().unbind(1)
        dy = state["dy"].double()
        z = (x - mean[:, None]) * rstd[:, None]
        slope = torch.einsum("rc,c->rc", dy, gain)
        inner = torch.einsum("rc,rc->r", slope, z) / case["cols"]
        dx = torch.einsum("rc,r->rc", slope - slope.sum(1)[:, None] / case["cols"] - z * inner[:, None], rstd)
        if case["residual"]:
            dx = dx + state["dres"].double()
        return dx, torch.einsum("rc,rc->c", dy, z), torch.ones(case["rows"], dtype=torch.float64, device=dy.device) @ dy
    if op == "grad_clip":
        norm = torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(g.double()) for g in state["grads"]]))
        by = min(1.0, case["bound"] / norm.item())
        return [norm.view(1)] + [g.double() * by for g in state["flat"]]
    lengths = _group_lengths(case)
    if op == "linear":
        parts = []
        for g, x in enumerate(state["x"].split(lengths)):
            part = torch.einsum("rk,nk->rn", x.double(), state["w"][g].double())
            parts.append(part + state["bias"][g].double() if case["bias"] else part)
        pre = torch.cat(parts)
        if case["epilogue"] == 2:
            return pre + state["residual"].double()
        if case["epilogue"] == 0:
            return pre
        out = pre * _normal_cdf(pre)
        return (out, pre) if case["pre"] else out
    if op == "linear_input_grad":
        dx = torch.cat([torch.einsum("rn,nk->rk", d.double(), state["w"][g].double()) for g, d in enumerate(state["dout"].split(lengths))])
        if case["pre"]:
            v = state["pre"].double()
            dx = dx * (_normal_cdf(v) + v * torch.exp(torch.distributions.Normal(0.0, 1.0).log_prob(v)))
        return dx
    pairs = list(zip(state["x"].split(lengths), state["dout"].split(lengths)))
    dw = torch.stack([torch.einsum("rn,rk->nk", d.double(), x.double()) for x, d in pairs])
    return (dw, torch.stack([d.double().sum(0) for _, d in pairs])) if case["bias"] else dw
