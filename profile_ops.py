"""Runs one kernel of the library a few times on random device data, for ncu captures and
quick timing:  python profile_ops.py --op linear --M 32896 --N 5120 --K 1280 --epilogue 1
Prints the mean CUDA-event time per launch."""
import argparse

import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import paper_2110_14895_b200 as vit  # noqa: E402


class _Shape:
    image_size, patch_size, channels, hidden, layers, heads, mlp_dim, num_classes, ln_eps = 32, 16, 3, 64, 1, 1, 64, 8, 1e-6


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--op", required=True, choices=["linear", "linear_ln", "attention", "layernorm", "rowstats", "rope_axes", "qk_norm_rope",
                                                   "qk_norm_rope_backward", "attention_packed", "attention_packed_backward", "layernorm_forward",
                                                   "layernorm_backward", "linear_grouped", "linear_grouped_backward_input",
                                                   "linear_grouped_backward_weights", "grad_clip"])
    ap.add_argument("--M", type=int, default=32896)
    ap.add_argument("--N", type=int, default=1280)
    ap.add_argument("--K", type=int, default=1280)
    ap.add_argument("--epilogue", type=int, default=0)
    ap.add_argument("--images", type=int, default=128)
    ap.add_argument("--T", type=int, default=257)
    ap.add_argument("--heads", type=int, default=16)
    ap.add_argument("--d", type=int, default=80)
    ap.add_argument("--groups", type=int, default=1)
    ap.add_argument("--dtype", choices=["bf16", "fp32"], default="bf16", help="of the operations that training needs")
    ap.add_argument("--reps", type=int, default=5)
    a = ap.parse_args()
    cfg = vit.make_config(_Shape, vit.VIT_BF16, 1)
    blob = np.zeros(vit.vit_param_count(cfg), dtype=np.float32)
    h = vit.vit_create(cfg, blob)
    bf = torch.bfloat16
    if a.op == "linear":
        x = torch.randn(a.M, a.K, device="cuda").to(bf)
        w = (torch.randn(a.N, a.K, device="cuda") / a.K ** 0.5).to(bf)
        b = torch.randn(a.N, device="cuda")
        out = torch.randn(a.M, a.N, device="cuda").to(bf)
        res = out.data_ptr() if a.epilogue == 2 else 0
        run = lambda: vit.vit_op_linear(h, vit.VIT_BF16, a.M, a.N, a.K, x.data_ptr(), w.data_ptr(), b.data_ptr(),
                                        a.epilogue, res, out.data_ptr())
        work = 2.0 * a.M * a.N * a.K
        unit = "TFLOP/s"
    elif a.op == "linear_ln":
        # the QKV / fc1 product with the LayerNorm folded in (epilogue 0 = plain, 1 = GELU)
        x = torch.randn(a.M, a.K, device="cuda").to(bf)
        w = (torch.randn(a.N, a.K, device="cuda") / a.K ** 0.5).to(bf)
        c1 = w.float().sum(-1).contiguous()
        c0 = torch.randn(a.N, device="cuda")
        stats = torch.empty(a.M, 2, device="cuda")
        out = torch.empty(a.M, a.N, device="cuda", dtype=bf)
        vit.vit_op_rowstats(h, a.M, a.K, x.data_ptr(), 1e-6, stats.data_ptr())
        run = lambda: vit.vit_op_linear_ln(h, a.M, a.N, a.K, x.data_ptr(), stats.data_ptr(), w.data_ptr(), c1.data_ptr(),
                                           c0.data_ptr(), a.epilogue, out.data_ptr())
        work = 2.0 * a.M * a.N * a.K
        unit = "TFLOP/s"
    elif a.op == "rowstats":
        x = torch.randn(a.M, a.N, device="cuda").to(bf)
        stats = torch.empty(a.M, 2, device="cuda")
        run = lambda: vit.vit_op_rowstats(h, a.M, a.N, x.data_ptr(), 1e-6, stats.data_ptr())
        work = (a.M * a.N * 2 + a.M * 8) / 1e-3     # bytes, scaled so the print below reads GB/s
        unit = "GB/s"
    elif a.op == "attention":
        H = a.heads * a.d
        qkv = torch.randn(a.images * a.T, 3 * H, device="cuda").to(bf)
        out = torch.empty(a.images * a.T, H, device="cuda", dtype=bf)
        run = lambda: vit.vit_op_attention(h, vit.VIT_BF16, a.images, a.T, a.heads, a.d, qkv.data_ptr(), out.data_ptr())
        work = 4.0 * a.images * a.T * a.T * H
        unit = "TFLOP/s"
    elif a.op.startswith("attention_packed"):
        # --images sequences of T tokens each, in the column blocks of one QKV buffer
        rows, H = a.images * a.T, a.heads * a.d
        qkv = torch.randn(rows, 3 * H, device="cuda").to(bf)
        dout = torch.randn(rows, H, device="cuda").to(bf)
        out, dqkv = torch.empty_like(dout), torch.empty_like(qkv)
        lse = torch.empty(a.heads, rows, device="cuda")
        off = (torch.arange(a.images + 1, device="cuda") * a.T).to(torch.int32)
        p = vit.make_attention_problem(a.images, a.heads, a.heads, a.d, rows, a.T, off.data_ptr(), rows, a.T, off.data_ptr(), a.d ** -0.5)
        n = max(vit.vit_attention_packed_bytes(vit.VIT_BF16, p, b) for b in (False, True))
        ws = torch.empty(n, dtype=torch.uint8, device="cuda")
        q, dq = qkv.data_ptr(), dqkv.data_ptr()
        fwd = lambda: vit.vit_op_attention_packed(h, vit.VIT_BF16, p, q, 3 * H, q + 2 * H, 3 * H, q + 4 * H, 3 * H, out.data_ptr(), H,
                                                  lse.data_ptr(), ws.data_ptr(), n)
        bwd = lambda: vit.vit_op_attention_packed_backward(
            h, vit.VIT_BF16, p, q, 3 * H, q + 2 * H, 3 * H, q + 4 * H, 3 * H, out.data_ptr(), H, lse.data_ptr(), dout.data_ptr(), H, dq,
            3 * H, dq + 2 * H, 3 * H, dq + 4 * H, 3 * H, ws.data_ptr(), n)
        fwd()
        backward = a.op.endswith("backward")
        run = bwd if backward else fwd
        work = (10.0 if backward else 4.0) * a.images * a.T * a.T * H
        unit = "TFLOP/s"
    elif a.op in ("rope_axes", "qk_norm_rope", "qk_norm_rope_backward"):
        # --M rows, query and key heads of a QKV buffer, two position axes
        H = 2 * a.heads * a.d
        x = torch.randn(a.M, 3 * a.heads * a.d, device="cuda").to(bf)
        dy, y = torch.randn(a.M, H, device="cuda").to(bf), torch.empty(a.M, H, device="cuda", dtype=bf)
        g, dg = torch.ones(2, a.d, device="cuda"), torch.empty(2, a.d, device="cuda")
        freqs = (100.0 ** (-torch.arange(a.d // 2, device="cuda") / (a.d // 2))).float()
        pos = torch.randint(0, 64, (2, a.M), device="cuda").to(torch.int32)
        rope = vit.make_rope((a.d // 4, a.d // 2 - a.d // 4), freqs.data_ptr(), pos.data_ptr())
        n = vit.vit_qk_norm_rope_backward_bytes(a.M, a.heads, a.heads, a.d)
        ws = torch.empty(n, dtype=torch.uint8, device="cuda")
        common = (h, vit.VIT_BF16, a.M, a.heads, a.heads, a.d, g[0].data_ptr(), g[1].data_ptr(), 1e-6, rope, x.data_ptr(), x.stride(0))
        run = {"rope_axes": lambda: vit.vit_op_rope_axes(h, vit.VIT_BF16, a.M, 2 * a.heads, a.d, rope, 0, x.data_ptr(), x.stride(0),
                                                         y.data_ptr(), H),
               "qk_norm_rope": lambda: vit.vit_op_qk_norm_rope(*common, y.data_ptr(), H),
               "qk_norm_rope_backward": lambda: vit.vit_op_qk_norm_rope_backward(*common, dy.data_ptr(), H, y.data_ptr(), H,
                                                                                 dg[0].data_ptr(), dg[1].data_ptr(), ws.data_ptr(), n)}[a.op]
        work = a.M * H * 2 * (3.0 if a.op.endswith("backward") else 2.0) / 1e-3   # bytes, scaled so the print below reads GB/s
        unit = "GB/s"
    elif a.op in ("layernorm_forward", "layernorm_backward"):
        # --M rows of --N columns; the backward pass with the residual path's gradient
        dt, t = (vit.VIT_BF16, bf) if a.dtype == "bf16" else (vit.VIT_FP32, torch.float32)
        x, dy, dres = (torch.randn(a.M, a.N, device="cuda").to(t) for _ in range(3))
        y, stats = torch.empty_like(x), torch.empty(a.M, 2, device="cuda")
        g, dg = torch.ones(2, a.N, device="cuda"), torch.empty(2, a.N, device="cuda")
        n = vit.vit_layernorm_backward_bytes(a.M, a.N)
        ws = torch.empty(n, dtype=torch.uint8, device="cuda")
        fwd = lambda: vit.vit_op_layernorm_forward(h, dt, a.M, a.N, x.data_ptr(), a.N, g[0].data_ptr(), g[1].data_ptr(), 1e-6, y.data_ptr(),
                                                   a.N, stats.data_ptr())
        fwd()
        run = fwd if a.op == "layernorm_forward" else lambda: vit.vit_op_layernorm_backward(
            h, dt, a.M, a.N, x.data_ptr(), a.N, g[0].data_ptr(), stats.data_ptr(), dy.data_ptr(), a.N, dres.data_ptr(), a.N, y.data_ptr(), a.N,
            dg[0].data_ptr(), dg[1].data_ptr(), ws.data_ptr(), n)
        work = a.M * a.N * x.element_size() * (2.0 if a.op == "layernorm_forward" else 4.0) / 1e-3   # bytes, as above
        unit = "GB/s"
    elif a.op.startswith("linear_grouped"):
        # --M rows in --groups groups of growing lengths, --K in, --N out; --epilogue 1 keeps GELU's argument (or reads it, backwards)
        dt, t = (vit.VIT_BF16, bf) if a.dtype == "bf16" else (vit.VIT_FP32, torch.float32)
        edges = [a.M * g * (g + a.groups) // (2 * a.groups * a.groups) for g in range(a.groups + 1)]
        off = torch.tensor(edges, dtype=torch.int32, device="cuda")
        x, dx, pre_k = (torch.randn(a.M, a.K, device="cuda").to(t) for _ in range(3))
        out, res, pre_n = (torch.randn(a.M, a.N, device="cuda").to(t) for _ in range(3))
        w = (torch.randn(a.groups, a.N, a.K, device="cuda") / a.K ** 0.5).to(t)
        b, db, dw = torch.randn(a.groups, a.N, device="cuda"), torch.empty(a.groups, a.N, device="cuda"), torch.empty_like(w)
        p = vit.make_grouped_problem(a.groups, a.M, a.K, a.N, off.data_ptr())
        n = vit.vit_linear_grouped_backward_weights_bytes(dt, p)
        ws = torch.empty(n, dtype=torch.uint8, device="cuda")
        run = {"linear_grouped": lambda: vit.vit_op_linear_grouped(
                   h, dt, p, x.data_ptr(), a.K, w.data_ptr(), b.data_ptr(), a.epilogue, res.data_ptr(), a.N, out.data_ptr(), a.N,
                   pre_n.data_ptr() if a.epilogue == 1 else 0, a.N),
               "linear_grouped_backward_input": lambda: vit.vit_op_linear_grouped_backward_input(
                   h, dt, p, res.data_ptr(), a.N, w.data_ptr(), pre_k.data_ptr() if a.epilogue == 1 else 0, a.K, dx.data_ptr(), a.K),
               "linear_grouped_backward_weights": lambda: vit.vit_op_linear_grouped_backward_weights(
                   h, dt, p, x.data_ptr(), a.K, res.data_ptr(), a.N, dw.data_ptr(), db.data_ptr(), ws.data_ptr(), n)}[a.op]
        work = 2.0 * a.M * a.N * a.K
        unit = "TFLOP/s"
    elif a.op == "grad_clip":
        # --groups tensors of --M x --N values
        grads = [torch.randn(a.M, a.N, device="cuda").to(bf) for _ in range(a.groups)]
        clipped = [torch.empty_like(t) for t in grads]
        tensors = vit.make_tensors([(t.data_ptr(), c.data_ptr(), t.numel(), vit.VIT_BF16) for t, c in zip(grads, clipped)])
        n, norm = vit.vit_grad_clip_bytes(a.groups), torch.empty(1, device="cuda")
        ws = torch.empty(n, dtype=torch.uint8, device="cuda")
        run = lambda: vit.vit_op_grad_clip(h, tensors, a.groups, 1.0, norm.data_ptr(), ws.data_ptr(), n)
        work = 2.0 * a.groups * a.M * a.N * 2 / 1e-3   # bytes, as above
        unit = "GB/s"
    else:
        x = torch.randn(a.M, a.N, device="cuda").to(bf)
        y = torch.empty_like(x)
        g = torch.ones(a.N, device="cuda")
        b = torch.zeros(a.N, device="cuda")
        run = lambda: vit.vit_op_layernorm(h, vit.VIT_BF16, a.M, a.N, x.data_ptr(), g.data_ptr(), b.data_ptr(), 1e-6, y.data_ptr())
        work = 2.0 * a.M * a.N * 2 / 1e-3   # bytes, scaled so the print below reads GB/s
        unit = "GB/s"
    run()
    torch.cuda.synchronize()
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    e0.record()
    for _ in range(a.reps):
        run()
    e1.record()
    torch.cuda.synchronize()
    vit.vit_check_status(h)
    ms = e0.elapsed_time(e1) / a.reps
    print(f"{a.op}: {ms * 1e3:.1f} us per launch, {work / (ms * 1e-3) / 1e12:.1f} {unit}")
    vit.vit_destroy(h)


if __name__ == "__main__":
    main()
