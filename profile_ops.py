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
                                                   "qk_norm_rope_backward", "attention_packed", "attention_packed_backward"])
    ap.add_argument("--M", type=int, default=32896)
    ap.add_argument("--N", type=int, default=1280)
    ap.add_argument("--K", type=int, default=1280)
    ap.add_argument("--epilogue", type=int, default=0)
    ap.add_argument("--images", type=int, default=128)
    ap.add_argument("--T", type=int, default=257)
    ap.add_argument("--heads", type=int, default=16)
    ap.add_argument("--d", type=int, default=80)
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
