"""Cases of the operators for prompts, training batches and 4-bit experts, run on both
flavours of the library by test_gpu_debug_more_operators.py (run as a script: on the
checking flavour, results to the .npz file named on the command line)."""
import os
import sys

import numpy as np

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

# N, K, d, f, M
CASES = [(16, 2, 256, 512, 1), (32, 4, 2880, 288, 37), (128, 8, 512, 128, 900),
         (3, 2, 264, 80, 1500), (256, 3, 64, 48, 301)]


def run_cases(P) -> dict:
    import torch
    out = {}

    def keep(name, *ts):
        for i, t in enumerate(ts):
            t = t.contiguous()
            out[f"{name}-{i}"] = t.view(torch.uint8).cpu().numpy()
    for N, K, d, f, M in CASES:
        g = torch.Generator(device="cuda").manual_seed(N + M)
        new = lambda *s, k=1.0: (torch.randn(s, device="cuda", generator=g) * k).bfloat16()  # noqa: E731,B023
        tag = f"{N}-{K}-{d}-{f}-{M}"
        topk = torch.randint(0, min(256, N + 1), (M, K), device="cuda", generator=g).to(torch.uint8)
        x, w13, w2 = new(M, d), new(N, 2, f, d, k=d ** -0.5), new(N, d, f, k=f ** -0.5)
        gates = torch.rand((M, K), device="cuda", generator=g)
        off, rows, place = P.group_choices(topk, N)
        n = int(off[-1])
        keep(tag + "-order", off, rows, place)
        h = P.group_matmul(x, w13, off, rows=rows, K=K)
        h[n:] = 0
        y = P.group_matmul(h, w2, off)
        y[n:] = 0
        keep(tag + "-layer", h, y, P.sum_choices(y, place, gates=gates))
        if d % 16 == 0:                                  # rows of 8 bits, 16 bytes apart
            (x8, xs), (q13, s13) = P.quantize_rows(x), P.quantize_rows(w13)
            keep(tag + "-8bit", P.group_matmul(x8, q13, off, rows=rows, K=K, x_scale=xs,
                                               w_scale=s13)[:n])
        dy = new(M * K, d)
        dx, dw = P.group_matmul_grad(dy, h, w2, off)
        keep(tag + "-grad", dx[:n], dw)
        _, dw = P.group_matmul_grad(new(M * K, 2 * f), x, w13.flatten(1, 2), off, rows=rows, K=K,
                                    want_dx=False,
                                    dw=torch.empty((N, 2 * f, d), dtype=torch.bfloat16,
                                                   device="cuda"))
        keep(tag + "-gathered", dw)
        ds, dg = P.sum_choices_grad(new(M, d), place, gates=gates, y=y)
        keep(tag + "-sum", ds[:n], dg)
        if d % 32 == 0 and M <= 1024:
            q, a = P.quantize_rows4(w13, 32)
            keep(tag + "-4bit", q, a, P.matvec4(x, q, a, topk=topk))
    out["error"] = np.array(P.crc.crc_device_error())
    return out


if __name__ == "__main__":
    import paper_2609_04895_gb300 as P
    from paper_2609_04895_gb300 import build
    P.crc.load(build.DEBUG_LIB)
    np.savez(sys.argv[1], **run_cases(P))
