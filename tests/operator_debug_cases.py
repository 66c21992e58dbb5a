"""Cases of the MoE layer run on both flavours of the library by
test_gpu_debug_operators.py (run as a script: on the checking flavour, results to the
.npz file named on the command line)."""
import os
import sys

import numpy as np

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

# N, K, d, f, M, slots
CASES = [(16, 2, 256, 512, 1, 16), (32, 4, 2880, 288, 5, 32), (64, 6, 512, 96, 17, 20),
         (128, 8, 512, 128, 33, 128), (128, 8, 256, 64, 200, 128), (16, 2, 256, 64, 300, 9),
         (128, 8, 128, 64, 1024, 128)]


def run_cases(P) -> dict:
    import torch
    out = {}
    for N, K, d, f, M, S in CASES:
        for w8, x8 in ((False, False), (True, False), (True, True)):
            g = torch.Generator(device="cuda").manual_seed(N + M)
            new = lambda *s, k=1.0: (torch.randn(s, device="cuda", generator=g) * k).bfloat16()  # noqa: E731,B023
            x, router = new(M, d), new(N, d, k=d ** -0.5)
            w13, w2 = new(S, 2, f, d, k=d ** -0.5), new(S, d, f, k=f ** -0.5)
            s13 = s2 = q = sc = None
            if w8:
                (w13, s13), (w2, s2) = P.quantize_rows(w13), P.quantize_rows(w2)
            if x8:
                q, sc = P.quantize_rows(x)
            slot = (torch.arange(N, device="cuda") - (N - S)).to(torch.int32)
            layer = P.MoeLayer(w13, w2, K=K, router=router, expert_slot=slot, gate_up_scale=s13,
                               down_scale=s2)
            y = layer(x, x8=q, x_scale=sc)
            out[f"{N}-{K}-{d}-{f}-{M}-{S}-{w8:d}{x8:d}"] = y.view(torch.int16).cpu().numpy()
    out["error"] = np.array(P.crc.crc_device_error())
    return out


if __name__ == "__main__":
    import paper_2609_04895_gb300 as P
    from paper_2609_04895_gb300 import build
    P.crc.load(build.DEBUG_LIB)
    np.savez(sys.argv[1], **run_cases(P))
