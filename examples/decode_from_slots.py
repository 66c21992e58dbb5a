"""Decoding one stream from expert slots, with the operators around the router heads.

Two passes over the same tokens of a small synthetic model (per layer: norm with the
residual's addition, router, mixture of experts on 8-bit weights):

1. with every expert on the GPU; the hidden states of each token go through
   route_and_cache, whose trace becomes the plan of expert copies;
2. with C slots a layer: before each layer the planned copies bring the experts it
   takes from the pinned host pool into slots, and the layer reads them there.

An expert's results do not depend on the slot it lies in, so both passes give the
same bits.  Run: python examples/decode_from_slots.py [tokens]
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2609_04895_gb300 as P  # noqa: E402

L, N, K, D, F, C, R = 4, 16, 2, 256, 512, 4, 1
IMAGE = 3 * F * D + 4 * (2 * F + D)          # e4m3 gate, up, down, then their fp32 row scales
EPS = 1e-6


def expert_images(seed: int):
    """The pool: uint8 [L * N][IMAGE] in pinned memory, experts brought to 8 bits."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    gate_up = torch.randn(L * N, 2, F, D, device="cuda", generator=g).mul_(D ** -0.5).bfloat16()
    down = torch.randn(L * N, D, F, device="cuda", generator=g).mul_(F ** -0.5).bfloat16()
    q13, s13 = P.quantize_rows(gate_up)
    q2, s2 = P.quantize_rows(down)
    flat = [t.reshape(L * N, -1).view(torch.uint8) for t in (q13, q2, s13, s2)]
    pool = P.pinned_empty((L * N, IMAGE), torch.uint8)
    pool.copy_(torch.cat(flat, dim=1))
    return pool


def layer_of(slots, router, slot_map):
    """MoeLayer over uint8 [S][IMAGE] expert images; slot_map: where each expert lies."""
    q = slots[:, :3 * F * D].view(torch.float8_e4m3fn)
    scales = slots.view(torch.float32)[:, 3 * F * D // 4:]
    S, st = scales.shape[0], scales.stride(0)
    gate_up, down = P.expert_views(q, F, D)
    s13 = scales.as_strided((S, 2, F), (st, F, 1))
    s2 = scales.as_strided((S, D), (st, 1), scales.storage_offset() + 2 * F)
    return P.MoeLayer(gate_up, down, K=K, router=router, expert_slot=slot_map, gate_up_scale=s13,
                      down_scale=s2)


class Model:
    """The decode step of one token; `before(t, l)` runs before layer l's experts."""

    def __init__(self, layers, norms):
        self.layers, self.norms = layers, norms
        new = lambda *s, **k: torch.empty(s, device="cuda", **k)       # noqa: E731
        self.hidden = new(1, 1, L, D, dtype=torch.bfloat16)
        self.h8, self.scale = new(1, D, dtype=torch.float8_e4m3fn), new(1)
        self.topk = new(L, 1, K, dtype=torch.uint8)
        self.ws = new(layers[0].workspace_bytes(1), dtype=torch.uint8)

    def step(self, x, t, before=None):
        """x [1][D]: the token's embedding.  Returns the residual stream behind the
        last layer; self.hidden keeps what each router read."""
        residual = None
        for l in range(L):
            h, total = self.hidden[:, 0, l], torch.empty_like(x)
            P.rms_norm(x, self.norms[l], EPS, residual=residual, residual_out=total, out=h,
                       out8=self.h8, scale8=self.scale)
            if before:
                before(t, l)
            x = self.layers[l](h, x8=self.h8, x_scale=self.scale, topk=self.topk[l],
                               workspace=self.ws)
            residual = total
        return residual + x


def run(tokens: int = 64, seed: int = 0) -> dict:
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    w_cat = P.synth_weights(L, N, D, seed=seed)
    norms = [(1 + 0.1 * torch.randn(D, device="cuda", generator=g)).bfloat16() for _ in range(L)]
    pool = expert_images(seed)
    # a stream whose tokens resemble the ones before them, as decoded text does
    x = torch.randn(tokens, 1, D, device="cuda", generator=g)
    for t in range(1, tokens):
        x[t] = 0.9 * x[t - 1] + 0.19 ** 0.5 * x[t]
    x = x.bfloat16()

    # 1: every expert resident; cache decisions per token from what the routers read
    whole = pool.cuda().view(L, N, IMAGE)
    model = Model([layer_of(whole[l], w_cat[l, :N], None) for l in range(L)], norms)
    p = P.problem(L, N, K, D, C, R, 1, IMAGE)
    state = P.State(p)
    out, topk, mid, after = [], [], [], []
    for t in range(tokens):
        out.append(model.step(x[t], t))
        topk.append(model.topk.clone())
        trace = P.Trace.alloc(p, 1, caches=True)
        P.route_and_cache(p, model.hidden, w_cat, state, trace)
        assert torch.equal(trace.topk[0, 0], topk[-1][:, 0])      # the same Top-K in the same order
        mid.append(trace.cache_mid[0])
        after.append(trace.cache_after[0])
    plan, _ = P.transfer_plan(p, torch.cat(mid).cpu().numpy(), torch.cat(after).cpu().numpy())

    # 2: C slots a layer, filled by the plan
    slots = torch.zeros((L, C, IMAGE), dtype=torch.uint8, device="cuda")
    maps = torch.full((L, N), -1, dtype=torch.int32, device="cuda")
    model = Model([layer_of(slots[l], w_cat[l, :N], maps[l]) for l in range(L)], norms)

    def fetch(t, l):
        copies = plan[(plan["t"] == t) & (plan["l"] == l)]
        P.transfer_replay(p, copies, pool, slots)
        for c in copies:
            if c["evicted"] >= 0:
                maps[l, int(c["evicted"])] = -1
        for c in copies:
            maps[l, int(c["expert"])] = int(c["slot"])

    same = all(torch.equal(model.step(x[t], t, fetch), out[t]) for t in range(tokens))
    stats = state.read()
    return {"same": same, "copies": len(plan), "planned": stats["misses"] + stats["proactive"],
            "hit": P.metrics(stats, p)["hit"], "bytes": len(plan) * IMAGE,
            "resident": L * C * IMAGE, "whole": L * N * IMAGE,
            "finite": all(bool(torch.isfinite(o.float()).all()) for o in out),
            "error": P.crc.crc_device_error()}


if __name__ == "__main__":
    n = int(sys.argv[1]) if len(sys.argv) > 1 else 64
    r = run(n)
    assert r["same"] and r["finite"] and r["error"] == 0 and r["copies"] == r["planned"], r
    print(f"{n} tokens from {r['resident'] / 1e6:.1f} MB of slots (all experts: {r['whole'] / 1e6:.1f} "
          f"MB): hit rate {r['hit']:.3f}, {r['copies']} copies, {r['bytes'] / n / 1e6:.2f} MB a token; "
          "the outputs equal those with every expert resident")
