"""The operators of a decode step around the expert cache, as a program calls them.

A layer's root-mean-square norm with the residual's addition makes the hidden
state that the router heads read (and its 8-bit form for the experts), the
mixture-of-experts layer reads the experts from the slots the cache keeps, and
the rows of an expert are brought to 8 bits once, when it is loaded.  A trainer
of the router heads takes the norm's gradient.

Sizes are those of the repository's workloads and generic ragged ones: hidden
sizes, experts, Top-K, and the expert widths that the workloads' expert bytes
stand for (3 * d * f * 2).  Hidden states have unit variance, router rows and
expert rows N(0, 1 / row length).
"""
import math

import torch

own = False

EPS = 1e-6
E4M3_MAX = 448.0
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}

# experts, Top-K, hidden size, expert width, cache slots of the repository's workloads
SHAPES = {
    "tiny": dict(N=16, K=2, d=256, f=512, C=4),
    "gptoss": dict(N=32, K=4, d=2880, f=2880, C=8),
    "n64": dict(N=64, K=6, d=2048, f=1024, C=16),
    "qwen3": dict(N=128, K=8, d=2048, f=768, C=32),
    "large": dict(N=128, K=8, d=4096, f=1536, C=32),
}


def _moe(name, shape, M, weights, **over):
    c = dict(name=name, kind="moe", shape=shape, **SHAPES[shape], M=M, weights=weights, x8=False,
             cached=False, renorm=True)
    c.update(over)
    return c


def _norm(name, M, d, stream, **over):
    c = dict(name=name, kind="norm", M=M, d=d, stream=stream, residual=True, bits8=True)
    c.update(over)
    return c


def listed():
    return [
        # one token of the smallest configuration: launches and latency only
        _moe("moe-tiny-1", "tiny", 1, "bf16"),
        # one decoded token of one stream, its 8 experts among the 32 resident in cache slots
        _moe("moe-qwen3-1", "qwen3", 1, "bf16", cached=True),
        # the same from 8-bit experts with the 8-bit hidden state of the norm
        _moe("moe-qwen3-1-8bit", "qwen3", 1, "e4m3", x8=True, cached=True),
        # a few streams (or draft tokens) of the 32-expert backbone, an odd number of them
        _moe("moe-gptoss-5", "gptoss", 5, "bf16"),
        # a full serving batch, one token each: nearly every expert is read
        _moe("moe-qwen3-64", "qwen3", 64, "bf16"),
        # a ragged batch on 8-bit experts with the hidden state in 16 bits, wide rows
        _moe("moe-gptoss-37-8bit", "gptoss", 37, "e4m3"),
        # the largest configuration, several tokens of many streams: every expert, many rows each
        _moe("moe-large-200-8bit", "large", 200, "e4m3", x8=True),
        # one decoded token before the router: launches and latency only
        _norm("norm-1", 1, 2048, "bf16"),
        # a chunk of prompts with the residual stream in 32 bits, a row count that fills no tile
        _norm("norm-4097", 4097, 2880, "f32"),
        # a trainer's step over 8 sequences of 1000 tokens
        dict(name="norm-grad-8000", kind="norm_grad", M=8000, d=2048, stream="bf16", dres=True),
        # one matrix of one expert, brought to 8 bits after its copy into a slot
        dict(name="quantize-768", kind="quantize", M=768, d=2048),
        # a layer's gate and up matrices, all 32 experts, when a model is loaded
        dict(name="quantize-184320", kind="quantize", M=184320, d=2880),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["moe", "moe", "moe", "moe", "norm", "norm_grad", "quantize"])
    if kind == "moe":
        shape = rng.choice(["tiny", "gptoss", "n64", "qwen3", "qwen3", "large"])
        weights = "e4m3" if shape == "large" else rng.choice(["bf16", "e4m3"])
        M = _log_int(rng, 1, 200)
        K = rng.randint(1, SHAPES[shape]["K"])
        c = _moe("", shape, M, weights, K=K, x8=weights == "e4m3" and rng.random() < 0.5,
                 cached=M * K <= SHAPES[shape]["C"], renorm=rng.random() < 0.75)
        del c["name"]
        return c
    d = 8 * _log_int(rng, 25, 768)              # 200 to 6144, any multiple of 8
    if d == 3072:
        d += 8
    if kind == "norm":
        c = _norm("", _log_int(rng, 1, 8192), d, rng.choice(["bf16", "f32"]),
                  residual=rng.random() < 0.75, bits8=rng.random() < 0.75)
        del c["name"]
        return c
    if kind == "norm_grad":
        return dict(kind=kind, M=_log_int(rng, 1, 8192), d=d, stream=rng.choice(["bf16", "f32"]),
                    dres=rng.random() < 0.75)
    return dict(kind=kind, M=_log_int(rng, 1, 65536), d=d)


# --------------------------------------------------------------------------- #
# inputs
# --------------------------------------------------------------------------- #
def _randn(g, shape, dtype, scale=1.0):
    x = torch.randn(shape, device="cuda", generator=g, dtype=dtype)
    return x.mul_(scale) if scale != 1.0 else x


def _bits8(w):
    """e4m3 rows with one scale a row, amax / 448."""
    a = w.abs().amax(-1).float() / E4M3_MAX
    a = torch.where(a > 0, a, torch.ones_like(a))
    return (w / a.unsqueeze(-1)).to(torch.float8_e4m3fn), a


def _inputs(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"c": c}
    M, d = c["M"], c["d"]
    if c["kind"] == "moe":
        N, K, f = c["N"], c["K"], c["f"]
        slots = c["C"] if c["cached"] else N
        s["x"] = _randn(g, (M, d), torch.bfloat16)
        s["router"] = _randn(g, (N, d), torch.bfloat16, d ** -0.5)
        s["w13"] = _randn(g, (slots, 2, f, d), torch.bfloat16, d ** -0.5)
        s["w2"] = _randn(g, (slots, d, f), torch.bfloat16, f ** -0.5)
        if c["weights"] == "e4m3":
            s["w13"], s["s13"] = _bits8(s["w13"])
            s["w2"], s["s2"] = _bits8(s["w2"])
        if c["x8"]:
            s["x8"], s["xs"] = _bits8(s["x"])
        # where each expert lies: everywhere in a full layer, or (cached) the
        # experts of this step's tokens and some others in the slots there are
        order = torch.randperm(N, device="cuda", generator=g)
        if c["cached"]:
            z = s["x"].double() @ s["router"].double().t()
            wanted = torch.zeros(N, dtype=torch.bool, device="cuda")
            wanted[z.topk(K, dim=-1).indices.flatten()] = True
            order = order[torch.argsort(wanted[order].logical_not(), stable=True)]
        s["slot"] = torch.full((N,), -1, dtype=torch.int32, device="cuda")
        at = torch.randperm(slots, device="cuda", generator=g).to(torch.int32)
        s["slot"][order[:slots]] = at
    elif c["kind"] == "norm":
        s["x"] = _randn(g, (M, d), DT[c["stream"]])
        s["w"] = 1.0 + 0.1 * _randn(g, (d,), torch.float32)
        s["w"] = s["w"].to(torch.bfloat16)
        # a residual stream is larger than what a block adds to it
        s["res"] = _randn(g, (M, d), DT[c["stream"]], 3.0) if c["residual"] else None
    elif c["kind"] == "norm_grad":
        s["s"] = _randn(g, (M, d), DT[c["stream"]], 3.0)
        s["dy"] = _randn(g, (M, d), torch.bfloat16, 1e-2)
        s["dres"] = _randn(g, (M, d), DT[c["stream"]], 1e-2) if c["dres"] else None
        s["w"] = (1.0 + 0.1 * _randn(g, (d,), torch.float32)).to(torch.bfloat16)
        s["rstd"] = torch.rsqrt(s["s"].double().square().mean(-1) + EPS).float()
    else:
        s["x"] = _randn(g, (M, d), torch.bfloat16, d ** -0.5)
    return s


def prepare(case, seed):
    return _inputs(case, seed)


# --------------------------------------------------------------------------- #
# plain forms: 32 bits, rounded once
# --------------------------------------------------------------------------- #
def _plain_bits8(y):
    a = y.abs().amax(-1) / E4M3_MAX
    a = torch.where(a > 0, a, torch.ones_like(a))
    return (y / a.unsqueeze(-1)).to(torch.float8_e4m3fn), a


def _glu(gate, up):
    return gate / (1.0 + torch.exp(-gate)) * up


def _plain_moe(s):
    c = s["c"]
    N, K = c["N"], c["K"]
    M = s["x"].shape[0]
    z = s["x"].float() @ s["router"].float().t()
    e = torch.exp(z - z.amax(-1, keepdim=True))
    p = e / e.sum(-1, keepdim=True)
    ids = torch.sort(z, dim=-1, descending=True, stable=True).indices[:, :K]
    g = p.gather(-1, ids)
    if c["renorm"]:
        g = g / g.sum(-1, keepdim=True)
    x = s["x8"].float() * s["xs"][:, None] if c["x8"] else s["x"].float()
    slot = s["slot"].long()

    def mats(w, sc, at):
        w = s[w][at].float()
        return w * s[sc][at].unsqueeze(-1) if sc in s else w

    if M * K < N:           # the experts of each choice, gathered
        at = slot[ids]
        w13 = mats("w13", "s13", at)                                    # [M][K][2][f][d]
        h = _glu((w13[:, :, 0] @ x[:, None, :, None])[..., 0],
                 (w13[:, :, 1] @ x[:, None, :, None])[..., 0])          # [M][K][f]
        y = (mats("w2", "s2", at) @ h[..., None])[..., 0]               # [M][K][d]
        out = (g[..., None] * y).sum(1)
    else:                   # every expert for every token
        w13 = mats("w13", "s13", slot)
        h = _glu(x @ w13[:, 0].mT, x @ w13[:, 1].mT)                    # [N][M][f]
        del w13
        full = torch.zeros((M, N), device=x.device).scatter_(1, ids, g)
        h = h * full.t()[..., None]
        out = (h @ mats("w2", "s2", slot).mT).sum(0)
    return {"out": out.to(torch.bfloat16), "topk": ids.to(torch.uint8), "gates": g}


def _plain_norm(s):
    c = s["c"]
    t = s["x"].float()
    out = {}
    if s["res"] is not None:
        t = t + s["res"].float()
        out["residual"] = t.to(DT[c["stream"]])
    rstd = torch.rsqrt(t.square().mean(-1) + EPS)
    y = t * rstd[:, None] * s["w"].float()
    out["h"] = y.to(torch.bfloat16)
    out["rstd"] = rstd
    if c["bits8"]:
        out["q"], out["scale"] = _plain_bits8(y)
    return out


def _plain_norm_grad(s):
    c = s["c"]
    dy, r = s["dy"].float(), s["rstd"][:, None]
    xhat = s["s"].float() * r
    v = dy * s["w"].float()
    dx = r * (v - xhat * (v * xhat).mean(-1, keepdim=True))
    if s["dres"] is not None:
        dx = dx + s["dres"].float()
    return {"dx": dx.to(DT[c["stream"]]), "dw": (dy * xhat).sum(0)}


def _plain(s):
    kind = s["c"]["kind"]
    if kind == "moe":
        return _plain_moe(s)
    if kind == "norm":
        return _plain_norm(s)
    if kind == "norm_grad":
        return _plain_norm_grad(s)
    q, a = _plain_bits8(s["x"].float())
    return {"q": q, "scale": a}


# --------------------------------------------------------------------------- #
# the framework's operators, with the buffers that a program keeps
# --------------------------------------------------------------------------- #
def _kept(s):
    """The layer handle, outputs and workspace of a program's own, made once."""
    import paper_2609_04895_gb300 as P
    c, k = s["c"], {"P": P}
    M, d = c["M"], c["d"]

    def new(shape, dtype):
        return torch.empty(shape, dtype=dtype, device="cuda")

    if c["kind"] == "moe":
        k["layer"] = P.MoeLayer(s["w13"], s["w2"], K=c["K"], router=s["router"],
                                expert_slot=s["slot"], gate_up_scale=s.get("s13"),
                                down_scale=s.get("s2"), renormalize=c["renorm"])
        k["out"] = new((M, d), torch.bfloat16)
        k["topk"] = new((M, c["K"]), torch.uint8)
        k["gates"] = new((M, c["K"]), torch.float32)
        k["ws"] = new((k["layer"].workspace_bytes(M),), torch.uint8)
    elif c["kind"] == "norm":
        k["h"], k["rstd"] = new((M, d), torch.bfloat16), new((M,), torch.float32)
        k["residual"] = new((M, d), DT[c["stream"]]) if c["residual"] else None
        k["q"] = new((M, d), torch.float8_e4m3fn) if c["bits8"] else None
        k["scale"] = new((M,), torch.float32) if c["bits8"] else None
    elif c["kind"] == "norm_grad":
        k["dx"], k["dw"] = new((M, d), DT[c["stream"]]), new((d,), torch.float32)
        k["ws"] = new((P.crc.crc_rms_norm_grad_workspace_bytes(M, d),), torch.uint8)
    else:
        k["q"], k["scale"] = new((M, d), torch.float8_e4m3fn), new((M,), torch.float32)
    return k


def _calls(s):
    c = s["c"]
    if "kept" not in s:
        s["kept"] = _kept(s)
    k = s["kept"]
    P = k["P"]
    if c["kind"] == "moe":
        k["layer"](s["x"], out=k["out"], x8=s.get("x8"), x_scale=s.get("xs"), topk=k["topk"],
                   gates=k["gates"], workspace=k["ws"])
        return {"out": k["out"], "topk": k["topk"], "gates": k["gates"]}
    if c["kind"] == "norm":
        P.rms_norm(s["x"], s["w"], EPS, residual=s["res"], residual_out=k["residual"], out=k["h"],
                   out8=k["q"], scale8=k["scale"], rstd=k["rstd"])
        names = ["h", "rstd"] + ["residual"] * c["residual"] + ["q", "scale"] * c["bits8"]
        return {n: k[n] for n in names}
    if c["kind"] == "norm_grad":
        P.rms_norm_grad(s["dy"], s["s"], s["w"], s["rstd"], dres=s["dres"], dx=k["dx"],
                        dw=k["dw"], workspace=k["ws"])
        return {"dx": k["dx"], "dw": k["dw"]}
    P.quantize_rows(s["x"], out8=k["q"], scale=k["scale"])
    return {"q": k["q"], "scale": k["scale"]}


def run(state):
    return _calls(state) if own else _plain(state)


# --------------------------------------------------------------------------- #
def work(case):
    """What a pass has to read, write and multiply, each array once."""
    c = case
    M, d = c["M"], c["d"]
    if c["kind"] == "moe":
        N, K, f = c["N"], c["K"], c["f"]
        active = N * (1.0 - (1.0 - K / N) ** M)         # experts that some token takes
        wb = 2 if c["weights"] == "bf16" else 1
        b = active * 3 * d * f * wb + N * d * 2 + 2 * M * d * 2 + M * K * 5
        if wb == 1:
            b += active * (2 * f + d) * 4
        if c["x8"]:
            b += M * (d + 4)
        return {"bytes": b, "flops": 2.0 * M * (K * 3 * d * f + N * d)}
    if c["kind"] == "norm":
        z = SIZE[c["stream"]]
        b = M * d * (z + 2 + (2 * z if c["residual"] else 0) + (1 if c["bits8"] else 0)) + 2 * d
        return {"bytes": b + M * 8, "flops": 6.0 * M * d}
    if c["kind"] == "norm_grad":
        z = SIZE[c["stream"]]
        return {"bytes": M * d * (2 + 2 * z + (z if c["dres"] else 0)) + M * 4 + d * 6,
                "flops": 10.0 * M * d}
    return {"bytes": M * d * 3 + M * 4, "flops": 3.0 * M * d}


# --------------------------------------------------------------------------- #
# the definitions in 64 bits
# --------------------------------------------------------------------------- #
def _exact_moe(s):
    c = s["c"]
    K = c["K"]
    z = s["x"].double() @ s["router"].double().t()
    p = torch.softmax(z, -1)
    ids = torch.sort(z, dim=-1, descending=True, stable=True).indices[:, :K]
    g = torch.gather(p, 1, ids)
    if c["renorm"]:
        g = g / g.sum(1, keepdim=True)
    x = s["x"].double()
    if c["x8"]:
        x = s["x8"].double() * s["xs"].double()[:, None]
    out = torch.zeros_like(x)
    where = s["slot"].tolist()
    for e in torch.unique(ids).tolist():
        m, k = torch.nonzero(ids == e, as_tuple=True)
        at = where[e]
        w13, w2 = s["w13"][at].double(), s["w2"][at].double()
        if "s13" in s:
            w13 = w13 * s["s13"][at].double()[..., None]
            w2 = w2 * s["s2"][at].double()[..., None]
        a, b = x[m] @ w13[0].t(), x[m] @ w13[1].t()
        y = (torch.nn.functional.silu(a) * b) @ w2.t()
        out.index_add_(0, m, y * g[m, k][:, None])
    return {"out": out, "topk": None, "gates": g}


def exact(case, seed):
    c = case
    s = _inputs(c, seed)
    if c["kind"] == "moe":
        return _exact_moe(s)
    if c["kind"] == "quantize":
        x = s["x"].double()
        a = x.abs().amax(1) / E4M3_MAX
        return {"q": x / a[:, None], "scale": a}
    r = s["w"].double()
    if c["kind"] == "norm":
        t = s["x"].double()
        out = {}
        if c["residual"]:
            t = out["residual"] = t + s["res"].double()
        out["rstd"] = (t.square().mean(1) + EPS) ** -0.5
        y = out["h"] = t * out["rstd"][:, None] * r
        if c["bits8"]:
            out["scale"] = y.abs().amax(1) / E4M3_MAX
            out["q"] = y / out["scale"][:, None]
        return out
    t = s["s"].double().requires_grad_(True)
    wd = r.clone().requires_grad_(True)
    # the statistics that the forward pass handed over stand for rsqrt(mean + eps)
    y = t * (t.square().mean(1, keepdim=True) + EPS) ** -0.5 * wd
    dt, dw = torch.autograd.grad((y * s["dy"].double()).sum(), (t, wd))
    if c["dres"]:
        dt = dt + s["dres"].double()
    return {"dx": dt, "dw": dw}
