"""The experts' products for prompts and training batches, and from 4-bit slots.

A prompt (or a training batch) has far more tokens than a decode step: its Top-K
choices are brought into the order of their experts, each expert's matrices
multiply that expert's rows, and every token sums its choices again.  A trainer
takes the gradients of those products and of the sum.  A decode step may read its
experts from slots that hold them in 4 bits, half the bytes of a transfer in 8.

Sizes are those of the repository's workloads (hidden sizes, experts, Top-K and
the expert widths that their expert bytes stand for) and generic ragged ones.
Hidden states have unit variance, expert rows N(0, 1 / row length); the router
likes some experts more than others.
"""
import math

import torch

own = False

E4M3_MAX = 448.0
DT = {"bf16": torch.bfloat16, "f32": torch.float32}

# experts, Top-K, hidden size, expert width, cache slots of the repository's workloads
SHAPES = {
    "tiny": dict(N=16, K=2, d=256, f=512, C=4),
    "gptoss": dict(N=32, K=4, d=2880, f=2880, C=8),
    "n64": dict(N=64, K=6, d=2048, f=1024, C=16),
    "qwen3": dict(N=128, K=8, d=2048, f=768, C=32),
    "large": dict(N=128, K=8, d=4096, f=1536, C=32),
}


def _case(name, kind, shape, M, **over):
    c = dict(name=name, kind=kind, shape=shape, **SHAPES[shape], M=M)
    c.update(over)
    return c


def listed():
    return [
        # a few tokens of the 32-expert backbone, an odd number: launches and latency only
        _case("choices-37", "choices", "gptoss", 37, padded=0),
        # a prompt batch, its last 700 tokens padding
        _case("choices-32768", "choices", "qwen3", 32768, padded=700),
        # a prompt's first product: rows gathered by token, gate and up, silu in the epilogue
        _case("products-gate-up-4096", "products", "qwen3", 4096, part="gate_up", weights="bf16"),
        # a short prompt's second product on 8-bit experts, rows in the experts' order
        _case("products-down-8bit-301", "products", "gptoss", 301, part="down", weights="e4m3"),
        # a trainer's second product: gradients of the rows and of all experts' matrices
        _case("products-grad-down-4096", "products_grad", "qwen3", 4096, part="down", dw="f32"),
        # a small batch's first product, ragged, rows gathered by token
        _case("products-grad-gate-up-613", "products_grad", "gptoss", 613, part="gate_up",
              dw="bf16"),
        # every token of a prompt sums its choices with their gates
        _case("sum-4096", "sum", "qwen3", 4096, gated=True),
        # the sum's gradient in an odd batch, gates' gradients too
        _case("sum-grad-1001", "sum_grad", "gptoss", 1001, gated=True),
        # one expert's gate and up, brought to 4 bits
        _case("quantize4-expert", "quantize4", "qwen3", 0, experts=1, part="gate_up", group=32),
        # a layer's gate and up matrices, all 64 experts, when a model is loaded
        _case("quantize4-layer", "quantize4", "n64", 0, experts=64, part="gate_up", group=64),
        # one decoded token, its 8 experts among the 32 resident slots: gate and up with silu
        _case("matvec4-gate-up-1", "matvec4", "qwen3", 1, part="gate_up", group=32, cached=True),
        # a serving batch of one token each: nearly every expert's second matrix is read
        _case("matvec4-down-64", "matvec4", "qwen3", 64, part="down", group=128, cached=False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["choices", "products", "products", "products", "products_grad",
                       "products_grad", "sum", "sum_grad", "quantize4", "matvec4", "matvec4",
                       "matvec4"])
    part = rng.choice(["gate_up", "down"])
    if kind == "choices":
        shape = rng.choice(list(SHAPES))
        M = _log_int(rng, 1, 32768)
        c = _case("", kind, shape, M, K=rng.randint(1, SHAPES[shape]["K"]),
                  padded=rng.randint(0, M // 3))
    elif kind == "products":
        weights = rng.choice(["bf16", "bf16", "e4m3"])
        shape = rng.choice(["tiny", "gptoss", "n64", "qwen3", "large"])
        most = {"tiny": 4096, "gptoss": 1500, "n64": 4096, "qwen3": 4096, "large": 1000}[shape]
        c = _case("", kind, shape, _log_int(rng, 1, most), part=part, weights=weights,
                  K=rng.randint(1, SHAPES[shape]["K"]))
    elif kind == "products_grad":
        shape = rng.choice(["tiny", "gptoss", "n64", "qwen3"])
        most = {"tiny": 4096, "gptoss": 613, "n64": 2000, "qwen3": 2000}[shape]
        c = _case("", kind, shape, _log_int(rng, 1, most), part=part, dw=rng.choice(["bf16", "f32"]),
                  K=rng.randint(1, SHAPES[shape]["K"]))
        if shape == "gptoss":
            c["dw"] = "bf16"
    elif kind in ("sum", "sum_grad"):
        shape = rng.choice(list(SHAPES))
        K = rng.randint(1, SHAPES[shape]["K"])
        c = _case("", kind, shape, _log_int(rng, 1, 16384 // K), K=K, d=8 * _log_int(rng, 16, 512),
                  gated=rng.random() < 0.75)
    elif kind == "quantize4":
        shape = rng.choice(["tiny", "gptoss", "n64", "qwen3"])
        group = rng.choice([32, 64]) if shape == "gptoss" else rng.choice([32, 64, 128])
        c = _case("", kind, shape, 0, experts=_log_int(rng, 1, 16), part=part, group=group)
    else:
        shape = rng.choice(["tiny", "gptoss", "n64", "qwen3", "qwen3", "large"])
        K = rng.randint(1, SHAPES[shape]["K"])
        M = _log_int(rng, 1, 100)
        group = rng.choice([32, 64]) if shape == "gptoss" else rng.choice([32, 64, 128])
        c = _case("", kind, shape, M, K=K, part=part, group=group,
                  cached=M * K <= SHAPES[shape]["C"])
    del c["name"]
    return c


# --------------------------------------------------------------------------- #
# inputs
# --------------------------------------------------------------------------- #
def _randn(g, shape, scale=1.0, dtype=torch.bfloat16):
    x = torch.randn(shape, device="cuda", generator=g, dtype=dtype)
    return x.mul_(scale) if scale != 1.0 else x


def _bits8(w):
    """e4m3 rows with one scale a row, amax / 448."""
    a = w.abs().amax(-1).float() / E4M3_MAX
    a = torch.where(a > 0, a, torch.ones_like(a))
    return (w / a.unsqueeze(-1)).to(torch.float8_e4m3fn), a


def _bits4(w, G):
    """Codes -7..7 (two a byte, the even column in the low half) and bf16 group scales."""
    v = w.unflatten(-1, (-1, G)).float()
    # (in 64 bits: a division by a plain number is a product with its reciprocal)
    a = (v.abs().amax(-1).double() / 7).to(torch.bfloat16)
    a = torch.where(a > 0, a, torch.ones_like(a))
    q = torch.round(v / a.float().unsqueeze(-1)).clamp_(-7, 7).flatten(-2).to(torch.int8)
    q = q.view(torch.uint8) & 15
    return q[..., 0::2] | (q[..., 1::2] << 4), a.transpose(-1, -2).contiguous()


def _choices(c, g):
    """Top-K of router logits that like some experts more than others, and their gates."""
    z = _randn(g, (c["M"], c["N"]), dtype=torch.float32)
    z = z + 0.7 * _randn(g, (c["N"],), dtype=torch.float32)
    top = z.topk(c["K"], dim=-1)
    return top.indices.to(torch.uint8), torch.softmax(top.values, -1)


def _order(c, s):
    """The choices in their experts' order, as group_choices defines it; host counts too."""
    flat = s["topk"].flatten().long()
    s["rows"] = torch.argsort(flat, stable=True).to(torch.int32)
    counts = torch.bincount(flat, minlength=c["N"])
    s["offsets"] = torch.zeros(c["N"] + 1, dtype=torch.int32, device="cuda")
    s["offsets"][1:] = counts.cumsum(0).to(torch.int32)
    s["counts"] = counts.tolist()
    s["place"] = torch.empty_like(s["rows"])
    s["place"][s["rows"].long()] = torch.arange(flat.numel(), dtype=torch.int32, device="cuda")
    s["place"] = s["place"].view(c["M"], c["K"])


def _matrices(c, g, slots):
    if c["part"] == "gate_up":
        return _randn(g, (slots, 2, c["f"], c["d"]), c["d"] ** -0.5)
    return _randn(g, (slots, c["d"], c["f"]), c["f"] ** -0.5)


def _inputs(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"c": c}
    kind, M, N, K, d, f = c["kind"], c["M"], c["N"], c["K"], c["d"], c["f"]
    E = M * K
    if kind == "quantize4":
        s["x"] = _matrices(c, g, c["experts"])
        return s
    s["topk"], s["gates"] = _choices(c, g)
    if kind == "choices":
        if c["padded"]:
            s["topk"][M - c["padded"]:] = 255
        return s
    if kind in ("products", "products_grad"):
        _order(c, s)
        s["w"] = _matrices(c, g, N)
        # the first product reads tokens, the second what the first one made of each choice
        s["x"] = _randn(g, (M, d)) if c["part"] == "gate_up" else _randn(g, (E, f), 0.5)
        if kind == "products" and c["weights"] == "e4m3":
            s["w"], s["ws"] = _bits8(s["w"])
            s["x"], s["xs"] = _bits8(s["x"])
        if kind == "products_grad":
            s["w"] = s["w"].flatten(1, -2)
            s["dy"] = _randn(g, (E, s["w"].shape[1]), 1e-2)
    elif kind in ("sum", "sum_grad"):
        _order(c, s)
        s["y"] = _randn(g, (E, d))
        if kind == "sum_grad":
            s["dout"] = _randn(g, (M, d), 1e-2)
    else:
        slots = c["C"] if c["cached"] else N
        s["w"], s["ws"] = _bits4(_matrices(c, g, slots), c["group"])
        s["x"] = _randn(g, (M, d)) if c["part"] == "gate_up" else _randn(g, (M, K, f), 0.5)
        # where each expert lies: everywhere in a full layer, or (cached) the experts of
        # this step's tokens and some others in the slots there are
        order = torch.randperm(N, device="cuda", generator=g)
        wanted = torch.zeros(N, dtype=torch.bool, device="cuda")
        wanted[s["topk"].flatten().long()] = True
        order = order[torch.argsort(wanted[order].logical_not(), stable=True)]
        s["slot"] = torch.full((N,), -1, dtype=torch.int32, device="cuda")
        at = torch.randperm(slots, device="cuda", generator=g).to(torch.int32)
        s["slot"][order[:slots]] = at
    return s


def prepare(case, seed):
    return _inputs(case, seed)


# --------------------------------------------------------------------------- #
# plain forms: 32 bits, rounded once
# --------------------------------------------------------------------------- #
def _glu(gate, up):
    return gate / (1.0 + torch.exp(-gate)) * up


def _plain_choices(s):
    c = s["c"]
    N, E = c["N"], c["M"] * c["K"]
    flat = s["topk"].flatten().long()
    valid = flat < N
    order = torch.sort(torch.where(valid, flat, N), stable=True)
    rows = torch.where(order.values < N, order.indices, -1).to(torch.int32)
    offsets = (flat[None, :] < torch.arange(N + 1, device="cuda")[:, None]).sum(1).to(torch.int32)
    place = torch.empty(E, dtype=torch.int32, device="cuda")
    place[order.indices] = torch.arange(E, dtype=torch.int32, device="cuda")
    place = torch.where(valid, place, -1)
    return {"offsets": offsets, "rows": rows, "place": place.view(c["M"], c["K"])}


def _groups(s):
    at = 0
    for e, n in enumerate(s["counts"]):
        if n:
            yield e, at, at + n
        at += n


def _rows_of(s, a, b):
    """The rows of x that sorted choices a .. b - 1 multiply."""
    if s["c"]["part"] == "gate_up":
        at = s["rows"][a:b].long() // s["c"]["K"]
        return s["x"][at].float(), (s["xs"][at] if "xs" in s else None)
    return s["x"][a:b].float(), (s["xs"][a:b] if "xs" in s else None)


def _plain_products(s):
    c = s["c"]
    E = c["M"] * c["K"]
    y = torch.empty((E, s["w"].shape[-2]), dtype=torch.bfloat16, device="cuda")
    for e, a, b in _groups(s):
        x, xs = _rows_of(s, a, b)
        w = s["w"][e].float()
        if xs is not None:
            x, w = x * xs[:, None], w * s["ws"][e][..., None]
        if c["part"] == "gate_up":
            y[a:b] = _glu(x @ w[0].t(), x @ w[1].t()).to(torch.bfloat16)
        else:
            y[a:b] = (x @ w.t()).to(torch.bfloat16)
    return {"y": y}


def _plain_products_grad(s):
    c = s["c"]
    dx = torch.empty((c["M"] * c["K"], s["w"].shape[2]), dtype=torch.bfloat16, device="cuda")
    dw = torch.zeros(s["w"].shape, dtype=DT[c["dw"]], device="cuda")
    for e, a, b in _groups(s):
        x, _ = _rows_of(s, a, b)
        dy = s["dy"][a:b].float()
        dx[a:b] = (dy @ s["w"][e].float()).to(torch.bfloat16)
        dw[e] = (dy.t() @ x).to(DT[c["dw"]])
    return {"dx": dx, "dw": dw}


def _plain_sum(s):
    y = s["y"][s["place"].long()].float()                   # [M][K][d]
    if s["c"]["gated"]:
        y = y * s["gates"][..., None]
    return {"out": y.sum(1).to(torch.bfloat16)}


def _plain_sum_grad(s):
    c = s["c"]
    place = s["place"].long()
    do = s["dout"].float()[:, None].expand(-1, c["K"], -1)
    out = {}
    dy = torch.empty((c["M"] * c["K"], c["d"]), dtype=torch.bfloat16, device="cuda")
    if c["gated"]:
        out["dgates"] = (do * s["y"][place].float()).sum(-1)
        do = do * s["gates"][..., None]
    dy[place.flatten()] = do.flatten(0, 1).to(torch.bfloat16)
    out["dy"] = dy
    return out


def _values4(q, scale):
    """What 4-bit codes [..][n][k / 2] with scales [..][k / G][n] stand for, in 32 bits."""
    lo, hi = (q & 15).to(torch.int8), (q >> 4).to(torch.int8)
    v = torch.stack((lo, hi), -1).flatten(-2)
    v = torch.where(v > 7, v - 16, v).float()
    groups = scale.shape[-2]
    v = v.unflatten(-1, (groups, -1)) * scale.transpose(-1, -2).float()[..., None]
    return v.flatten(-2)


def _plain_quantize4(s):
    # the codes are whole numbers, two a byte, as a program keeps them
    q, a = _bits4(s["x"], s["c"]["group"])
    return {"q": q, "scale": a}


def _plain_matvec4(s):
    c = s["c"]
    M, K = c["M"], c["K"]
    at = s["slot"].long()[s["topk"].long()]                             # [M][K]
    x = s["x"].float()
    if c["part"] == "gate_up":
        x = x[:, None].expand(M, K, c["d"])
    y = torch.empty((M, K, s["w"].shape[-2]), dtype=torch.bfloat16, device="cuda")
    for m in range(0, M, 4):                # a few tokens' matrices at a time
        w = _values4(s["w"][at[m:m + 4]], s["ws"][at[m:m + 4]])         # [4][K](2)[n][k]
        v = x[m:m + 4, :, :, None]
        if c["part"] == "gate_up":
            r = _glu((w[:, :, 0] @ v)[..., 0], (w[:, :, 1] @ v)[..., 0])
        else:
            r = (w @ v)[..., 0]
        y[m:m + 4] = r.to(torch.bfloat16)
    return {"y": y}


PLAIN = {"choices": _plain_choices, "products": _plain_products,
         "products_grad": _plain_products_grad, "sum": _plain_sum, "sum_grad": _plain_sum_grad,
         "quantize4": _plain_quantize4, "matvec4": _plain_matvec4}


# --------------------------------------------------------------------------- #
# the framework's operators, with the buffers that a program keeps
# --------------------------------------------------------------------------- #
def _kept(s):
    """Outputs and workspaces of a program's own, made once."""
    import paper_2609_04895_gb300 as P
    c, k = s["c"], {"P": P}
    kind, M, N, K, d = c["kind"], c["M"], c["N"], c["K"], c["d"]
    E = M * K

    def new(shape, dtype):
        return torch.empty(shape, dtype=dtype, device="cuda")

    if kind == "choices":
        k["offsets"], k["rows"] = new((N + 1,), torch.int32), new((E,), torch.int32)
        k["place"] = new((M, K), torch.int32)
        k["ws"] = new((P.crc.crc_group_choices_workspace_bytes(M, K, N),), torch.uint8)
    elif kind == "products":
        k["y"] = new((E, s["w"].shape[-2]), torch.bfloat16)
    elif kind == "products_grad":
        k["dx"] = new((E, s["w"].shape[2]), torch.bfloat16)
        k["dw"] = new(s["w"].shape, DT[c["dw"]])
    elif kind == "sum":
        k["out"] = new((M, d), torch.bfloat16)
    elif kind == "sum_grad":
        k["dy"] = new((E, d), torch.bfloat16)
        k["dgates"] = new((M, K), torch.float32) if c["gated"] else None
    elif kind == "quantize4":
        *lead, n, cols = s["x"].shape
        k["q"] = new((*lead, n, cols // 2), torch.uint8)
        k["scale"] = new((*lead, cols // c["group"], n), torch.bfloat16)
    else:
        k["y"] = new((M, K, s["w"].shape[-2]), torch.bfloat16)
    return k


def _calls(s):
    c = s["c"]
    if "kept" not in s:
        s["kept"] = _kept(s)
    k = s["kept"]
    P, kind = k["P"], c["kind"]
    if kind == "choices":
        P.group_choices(s["topk"], c["N"], offsets=k["offsets"], rows=k["rows"], place=k["place"],
                        workspace=k["ws"])
        return {n: k[n] for n in ("offsets", "rows", "place")}
    if kind in ("products", "products_grad"):
        # tokens are gathered by their choices' rows; the second product's are in order
        by = dict(rows=s["rows"], K=c["K"]) if c["part"] == "gate_up" else {}
        if kind == "products":
            P.group_matmul(s["x"], s["w"], s["offsets"], x_scale=s.get("xs"), w_scale=s.get("ws"),
                           y=k["y"], **by)
            return {"y": k["y"]}
        P.group_matmul_grad(s["dy"], s["x"], s["w"], s["offsets"], dx=k["dx"], dw=k["dw"], **by)
        return {"dx": k["dx"], "dw": k["dw"]}
    gates = s["gates"] if c.get("gated") else None
    if kind == "sum":
        P.sum_choices(s["y"], s["place"], gates=gates, out=k["out"])
        return {"out": k["out"]}
    if kind == "sum_grad":
        P.sum_choices_grad(s["dout"], s["place"], gates=gates, y=s["y"] if c["gated"] else None,
                           dy=k["dy"], dgates=k["dgates"])
        return {n: k[n] for n in ("dgates", "dy") if k[n] is not None}
    if kind == "quantize4":
        P.quantize_rows4(s["x"], c["group"], out4=k["q"], scale=k["scale"])
        return {"q": k["q"], "scale": k["scale"]}
    P.matvec4(s["x"], s["w"], s["ws"], topk=s["topk"], expert_slot=s["slot"], y=k["y"])
    return {"y": k["y"]}


def run(state):
    return _calls(state) if own else PLAIN[state["c"]["kind"]](state)


# --------------------------------------------------------------------------- #
def work(case):
    """What a pass has to read, write and multiply, each array once."""
    c = case
    kind, M, N, K, d, f = c["kind"], c["M"], c["N"], c["K"], c["d"], c["f"]
    E = M * K
    active = N * (1.0 - (1.0 - K / N) ** M)             # experts that some token takes
    n, k = (2 * f, d) if c.get("part") == "gate_up" else (d, f)
    out = f if c.get("part") == "gate_up" else d        # columns after the silu
    xrows = M if c.get("part") == "gate_up" else E
    if kind == "choices":
        return {"bytes": 9 * E + 4 * N, "flops": 0.0}
    if kind == "products":
        wb = 2 if c["weights"] == "bf16" else 1
        b = active * n * k * wb + xrows * k * wb + E * out * 2
        if wb == 1:
            b += active * n * 4 + xrows * 4
        return {"bytes": b + 4 * E * (c["part"] == "gate_up"), "flops": 2.0 * E * n * k}
    if kind == "products_grad":
        z = 2 if c["dw"] == "bf16" else 4
        b = active * n * k * 2 + N * n * k * z + 2 * (E * n + xrows * k + E * k)
        return {"bytes": b + 4 * E * (c["part"] == "gate_up"), "flops": 4.0 * E * n * k}
    if kind == "sum":
        return {"bytes": 2 * d * (E + M) + E * (8 if c["gated"] else 4),
                "flops": 2.0 * E * d}
    if kind == "sum_grad":
        b = 2 * d * (E + M) + 4 * E
        if c["gated"]:
            b += 2 * d * E + 8 * E
        return {"bytes": b, "flops": (3.0 if c["gated"] else 0.0) * E * d}
    if kind == "quantize4":
        return {"bytes": c["experts"] * n * k * (2.5 + 2.0 / c["group"]),
                "flops": 3.0 * c["experts"] * n * k}
    return {"bytes": active * n * k * (0.5 + 2.0 / c["group"]) + 2 * xrows * k + 2 * E * out + E,
            "flops": 2.0 * E * n * k}


# --------------------------------------------------------------------------- #
# the definitions in 64 bits
# --------------------------------------------------------------------------- #
def _exact_products(s):
    c = s["c"]
    K = c["K"]
    ids = s["topk"].flatten()
    pos = s["place"].flatten().long()
    x = s["x"].double()
    if "xs" in s:
        x = x * s["xs"].double()[:, None]
    y = torch.zeros((ids.numel(), s["w"].shape[-2]), dtype=torch.float64, device="cuda")
    for e in torch.unique(ids).tolist():
        ch = torch.nonzero(ids == e).squeeze(1)
        w = s["w"][e].double()
        if "ws" in s:
            w = w * s["ws"][e].double()[..., None]
        if c["part"] == "gate_up":
            v = torch.einsum("rk,hnk->hrn", x[torch.div(ch, K, rounding_mode="floor")], w)
            y[pos[ch]] = torch.nn.functional.silu(v[0]) * v[1]
        else:
            y[pos[ch]] = torch.einsum("rk,nk->rn", x[pos[ch]], w)
    return {"y": y}


def _exact_products_grad(s):
    c = s["c"]
    K = c["K"]
    ids = s["topk"].flatten()
    pos = s["place"].flatten().long()
    dx = torch.zeros((ids.numel(), s["w"].shape[2]), dtype=torch.float64, device="cuda")
    dw = torch.zeros(s["w"].shape, dtype=torch.float64, device="cuda")
    for e in torch.unique(ids).tolist():
        ch = torch.nonzero(ids == e).squeeze(1)
        src = torch.div(ch, K, rounding_mode="floor") if c["part"] == "gate_up" else pos[ch]
        x = s["x"][src].double().requires_grad_(True)
        w = s["w"][e].double().requires_grad_(True)
        gx, gw = torch.autograd.grad(torch.einsum("rk,nk->rn", x, w), (x, w),
                                     s["dy"][pos[ch]].double())
        dx[pos[ch]], dw[e] = gx, gw
    return {"dx": dx, "dw": dw}


def _exact_sum(s):
    c = s["c"]
    y = s["y"].double().requires_grad_(True)
    g = s["gates"].double() if c["gated"] else torch.ones_like(s["gates"], dtype=torch.float64)
    g.requires_grad_(True)
    out = torch.zeros((c["M"], c["d"]), dtype=torch.float64, device="cuda")
    for j in range(c["K"]):
        out = out + g[:, j, None] * y.index_select(0, s["place"][:, j].long())
    if c["kind"] == "sum":
        return {"out": out.detach()}
    dy, dg = torch.autograd.grad(out, (y, g), s["dout"].double())
    return {"dgates": dg, "dy": dy} if c["gated"] else {"dy": dy}


def _exact_matvec4(s):
    c = s["c"]
    G, K = c["group"], c["K"]
    ids = s["topk"].flatten()
    x = s["x"].double()
    y = torch.zeros((ids.numel(), s["w"].shape[-2]), dtype=torch.float64, device="cuda")
    where = s["slot"].tolist()
    for e in torch.unique(ids).tolist():
        q = s["w"][where[e]].to(torch.int32)
        w = torch.empty((*q.shape[:-1], 2 * q.shape[-1]), dtype=torch.float64, device="cuda")
        w[..., 0::2] = ((q % 16 + 8) % 16 - 8).double()
        w[..., 1::2] = ((q // 16 + 8) % 16 - 8).double()
        w = w * s["ws"][where[e]].double().mT.repeat_interleave(G, dim=-1)
        ch = torch.nonzero(ids == e).squeeze(1)
        if c["part"] == "gate_up":
            v = torch.einsum("rk,hnk->hrn", x[torch.div(ch, K, rounding_mode="floor")], w)
            y[ch] = torch.nn.functional.silu(v[0]) * v[1]
        else:
            y[ch] = torch.einsum("rk,nk->rn", x.flatten(0, 1)[ch], w)
    return {"y": y.view(c["M"], K, -1)}


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "choices":
        return None                                     # whole numbers
    if kind == "quantize4":
        a = s["x"].double().unflatten(-1, (-1, case["group"])).abs().amax(-1) / 7
        return {"q": None, "scale": a.mT}
    return {"products": _exact_products, "products_grad": _exact_products_grad,
            "sum": _exact_sum, "sum_grad": _exact_sum, "matvec4": _exact_matvec4}[kind](s)
