"""Timed cases of two operators of a training epoch: group norm with an activation over vertex features (rows are
vertices, channels last) and the AdamW step over many tensors at once, with clipping by the norm of all gradients.

``own`` false: the operators from elementary torch operations.  ``own`` true: the calls a user makes of the package
(Graph.dg_group_norm_fwd / _bwd, optim.AdamW.step).

A case of group norm: ``n`` rows of ``F`` channels in ``groups`` groups; ``graphs`` graphs share the rows (1: one
graph of all rows; more: ragged ones, some of them empty, ``behind`` rows behind the last one belong to none);
``x`` and ``y`` name the types of the input and of the output.  A case of AdamW: ``tensors`` names a list of
parameter shapes (see shapes()); ``param`` is their type, ``bits`` what a number of the two states takes,
``master``: fp32 master weights next to bf16 parameters; ``clip``: the largest norm of all gradients, 0 for no limit.
"""
from __future__ import annotations

import math
import random

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
EPS = 1e-5                                        # of the norm
LR, BETA1, BETA2, ADAM_EPS, DECAY = 1e-3, 0.9, 0.999, 1e-8, 0.01
BLOCK = 256                                       # 8-bit numbers that share a scale
LARGEST = 448.0                                   # of e4m3
WIDTHS = [8, 16, 41, 47, 64, 100, 128, 172, 256, 602]


def norm(name, kind, n, F, groups, act, x="f32", y="f32", graphs=1, behind=0):
    return {"name": name, "kind": kind, "n": n, "F": F, "groups": groups, "act": act, "x": x, "y": y,
            "graphs": graphs, "behind": behind}


def adamw(name, tensors, rows=0, width=0, count=0, param="f32", bits=32, master=False, clip=0.0):
    return {"name": name, "kind": "adamw", "tensors": tensors, "rows": rows, "width": width, "count": count,
            "param": param, "bits": bits, "master": master, "clip": clip}


def listed():
    return [
        # a small graph between two layers: launches count
        norm("norm fwd tiny", "fwd", 4096, 64, 8, "relu"),
        # hidden activations of a Reddit-like graph
        norm("norm fwd reddit", "fwd", 232965, 256, 32, "relu"),
        # a matrix far larger than the L2, stored as bf16 for the aggregation that gathers it next
        norm("norm fwd products bf16", "fwd", 2449029, 100, 20, "silu", "bf16", "bf16"),
        # a batch of graphs of very different sizes, with padding behind it; normalised rows leave as bf16
        norm("norm fwd batch", "fwd", 132534, 128, 8, "silu", "f32", "bf16", graphs=2048, behind=500),
        # class scores of a small graph: odd rows, one group
        norm("norm bwd odd", "bwd", 24490, 47, 1, "none"),
        norm("norm bwd reddit", "bwd", 232965, 256, 32, "relu"),
        norm("norm bwd batch", "bwd", 132534, 128, 8, "silu", "f32", "bf16", graphs=2048, behind=500),
        # the parameters of a three-layer model: the step is launches and host time
        adamw("adamw layers", "model", width=100, clip=1.0),
        # learnable features of every vertex, and the model
        adamw("adamw features", "features", 2449029, 100, clip=1.0),
        # the same with both states in 8 bits
        adamw("adamw8 features", "features", 2449029, 100, bits=8),
        # many tensors of odd sizes in bf16
        adamw("adamw8 many", "many", count=120, param="bf16", bits=8, clip=1.0),
        # bf16 features that a bf16 aggregation gathers, with fp32 master weights
        adamw("adamw master", "features", 232965, 602, param="bf16", master=True),
    ]


def shapes(case):
    """The parameters' shapes: of a model of three layers (dims width, 256, 256, 47) with norms between them; with a
    rows x width matrix of features before them; or `count` tensors of 4097 to about 2 M numbers."""
    if case["tensors"] == "many":
        rng = random.Random(case["count"])
        return [(int(math.exp(rng.uniform(math.log(4097), math.log(2e6)))) | 1,) for _ in range(case["count"])]
    first = [(case["rows"], case["width"])] if case["tensors"] == "features" else []
    dims = [case["width"], 256, 256, 47]
    rest = []
    for i in range(3):
        rest += [(dims[i + 1], dims[i]), (dims[i + 1],)]
        rest += [(dims[i + 1],), (dims[i + 1],)] if i < 2 else []
    return first + rest


def numbers(case):
    return [math.prod(s) for s in shapes(case)]


def work(case):
    if case["kind"] == "adamw":
        count = float(sum(numbers(case)))
        p = SIZE[case["param"]]
        each = 2 * (4 if case["master"] else p) + p + 4 * case["bits"] / 8 + (p if case["master"] else 0)
        scales = 16.0 * count / BLOCK if case["bits"] == 8 else 0.0
        return {"bytes": count * each + scales, "flops": 12.0 * count}
    cells = float(case["n"] - case["behind"]) * case["F"]
    x, y = SIZE[case["x"]], SIZE[case["y"]]
    stats = 8.0 * case["graphs"] * case["groups"]
    each, flops = (x + y, 10.0) if case["kind"] == "fwd" else (2 * x + y, 20.0)
    return {"bytes": cells * each + stats + 8.0 * case["F"] * (1 if case["kind"] == "fwd" else 3), "flops": cells * flops}


def between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Any operator, type and direction; sizes spread over their logarithm."""
    most = max(work(c)["bytes"] for c in listed())
    while True:
        if rng.random() < 0.6:
            F = rng.choice(WIDTHS) if rng.random() < 0.5 else between(rng, 4, 1024)
            groups = rng.choice([g for g in range(1, F + 1) if F % g == 0])
            n = between(rng, 500, 2.5e6)
            graphs = 1 if rng.random() < 0.5 else between(rng, 2, max(3, min(20000, n // 8)))
            x, y = rng.choice([("f32", "f32"), ("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32")])
            behind = rng.choice([0, rng.randint(1, n // 8)]) if graphs > 1 else 0
            case = norm("", rng.choice(["fwd", "bwd"]), n, F, groups, rng.choice(["none", "relu", "silu"]), x, y, graphs, behind)
        else:
            param = rng.choice(["f32", "bf16"])
            case = adamw("", rng.choice(["model", "features", "many"]), between(rng, 100, 1e6), between(rng, 8, 602),
                         between(rng, 2, 200), param, rng.choice([8, 32]), param == "bf16" and rng.random() < 0.5,
                         rng.choice([0.0, 1.0]))
            if case["tensors"] == "many":
                case["rows"] = case["width"] = 0
            else:
                case["count"] = 0
                case["rows"] *= case["tensors"] == "features"
        del case["name"]
        if work(case)["bytes"] <= most:
            return case


# ---- inputs ----------------------------------------------------------------------------------

def bounds(case, seed):
    """Where the graphs of a batch begin and end: sizes spread over a factor of a thousand, one in 64 graphs empty."""
    end = case["n"] - case["behind"]
    if case["graphs"] == 1:
        return [0, end]
    rng = random.Random(seed)
    size = [0.0 if rng.random() < 1 / 64 else math.exp(rng.gauss(0, 1.2)) for _ in range(case["graphs"])]
    size[rng.randrange(case["graphs"])] += 1e-3
    total, run_, cut = sum(size), 0.0, [0]
    for s in size:
        run_ += s
        cut.append(min(end, int(round(end * run_ / total))))
    cut[-1] = end
    return cut


def groups_of(case, seed, gen):
    """Inputs of group norm: channels of different means and spreads, as a Linear layer leaves them."""
    n, F, dev = case["n"], case["F"], "cuda"
    spread = torch.exp(0.5 * torch.randn(F, generator=gen, device=dev))
    X = torch.randn((n, F), generator=gen, device=dev).mul_(spread).add_(0.7 * torch.randn(F, generator=gen, device=dev))
    X = X.to(TYPES[case["x"]])
    weight = 1 + 0.2 * torch.randn(F, generator=gen, device=dev)
    bias = 0.2 * torch.randn(F, generator=gen, device=dev)
    cut = bounds(case, seed)
    st = {"case": case, "X": X, "weight": weight, "bias": bias, "bounds": torch.tensor(cut, dtype=torch.int64, device=dev)}
    if case["kind"] == "fwd":
        st["Y"] = torch.full((n, F), 0.5, dtype=TYPES[case["y"]], device=dev)
    else:
        st["dY"] = (torch.randn((n, F), generator=gen, device=dev) * 1e-2).to(TYPES[case["y"]])
        st["dX"] = torch.full((n, F), 0.5, dtype=TYPES[case["x"]], device=dev)
        st["stats"] = statistics(X, st["bounds"], case["groups"])[0]
    if own:
        from paper_2104_06700_b200 import binding
        empty = torch.zeros(n + 1, dtype=torch.int64, device=dev), torch.zeros(0, dtype=torch.int32, device=dev)
        st["graph"] = binding.dg_graph_create(n, 0, *empty, None)   # the norm does not look at the edges
        if case["graphs"] > 1:
            st["graph"].dg_graph_set_batch(torch.tensor(cut, dtype=torch.int64))
        st["act"] = {"none": binding.DG_ACT_NONE, "relu": binding.DG_ACT_RELU, "silu": binding.DG_ACT_SILU}[case["act"]]
    return st


def parameters_of(case, seed, gen):
    """Parameters, gradients and states after 100 steps, each kind in one flat tensor in which every parameter begins at a
    multiple of 256 numbers.  The gradients of a third of the features' rows are zero: their vertices were not reached."""
    dev, count = "cuda", numbers(case)
    blocks = [(c + BLOCK - 1) // BLOCK for c in count]
    total = sum(blocks) * BLOCK
    first = [0]
    for b in blocks:
        first.append(first[-1] + b)
    ids = torch.repeat_interleave(torch.arange(len(count), device=dev), torch.tensor(blocks, device=dev))
    start = torch.tensor(first[:-1], device=dev)[ids] * BLOCK
    at = torch.arange(total, device=dev).view(-1, BLOCK) - start.view(-1, 1)
    inside = (at < torch.tensor(count, device=dev)[ids].view(-1, 1)).view(-1)
    del at
    size = torch.exp(torch.randn(len(count), generator=gen, device=dev))[ids].view(-1, 1) * 1e-3
    alive = inside.view(-1, BLOCK)
    if case["tensors"] == "features":
        reached = torch.rand(case["rows"], generator=gen, device=dev) < 2 / 3
        alive = alive.clone()
        alive.view(-1)[:count[0]] &= reached.repeat_interleave(case["width"])

    def noise():
        return torch.randn((total // BLOCK, BLOCK), generator=gen, device=dev)

    g = (noise() * size * alive).view(-1)
    m = (noise() * size * 0.3 * alive).view(-1)
    u = ((noise().square_().add_(0.5)).sqrt_() * size * alive).view(-1)
    p = (noise() * 0.1).view(-1) * inside
    st = {"case": case, "g": g.to(TYPES[case["param"]]), "p": p.to(TYPES[case["param"]]), "ids": ids, "start": start,
          "step": torch.full((len(count),), 100, dtype=torch.int64, device=dev)}
    del g, alive, inside
    if case["master"]:
        st["master"] = p
    if case["bits"] == 8:
        largest = torch.stack([m.view(-1, BLOCK).abs().amax(1), u.view(-1, BLOCK).amax(1)], 1)
        st["scales"] = (largest / LARGEST).clamp_(min=2.0 ** -126)
        st["m"] = (m.view(-1, BLOCK) / st["scales"][:, :1]).to(torch.float8_e4m3fn).view(-1)
        u = u.view(-1, BLOCK) / st["scales"][:, 1:]
        st["v"] = torch.where(u > 0, u.clamp(2.0 ** -9, LARGEST), u).to(torch.float8_e4m3fn).view(-1)
    else:
        st["m"], st["v"] = m, u.square_()
    if own:
        from paper_2104_06700_b200 import optim
        params, cut = [], [(f * BLOCK, f * BLOCK + c) for f, c in zip(first, count)]
        for (a, b), shape in zip(cut, shapes(case)):
            params.append(torch.nn.Parameter(st["p"][a:b].view(shape)))
            params[-1].grad = st["g"][a:b].view(shape)
        opt = optim.AdamW(params, lr=LR, betas=(BETA1, BETA2), eps=ADAM_EPS, weight_decay=DECAY, state_bits=case["bits"],
                          min_8bit_size=1, master_weights=case["master"], max_norm=case["clip"] or None, seed=seed)
        for i, (q, (a, b), f, k) in enumerate(zip(params, cut, first, blocks)):
            s = opt.state[q]
            s["step"], s["exp_avg"], s["exp_avg_sq"] = st["step"][i], st["m"][a:b], st["v"][a:b]
            if case["bits"] == 8:
                s["scales"] = st["scales"][f:f + k]
            if case["master"]:
                s["master"] = st["master"][a:b]
        st["opt"] = opt
    st["seed"] = seed
    return st


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return parameters_of(case, seed, gen) if case["kind"] == "adamw" else groups_of(case, seed, gen)


# ---- plain forms -----------------------------------------------------------------------------

def graph_of_row(cut):
    return torch.repeat_interleave(torch.arange(cut.numel() - 1, device=cut.device), cut[1:] - cut[:-1])


def mean_of(values, row, cut, groups):
    """The mean of an (rows, F) matrix over each graph and group, (graphs, groups); long sums in 64 bits."""
    graphs, width = cut.numel() - 1, values.shape[1] // groups
    sums = values.view(-1, groups, width).sum(2, dtype=torch.float64)
    if graphs == 1:
        total = sums.sum(0, keepdim=True)
    else:
        total = torch.zeros((graphs, groups), dtype=torch.float64, device=values.device).index_add_(0, row, sums)
    return total / ((cut[1:] - cut[:-1]).clamp(min=1).double() * width).view(-1, 1)


def per_row(values, row, width):
    """(graphs, groups) to one value for each cell."""
    each = values.expand(row.numel(), -1) if values.shape[0] == 1 else values[row]
    return each.repeat_interleave(width, 1)


def statistics(X, cut, groups):
    """(mean, 1 / sqrt(variance + eps)) of every graph and group, and which graph a row belongs to."""
    row = graph_of_row(cut)
    x = X[:row.numel()].float()
    mean = mean_of(x, row, cut, groups)
    off = x - per_row(mean.float(), row, X.shape[1] // groups)
    var = mean_of(off.square_(), row, cut, groups)
    return torch.stack([mean, (var + EPS).rsqrt()], 2).float(), row


def activate(z, act):
    return torch.relu(z) if act == "relu" else z * torch.sigmoid(z) if act == "silu" else z


def norm_forward(st):
    case, X, Y = st["case"], st["X"], st["Y"]
    stats, row = statistics(X, st["bounds"], case["groups"])
    width = case["F"] // case["groups"]
    hat = (X[:row.numel()].float() - per_row(stats[..., 0], row, width)) * per_row(stats[..., 1], row, width)
    Y[:row.numel()] = activate(hat * st["weight"] + st["bias"], case["act"]).to(Y.dtype)
    return {"Y": Y, "stats": stats}


def norm_backward(st):
    case, dX, stats, cut, groups = st["case"], st["dX"], st["stats"], st["bounds"], st["case"]["groups"]
    row, width = graph_of_row(cut), case["F"] // groups
    rstd = per_row(stats[..., 1], row, width)
    hat = (st["X"][:row.numel()].float() - per_row(stats[..., 0], row, width)) * rstd
    d = st["dY"][:row.numel()].float()
    if case["act"] == "relu":       # 0 is a border: in 64 bits
        z = st["X"][:row.numel()].double() - per_row(stats[..., 0].double(), row, width)
        z = z.mul_(rstd).mul_(st["weight"]).add_(st["bias"])
        d = torch.where(z <= 0, 0.0, d)
    elif case["act"] == "silu":
        z = hat * st["weight"] + st["bias"]
        s = torch.sigmoid(z)
        d = d * (s * (1 + z * (1 - s)))
    dbias, dweight = d.sum(0, dtype=torch.float64).float(), (d * hat).sum(0, dtype=torch.float64).float()
    d = d * st["weight"]
    a = per_row(mean_of(d, row, cut, groups).float(), row, width)
    b = per_row(mean_of(d * hat, row, cut, groups).float(), row, width)
    dX[:row.numel()] = ((d - a - hat * b) * rstd).to(dX.dtype)
    return {"dX": dX, "dweight": dweight, "dbias": dbias}


LOW = 0xFFFFFFFF


def mix(x):
    """A 32-bit hash (lowbias32 of Chris Wellons) of whole numbers below 2^32, kept in 64 bits."""
    x = x ^ (x >> 16)
    x = (x * 0x7FEB352D) & LOW
    x = x ^ (x >> 15)
    x = (x * 0x846CA68B) & LOW
    return x ^ (x >> 16)


def random_bits(st):
    """32 random bits for every number: a hash of the seed, the step, the tensor and the place in it."""
    seed, ids = st["seed"], st["ids"]
    k = mix(mix((seed & LOW) + 0x9E3779B9 & LOW) ^ (seed >> 32 & LOW))
    key = mix(mix((k + st["step"]) & LOW)[ids] ^ ids)
    at = torch.arange(st["p"].numel(), device=ids.device).view(-1, BLOCK) - st["start"].view(-1, 1)
    return mix(((at & LOW) + mix(key.view(-1, 1) ^ (at >> 32))) & LOW)


def to_8_bits(x, r):
    """e4m3 numbers, and their scales, of the rows of x; r: 16 random bits for each, which round it up or down."""
    scale = (x.abs().amax(1, keepdim=True) / LARGEST).clamp(min=2.0 ** -126)
    y = (x.abs() * (1 / scale)).clamp(max=LARGEST)
    small = y < 2.0 ** -6
    bits = torch.where(small, y + 2.0 ** -6, y).view(torch.int32).long()
    code = ((bits + (r << 4) + 8) >> 20) - torch.where(small, 968, 960)
    return code.clamp(max=126), scale


def as_e4m3(code):
    return code.to(torch.uint8).view(torch.float8_e4m3fn)


def adamw_step(st):
    case = st["case"]
    dtype, g = TYPES[case["param"]], st["g"].float()
    p = st["master"] if case["master"] else st["p"].float()
    out = {}
    if case["clip"]:
        total = g.double().square().sum().sqrt().float()
        out["norm"] = total
        g = g * torch.clamp(case["clip"] / (total + 1e-6), max=1.0)
    ids, eight = st["ids"], case["bits"] == 8
    p, g = p.view(-1, BLOCK), g.view(-1, BLOCK)
    if eight or (dtype is torch.bfloat16 and not case["master"]):
        r = random_bits(st)
    m, v = st["m"].float().view(-1, BLOCK), st["v"].float().view(-1, BLOCK)
    if eight:
        m, v = m * st["scales"][:, :1], (v * st["scales"][:, 1:]).square()
    t = (st["step"] + 1).double()
    c1 = (LR / (1 - BETA1 ** t)).float()[ids].view(-1, 1)
    c2 = (1 / (1 - BETA2 ** t).sqrt()).float()[ids].view(-1, 1)
    m = m + (1 - BETA1) * (g - m)
    v = BETA2 * v + (1 - BETA2) * g * g
    u = v.sqrt()
    p = p * (1 - LR * DECAY) - c1 * (m / (u * c2 + ADAM_EPS))
    st["step"] += 1
    if case["master"]:
        st["master"].copy_(p.view(-1))
        st["p"].copy_(p.view(-1).to(dtype))
        out["master"] = st["master"]
    elif dtype is torch.bfloat16:
        st["p"].copy_(((p.view(torch.int32).long() + (r & 0xFFFF)) >> 16 << 16).to(torch.int32).view(torch.float32).view(-1).to(dtype))
    else:
        st["p"].copy_(p.view(-1))
    if eight:
        code, scale = to_8_bits(m, r & 0xFFFF)
        st["m"].copy_(as_e4m3(code + 128 * (m < 0)).view(-1))
        code, scale2 = to_8_bits(u, r >> 16)
        st["v"].copy_(as_e4m3(torch.where(u > 0, code.clamp(min=1), code)).view(-1))
        st["scales"].copy_(torch.cat([scale, scale2], 1))
    else:
        st["m"].copy_(m.view(-1))
        st["v"].copy_(v.view(-1))
    return out


def updated(st, out):
    out.update(p=st["p"], m=st["m"], v=st["v"], step=st["step"])
    if "scales" in st:
        out["scales"] = st["scales"]
    return out


def run(state):
    case = state["case"]
    if case["kind"] == "adamw":
        if not own:
            return updated(state, adamw_step(state))
        opt, out = state["opt"], {}
        opt.step()
        if case["clip"]:
            out["norm"] = opt.grad_norm
        if case["master"]:
            out["master"] = state["master"]
        return updated(state, out)
    if not own:
        return norm_forward(state) if case["kind"] == "fwd" else norm_backward(state)
    g = state["graph"]
    if case["kind"] == "fwd":
        Y, stats = g.dg_group_norm_fwd(state["X"], case["groups"], state["weight"], state["bias"], EPS, state["act"], Y=state["Y"])
        return {"Y": Y, "stats": stats}
    dX, dweight, dbias = g.dg_group_norm_bwd(state["dY"], state["X"], state["stats"], case["groups"], state["weight"],
                                             state["bias"], state["act"], dX=state["dX"])
    return {"dX": dX, "dweight": dweight, "dbias": dbias}


# ---- in 64 bits ------------------------------------------------------------------------------

def exact_norm(case, st):
    """Graph by graph, group by group of columns, in float64."""
    F, G = case["F"], case["groups"]
    cut, w, b = st["bounds"].tolist(), st["weight"].double(), st["bias"].double()
    forward = case["kind"] == "fwd"
    result = st["Y" if forward else "dX"].double()
    stats = torch.zeros((len(cut) - 1, G, 2), dtype=torch.float64, device=w.device)
    stats[..., 1] = 1 / math.sqrt(EPS)
    dw, db = torch.zeros_like(w), torch.zeros_like(w)
    for i, (lo, hi) in enumerate(zip(cut[:-1], cut[1:])):
        if lo == hi:
            continue
        x = st["X"][lo:hi].double().view(hi - lo, G, F // G)
        if forward:
            mean = x.mean((0, 2), keepdim=True)
            rstd = 1 / torch.sqrt(((x - mean) ** 2).mean((0, 2), keepdim=True) + EPS)
            stats[i] = torch.stack([mean.view(-1), rstd.view(-1)], 1)
        else:
            mean, rstd = (st["stats"][i, :, k].double().view(1, G, 1) for k in (0, 1))
        hat = (x - mean) * rstd
        z = hat * w.view(1, G, -1) + b.view(1, G, -1)
        if forward:
            y = z.clamp(min=0) if case["act"] == "relu" else z / (1 + torch.exp(-z)) if case["act"] == "silu" else z
            result[lo:hi] = y.view(hi - lo, F)
            continue
        dz = st["dY"][lo:hi].double().view_as(x)
        if case["act"] == "relu":
            dz = dz * (z > 0)
        elif case["act"] == "silu":
            e = torch.exp(-z)
            dz = dz * (1 / (1 + e) + z * e / (1 + e) ** 2)
        db += dz.sum(0).view(-1)
        dw += (dz * hat).sum(0).view(-1)
        q = dz * w.view(1, G, -1)
        result[lo:hi] = (rstd * (q - q.mean((0, 2), keepdim=True) - hat * (q * hat).mean((0, 2), keepdim=True))).view(hi - lo, F)
    return {"Y": result, "stats": stats} if forward else {"dX": result, "dweight": dw, "dbias": db}


def hash32(v):
    for shift, factor in ((16, 0x7FEB352D), (15, 0x846CA68B)):
        v = ((v ^ (v >> shift)) * factor) % 2 ** 32
    return v ^ (v >> 16)


def rounded_8(x, r):
    """(values, scales) of numbers in blocks of 256: the e4m3 numbers next to |x| / scale are r and its distance apart."""
    rows = lambda t: torch.nn.functional.pad(t.double(), (0, -t.numel() % BLOCK)).view(-1, BLOCK)  # noqa: E731
    y, r = rows(x).abs(), rows(r)
    scale = (y.amax(1) / LARGEST).clamp(min=2.0 ** -126)
    y = (y / scale.view(-1, 1)).clamp(max=LARGEST)
    unit = torch.exp2(torch.frexp(y)[1].double() - 4).clamp(min=2.0 ** -9)
    value = (torch.floor(y / unit + (r * 16 + 8) / 2 ** 20) * unit).clamp(max=LARGEST)
    return value.view(-1)[:x.numel()], scale


def exact_adamw(case, st):
    """Parameter by parameter in float64, from the formulas and the rounding rule."""
    count = numbers(case)
    bf16 = case["param"] == "bf16"
    g_all = st["g"].double()
    out = {"p": st["p"].double(), "m": st["m"].to(torch.float32).double(), "v": st["v"].to(torch.float32).double(), "step": None}
    factor = 1.0
    if case["clip"]:
        out["norm"] = torch.linalg.vector_norm(g_all)
        factor = min(1.0, case["clip"] / (float(out["norm"]) + 1e-6))
    if case["master"]:
        out["master"] = st["master"].double()
    if case["bits"] == 8:
        out["scales"] = st["scales"].double()
    at = 0
    for i, c in enumerate(count):
        blocks = (c + BLOCK - 1) // BLOCK
        s = slice(at, at + c)
        g = g_all[s] * factor
        p = (st["master"] if case["master"] else st["p"])[s].double()
        m, v = out["m"][s], out["v"][s]
        if case["bits"] == 8:
            scale = st["scales"][at // BLOCK:at // BLOCK + blocks].double().repeat_interleave(BLOCK, 0)[:c]
            m, v = m * scale[:, 0], (v * scale[:, 1]) ** 2
        t = int(st["step"][i]) + 1
        m = BETA1 * m + (1 - BETA1) * g
        v = BETA2 * v + (1 - BETA2) * g ** 2
        p = p - LR * DECAY * p - LR * (m / (1 - BETA1 ** t)) / (torch.sqrt(v / (1 - BETA2 ** t)) + ADAM_EPS)
        seed = st["seed"]
        key = hash32(hash32((hash32(hash32((seed % 2 ** 32 + 0x9E3779B9) % 2 ** 32) ^ (seed >> 32) % 2 ** 32) + t - 1) % 2 ** 32) ^ i)
        r = hash32((torch.arange(c, device=p.device) + hash32(key)) % 2 ** 32)
        if case["master"]:
            out["master"][s] = p
        if bf16 and not case["master"]:
            unit = torch.exp2(torch.frexp(p)[1].double() - 8).clamp(min=2.0 ** -133)
            p = p.sign() * torch.floor(p.abs() / unit + (r % 2 ** 16).double() / 2 ** 16) * unit
        out["p"][s] = p
        if case["bits"] != 8:
            out["m"][s], out["v"][s] = m, v
        else:
            u, part = torch.sqrt(v), out["scales"][at // BLOCK:at // BLOCK + blocks]
            value, part[:, 0] = rounded_8(m, r % 2 ** 16)
            out["m"][s] = value * m.sign()
            value, part[:, 1] = rounded_8(u, r >> 16)
            out["v"][s] = torch.where(u > 0, value.clamp(min=2.0 ** -9), value)
        at += blocks * BLOCK
    return out


def exact(case, seed):
    st = prepare(case, seed)
    return exact_adamw(case, st) if case["kind"] == "adamw" else exact_norm(case, st)
