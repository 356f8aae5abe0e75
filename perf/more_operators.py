"""What a second set of the training step's operators is measured on: cases over their real range, inputs, and each operator in
plain torch operations (32 bits inside, one rounding at the end) and in 64 bits.

Three operators, each in the directions that a training program calls: a step of hidden matrices by their orthogonalised momentum
(`muon`), layer norm forward and backward with the gradients of weight and bias (`layer_norm`), and the embedding lookup
with its gradient by sorted tokens (`embed`).  `own` selects the framework's kernels (True) or the plain forms (False); both take
the same state.
"""
import math
import random

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2, "none": 0}
QUINTIC = (3.4445, -4.7750, 2.0315)       # the published odd polynomial that drives singular values towards one
ITERATIONS = 5
BETA, MUON_EPS = 0.95, 1e-7
LN_EPS = 1e-5


def _groups(case):
    """[(count, rows, columns)] of a list of matrices: "12x768x768,..."."""
    return [tuple(int(n) for n in g.split("x")) for g in case["groups"].split(",")]


def _vit_b16():
    """ViT-B/16's hidden matrices as [out, in]: joint query-key-value, output, and the two of the multi-layer perceptron."""
    d = 768
    return ",".join("12x%dx%d" % s for s in ((3 * d, d), (d, d), (4 * d, d), (d, 4 * d)))


# ---- the cases -------------------------------------------------------------------------------------------

def _muon(name, **kw):
    c = {"op": "muon", "groups": "1x1x1", "workers": 1, "param": "f32", "grad": "f32", "copy": "none", "products": 3, "nesterov": True,
         "lr": 0.02, "decay": 0.01}
    c.update(kw)
    return dict(c, name=name) if name else c


def _layer_norm(name, **kw):
    c = {"op": "layer_norm", "pass": "forward", "rows": 1, "width": 1, "type": "bf16", "weight": "f32", "pad": 0}
    c.update(kw)
    return dict(c, name=name) if name else c


def _embed(name, **kw):
    c = {"op": "embed", "pass": "forward", "rows": 1, "vocab": 1, "width": 1, "table": "bf16", "out": "bf16", "scale": 1.0, "absent": 0.0,
         "accumulate": False}
    c.update(kw)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the hidden matrices of a toy next-token model, four replicas: nothing but latency
        _muon("muon 4x 128x128 bf16", groups="1x128x128", workers=4, param="bf16", grad="bf16", products=1),
        # a model trained in bf16 throughout: ViT-B/16's 48 hidden matrices
        _muon("muon vit_b16 bf16", groups=_vit_b16(), param="bf16", grad="bf16", products=1),
        # the same with fp32 parameters, whose steps have to be right to fp32: three products each, bf16 working copies
        _muon("muon vit_b16 f32", groups=_vit_b16(), grad="bf16", copy="bf16"),
        # odd shapes, tall and flat ones, two workers
        _muon("muon 2x ragged f32", groups="3x200x1001,2x1537x77,1x1x640,2x333x333,1x1023x2047", workers=2, grad="f16", nesterov=False),
        # one position of each of eight sequences: latency
        _layer_norm("layer_norm 8x768", rows=8, width=768),
        # 64 images of 196 patches through ViT-B/16
        _layer_norm("layer_norm 12544x768", rows=12544, width=768),
        # the same backwards
        _layer_norm("layer_norm 12544x768 grad", rows=12544, width=768, **{"pass": "gradient"}),
        # odd width in fp32, columns of a wider buffer, backwards
        _layer_norm("layer_norm 4099x5003 grad f32", rows=4099, width=5003, type="f32", pad=29, **{"pass": "gradient"}),
        # serving: one token of each of eight sequences
        _embed("embed 8x1024", rows=8, vocab=32768, width=1024),
        # a toy model's batch, backwards: 64 sequences of 32 tokens
        _embed("embed 2048x128 grad", rows=2048, vocab=1000, width=128, **{"pass": "gradient"}),
        # a language model's batch: odd vocabulary, fp32 table read into bf16, padding
        _embed("embed 65536x1024 f32 table", rows=65536, vocab=50001, width=1024, table="f32", scale=32.0, absent=0.1),
        # the same backwards, the gradient in fp32 written whole
        _embed("embed 65536x1024 grad f32", rows=65536, vocab=50001, width=1024, table="f32", scale=32.0, absent=0.1, **{"pass": "gradient"}),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _muon_flops(case):
    total = 0.0
    for count, r, c in _groups(case):
        m, n = min(r, c), max(r, c)
        total += count * case["workers"] * ITERATIONS * (3.0 * m * m * n + m * m * m)
    return total


def draw(rng):
    op = rng.choice(["muon", "layer_norm", "embed"])
    if op == "muon":
        param = rng.choice(["f32", "f32", "bf16", "f16"])
        kw = {"param": param, "grad": rng.choice(["f32", "bf16", "f16"]), "copy": rng.choice(["none", "bf16", "f16"]) if param == "f32" else "none",
              "products": 3 if param == "f32" else 1, "nesterov": rng.random() < 0.7, "lr": rng.choice([0.02, 0.002]),
              "decay": rng.choice([0.0, 0.1]), "workers": rng.choice([1, 1, 2, 4])}
        while True:
            groups = [(rng.choice([1, 1, 2, 7]), _log_int(rng, 1, 4096), _log_int(rng, 1, 4096)) for _ in range(rng.choice([1, 2, 4]))]
            case = _muon(None, groups=",".join("%dx%dx%d" % g for g in groups), **kw)
            if _muon_flops(case) < 1e12 and len({g[1:] for g in groups}) == len(groups):
                return case
    if op == "layer_norm":
        width = _log_int(rng, 8, 16384)
        return _layer_norm(None, rows=_log_int(rng, 1, max(1, min(65536, (1 << 26) // width))), width=width, type=rng.choice(["f32", "bf16", "f16"]),
                           weight=rng.choice(["f32", "bf16", "f16"]), pad=rng.choice([0, 0, 0, 8, 29]),
                           **{"pass": rng.choice(["forward", "gradient"])})
    width = _log_int(rng, 1, 4096)
    vocab = _log_int(rng, 2, min(150000, (1 << 27) // width))
    return _embed(None, rows=_log_int(rng, 1, min(131072, (1 << 27) // width)), vocab=vocab, width=width, table=rng.choice(["f32", "bf16", "f16"]),
                  out=rng.choice(["f32", "bf16", "f16"]), scale=rng.choice([1.0, 11.5]), absent=rng.choice([0.0, 0.2]),
                  accumulate=rng.random() < 0.5, **{"pass": rng.choice(["forward", "gradient", "gradient"])})


# ---- inputs ----------------------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _update_scale(r, c):
    return math.sqrt(max(1.0, r / c))


def _prepare_muon(case, seed):
    gen, K = _generator(seed), case["workers"]
    s = {"case": case, "param": [], "grad": [], "momentum": [], "copy": []}
    for count, r, c in _groups(case):
        def normal():
            return torch.randn(K, count, r, c, device=DEV, generator=gen)

        # gradients are a few directions (activations times errors) over noise; the momentum has seen more of the directions
        few = min(8, r, c)
        left = torch.randn(K, count, r, few, device=DEV, generator=gen)
        right = torch.randn(K, count, few, c, device=DEV, generator=gen)
        low = (left @ right).mul_(0.5 / math.sqrt(few))
        size = 2.0 ** -9
        s["param"].append(normal().mul_(0.02).to(TYPES[case["param"]]))
        s["grad"].append((low + normal()).mul_(size).to(TYPES[case["grad"]]))
        s["momentum"].append((low + normal().mul_(0.3)).mul_(size))
        if case["copy"] != "none":
            s["copy"].append(s["param"][-1].to(TYPES[case["copy"]]))
    if own:
        from paper_2310_14423_b200 import binding as B

        def views(name):
            return [m for k in range(K) for g in s[name] for m in g[k]] if s[name] else None

        params = views("param")
        s["workspace"] = torch.empty(B.qsr_muon_workspace_bytes([p.shape for p in params], K, case["products"]), dtype=torch.uint8, device=DEV)
        s["list"] = B.MuonList(params, views("grad"), views("momentum"), copies=views("copy"), update_scale=[_update_scale(*p.shape) for p in params],
                               workers=K, beta=BETA, nesterov=case["nesterov"], weight_decay=case["decay"], eps=MUON_EPS,
                               iterations=ITERATIONS, products=case["products"], workspace=s["workspace"],
                               stream=torch.cuda.current_stream().cuda_stream)
    return s


def _matrix(rows, width, pad, kind, value=None):
    """A [rows, width] matrix, the first columns of rows that are `pad` longer."""
    x = torch.zeros(rows, width + pad, device=DEV, dtype=TYPES[kind])[:, :width]
    return x if value is None else x.copy_(value)


def _prepare_layer_norm(case, seed):
    gen, R, N = _generator(seed), case["rows"], case["width"]
    # activations: a mean of their own in each row, and a few channels that are far larger than the others
    channel = torch.where(torch.rand(N, device=DEV, generator=gen) < 0.01, 20.0, 1.0)
    x = torch.randn(R, N, device=DEV, generator=gen).mul_(channel).add_(torch.randn(R, 1, device=DEV, generator=gen).mul_(0.5))
    s = {"case": case, "x": _matrix(R, N, case["pad"], case["type"], x)}
    del x
    s["weight"] = torch.randn(N, device=DEV, generator=gen).mul_(0.2).add_(1.0).to(TYPES[case["weight"]])
    s["bias"] = torch.randn(N, device=DEV, generator=gen).mul_(0.1).to(TYPES[case["weight"]])
    if case["pass"] == "forward":
        s["y"] = _matrix(R, N, case["pad"], case["type"])
        s["mean"], s["rstd"] = torch.empty(R, device=DEV), torch.empty(R, device=DEV)
    else:
        s["d_y"] = _matrix(R, N, case["pad"], case["type"], torch.randn(R, N, device=DEV, generator=gen))
        s["d_x"] = _matrix(R, N, case["pad"], case["type"])
        s["d_weight"], s["d_bias"] = torch.empty_like(s["weight"]), torch.empty_like(s["bias"])
        s["mean"], s["rstd"] = _row_statistics(s["x"])          # what the forward pass left
    if own:
        from paper_2310_14423_b200 import binding as B
        s["B"], s["stream"] = B, torch.cuda.current_stream().cuda_stream
        if case["pass"] == "gradient":
            s["workspace"] = torch.empty(B.qsr_layer_norm_workspace_bytes(R, N), dtype=torch.uint8, device=DEV)
    return s


def _prepare_embed(case, seed):
    gen, R, V, N = _generator(seed), case["rows"], case["vocab"], case["width"]
    # token frequencies fall off as one over the rank, frequent tokens first, as vocabularies are built
    rank = torch.exp(torch.rand(R, device=DEV, generator=gen, dtype=torch.float64) * math.log(V + 1.0))
    tokens = (rank - 1.0).long().clamp_(0, V - 1)
    tokens = torch.where(torch.rand(R, device=DEV, generator=gen) < case["absent"], torch.full_like(tokens, -1), tokens)
    s = {"case": case, "tokens": tokens}
    if case["pass"] == "forward":
        s["table"] = torch.randn(V, N, device=DEV, generator=gen).mul_(0.02).to(TYPES[case["table"]])
        s["out"] = torch.empty(R, N, device=DEV, dtype=TYPES[case["out"]])
    else:
        s["d_out"] = torch.randn(R, N, device=DEV, generator=gen).mul_(2.0 ** -9).to(TYPES[case["out"]])
        # a tied head has left its gradient there where it is added to
        s["d_table"] = torch.randn(V, N, device=DEV, generator=gen).mul_(2.0 ** -9).to(TYPES[case["table"]])
    if own:
        from paper_2310_14423_b200 import binding as B
        s["B"], s["stream"] = B, torch.cuda.current_stream().cuda_stream
        if case["pass"] == "gradient":
            s["workspace"] = torch.empty(B.qsr_embed_workspace_bytes(R, V, N), dtype=torch.uint8, device=DEV)
    return s


def prepare(case, seed):
    return {"muon": _prepare_muon, "layer_norm": _prepare_layer_norm, "embed": _prepare_embed}[case["op"]](case, seed)


# ---- one pass --------------------------------------------------------------------------------------------

def run(state):
    return {"muon": _run_muon, "layer_norm": _run_layer_norm, "embed": _run_embed}[state["case"]["op"]](state)


def _orthogonal(u):
    """Newton-Schulz iterations over a batch of matrices in fp32."""
    a, b, c = QUINTIC
    x = u / (u.square().sum((-2, -1), keepdim=True).sqrt() + MUON_EPS)
    tall = x.shape[-2] > x.shape[-1]
    x = x.mT if tall else x
    for _ in range(ITERATIONS):
        gram = x @ x.mT
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.mT if tall else x


def _run_muon(s):
    c = s["case"]
    if own:
        s["list"].qsr_muon_step(c["lr"])
    else:
        for i, (param, grad, m) in enumerate(zip(s["param"], s["grad"], s["momentum"])):
            g = grad.float()
            m.add_((g - m) * (1.0 - BETA))
            x = _orthogonal(g + BETA * (m - g) if c["nesterov"] else m)
            theta = param.float()
            theta = theta - (c["lr"] * c["decay"] * theta + c["lr"] * _update_scale(*param.shape[-2:]) * x)
            param.copy_(theta)
            if s["copy"]:
                s["copy"][i].copy_(theta)
    return {k: s[k] for k in ("param", "momentum", "copy")}


def _row_statistics(x):
    """Mean and reciprocal standard deviation of each row in fp32."""
    v, mean = torch.var_mean(x.double(), 1, correction=0)
    return mean.float(), (v + LN_EPS).rsqrt().float()


def _run_layer_norm(s):
    c = s["case"]
    if c["pass"] == "forward":
        if own:
            s["B"].qsr_layer_norm(s["x"], s["y"], weight=s["weight"], bias=s["bias"], mean=s["mean"], rstd=s["rstd"], eps=LN_EPS, stream=s["stream"])
        else:
            x = s["x"].float()
            mean = x.mean(1, keepdim=True)
            centred = x - mean
            rstd = (centred.square().mean(1, keepdim=True) + LN_EPS).rsqrt()
            s["y"].copy_(centred * rstd * s["weight"].float() + s["bias"].float())
            s["mean"].copy_(mean[:, 0])
            s["rstd"].copy_(rstd[:, 0])
        return {k: s[k] for k in ("y", "mean", "rstd")}
    if own:
        s["B"].qsr_layer_norm_grad(s["x"], s["d_y"], s["mean"], s["rstd"], d_x=s["d_x"], weight=s["weight"], d_weight=s["d_weight"],
                                   d_bias=s["d_bias"], workspace=s["workspace"], stream=s["stream"])
    else:
        dy = s["d_y"].float()
        hat = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
        s["d_weight"].copy_((dy * hat).sum(0))
        s["d_bias"].copy_(dy.sum(0))
        d = dy * s["weight"].float()
        s["d_x"].copy_((d - d.mean(1, keepdim=True) - hat * (d * hat).mean(1, keepdim=True)) * s["rstd"][:, None])
    return {k: s[k] for k in ("d_x", "d_weight", "d_bias")}


def _run_embed(s):
    c, tokens = s["case"], s["tokens"]
    if c["pass"] == "forward":
        if own:
            s["B"].qsr_embed(s["table"], tokens, s["out"], scale=c["scale"], stream=s["stream"])
        else:
            rows = s["table"][tokens.clamp_min(0)].float() * c["scale"]
            s["out"].copy_(torch.where((tokens >= 0)[:, None], rows, 0.0))
        return s["out"]
    if own:
        s["B"].qsr_embed_grad(s["d_out"], tokens, s["d_table"], scale=c["scale"], accumulate=c["accumulate"], workspace=s["workspace"],
                              stream=s["stream"])
    else:
        d = torch.where((tokens >= 0)[:, None], s["d_out"].float(), 0.0)
        total = torch.zeros(s["d_table"].shape, device=DEV).index_add_(0, tokens.clamp_min(0), d).mul_(c["scale"])
        s["d_table"].copy_(total + s["d_table"].float() if c["accumulate"] else total)
    return s["d_table"]


# ---- what a pass cannot do without -----------------------------------------------------------------------

def work(case):
    if case["op"] == "muon":
        n = sum(count * r * c for count, r, c in _groups(case)) * case["workers"]
        return {"bytes": n * (2 * BYTES[case["param"]] + BYTES[case["copy"]] + BYTES[case["grad"]] + 8.0), "flops": _muon_flops(case)}
    if case["op"] == "layer_norm":
        n, b = case["rows"] * case["width"], BYTES[case["type"]]
        back = case["pass"] == "gradient"
        return {"bytes": n * b * (3.0 if back else 2.0) + 8.0 * case["rows"] + (3 if back else 2) * case["width"] * BYTES[case["weight"]],
                "flops": n * (12.0 if back else 7.0)}
    n, present = case["rows"] * case["width"], min(case["rows"], case["vocab"]) * case["width"]
    table, out = BYTES[case["table"]], BYTES[case["out"]]
    if case["pass"] == "forward":
        return {"bytes": 8.0 * case["rows"] + n * out + present * table, "flops": float(n)}
    written = 2 * present if case["accumulate"] else case["vocab"] * case["width"]
    return {"bytes": 8.0 * case["rows"] + n * out + written * table, "flops": 2.0 * n}


# ---- the definitions in 64 bits --------------------------------------------------------------------------

def exact(case, seed):
    global own
    before, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = before
    return {"muon": _exact_muon, "layer_norm": _exact_layer_norm, "embed": _exact_embed}[case["op"]](s)


def _exact_muon(s):
    c = s["case"]
    out = {"param": [], "momentum": [], "copy": []}
    for p, g, m in zip(s["param"], s["grad"], s["momentum"]):
        r, n = p.shape[-2:]
        mean = BETA * m.double() + (1.0 - BETA) * g.double()
        u = ((1.0 - BETA) * g.double() + BETA * mean if c["nesterov"] else mean).flatten(0, 1)
        q = u / (torch.linalg.matrix_norm(u, keepdim=True) + MUON_EPS)
        unit = torch.eye(min(r, n), device=DEV, dtype=torch.float64)
        for _ in range(ITERATIONS):       # on the shorter side; the same polynomial of the singular values from either
            g2 = torch.matmul(q, q.mT) if r <= n else torch.matmul(q.mT, q)
            factor = QUINTIC[0] * unit + torch.matmul(g2, QUINTIC[1] * unit + QUINTIC[2] * g2)
            q = torch.matmul(factor, q) if r <= n else torch.matmul(q, factor)
        theta = p.double() * (1.0 - c["lr"] * c["decay"]) - c["lr"] * max(1.0, r / n) ** 0.5 * q.view(p.shape)
        out["param"].append(theta)
        out["momentum"].append(mean)
        if s["copy"]:
            out["copy"].append(theta)
    return out


def _exact_layer_norm(s):
    x = s["x"].double()
    w, b = s["weight"].double(), s["bias"].double()
    if s["case"]["pass"] == "forward":
        mean = x.sum(1) / x.shape[1]
        rstd = 1.0 / torch.sqrt(((x - mean[:, None]) ** 2).sum(1) / x.shape[1] + LN_EPS)
        return {"y": (x - mean[:, None]) * rstd[:, None] * w + b, "mean": mean, "rstd": rstd}
    mean, rstd, dy = s["mean"].double(), s["rstd"].double(), s["d_y"].double()
    hat = (x - mean[:, None]) * rstd[:, None]
    d, n = dy * w, x.shape[1]
    along = torch.einsum("rn,rn->r", d, hat) / n
    return {"d_x": rstd[:, None] * (d - (d.sum(1) / n)[:, None] - along[:, None] * hat), "d_weight": torch.einsum("rn,rn->n", dy, hat),
            "d_bias": torch.einsum("rn->n", dy)}


def _exact_embed(s):
    c, t = s["case"], s["tokens"]
    some = t >= 0
    if c["pass"] == "forward":
        out = torch.zeros(t.numel(), s["table"].shape[1], device=DEV, dtype=torch.float64)
        out[some] = s["table"].index_select(0, t[some]).double() * c["scale"]
        return out
    total = torch.zeros(s["d_table"].shape, device=DEV, dtype=torch.float64)
    total.index_put_((t[some],), s["d_out"][some].double(), accumulate=True)
    return s["d_table"].double() * float(c["accumulate"]) + c["scale"] * total
