"""What the operators of the training step are measured on: cases over their real range, inputs, and each operator in
plain torch operations (32 bits inside, one rounding at the end) and in 64 bits.

Three operators: the log probabilities of given tokens with entropy, top alternatives and gradient (`logprobs`), an AdamW
step over a list of tensors with states in 32 or 8 bits (`adamw`), and the replica mean that ends a round over such lists
(`sync`).  `own` selects the framework's kernels (True) or the plain forms (False); both take the same state.
"""
import math
import random

import torch

own = False

DEV = "cuda"
BLOCK = 256                     # elements that share one scale where optimizer states are held in 8 bits
E4M3_MAX = 448.0
E4M3_MIN = 2.0 ** -9            # smallest positive code
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2, "none": 0, "e4m3": 1}


# ---- tensor lists ----------------------------------------------------------------------------------------

def _vit_b16():
    """Sizes and weight-decay factors of ViT-B/16's trained tensors (vectors are exempt from weight decay)."""
    d, hidden, classes, patch = 768, 3072, 1000, 768
    sizes = [d * patch, d]
    for _ in range(12):
        sizes += [d, d, 3 * d * d, 3 * d, d * d, d, d, d, hidden * d, hidden, hidden * d, d]
    return sizes + [d, d, classes * d, classes]


def _resnet152():
    """Sizes of ResNet-152's convolution, normalization and classifier tensors."""
    sizes, inside = [64 * 3 * 49, 64, 64], 64
    for planes, blocks in ((64, 3), (128, 8), (256, 36), (512, 3)):
        for b in range(blocks):
            out = 4 * planes
            sizes += [planes * inside, planes, planes, planes * planes * 9, planes, planes, out * planes, out, out]
            if b == 0:
                sizes += [out * inside, out, out]
            inside = out
    return sizes + [1000 * 2048, 1000]


def _ragged(tensors, elements, split):
    """`tensors` sizes of all magnitudes, odd ones among them, that add up to about `elements`."""
    r = random.Random(split)
    weight = [r.lognormvariate(0.0, 2.0) for _ in range(tensors)]
    return [max(1, int(elements * w / sum(weight))) for w in weight]


def _sizes(case):
    if case["list"] == "vit_b16":
        return _vit_b16()
    if case["list"] == "resnet152":
        return _resnet152()
    return _ragged(case["tensors"], case["elements"], case["split"])


def _layout(case):
    """(sizes, offsets, extents, row length) of a worker's tensors in one flat row: each tensor starts on a multiple of
    256 elements, as separately allocated tensors do, or directly behind the one before it ("packed")."""
    sizes, offsets, at = _sizes(case), [], 0
    for n in sizes:
        offsets.append(at)
        at += n if case["packed"] else -(-n // BLOCK) * BLOCK
    extents = [b - a for a, b in zip(offsets, offsets[1:] + [at])]
    return sizes, offsets, extents, at


# ---- the cases -------------------------------------------------------------------------------------------

def _adamw(name, **kw):
    c = {"op": "adamw", "list": "ragged", "tensors": 0, "elements": 0, "split": 0, "packed": False, "workers": 1,
         "param": "f32", "grad": "f32", "copy": "none", "states": "f32", "clip": 0.0, "step": 1000, "lr": 8e-4, "decay": 0.05}
    c.update(kw)
    return dict(c, name=name) if name else c


def _sync(name, **kw):
    c = {"op": "sync", "list": "ragged", "tensors": 0, "elements": 0, "split": 0, "packed": False, "workers": 4,
         "param": "f32", "copy": "none", "states": "f32", "mode": "keep"}
    c.update(kw)
    return dict(c, name=name) if name else c


def _logprobs(name, **kw):
    c = {"op": "logprobs", "rows": 1, "vocab": 2, "type": "bf16", "top": 0, "temperature": 1.0, "gradient": "none",
         "masked": 0.0, "unscored": 0.0}
    c.update(kw)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a toy model's step (65,536 parameters in four tensors): nothing but latency
        _adamw("adamw 65536 f32", tensors=4, elements=65536, split=1),
        # ordinary mixed-precision training of ViT-B/16: fp32 parameters, bf16 gradients and working copy, fp32 states
        _adamw("adamw vit_b16 f32 states", list="vit_b16", grad="bf16", copy="bf16"),
        # the same with the states in 8 bits, as on a card that several replicas share
        _adamw("adamw vit_b16 e4m3 states", list="vit_b16", grad="bf16", copy="bf16", states="e4m3"),
        # many small tensors, everything that can be narrow narrow
        _adamw("adamw resnet152 bf16 e4m3", list="resnet152", param="bf16", grad="bf16", states="e4m3", lr=1e-3),
        # odd sizes directly behind one another (views of one buffer), fp16 gradients, each of two workers clipped
        _adamw("adamw packed f16 clipped", tensors=61, elements=4_000_037, split=5, packed=True, workers=2, grad="f16", clip=1.0, step=3),
        # serving: eight sequences, one position each, a large vocabulary, twenty alternatives
        _logprobs("logprobs 8x131072 top20", rows=8, vocab=131072, top=20, temperature=0.7),
        # a classifier's head (1000 classes) in fp32 with the loss's gradient
        _logprobs("logprobs 4096x1000 fused f32", rows=4096, vocab=1000, type="f32", gradient="fused"),
        # scoring, then the gradient by a second call (policy gradients need the log probability first); odd vocabulary, a
        # quarter of it masked, prompts without a score, entropy's gradient too
        _logprobs("logprobs 2048x50001 two calls", rows=2048, vocab=50001, top=5, gradient="separate", masked=0.25, unscored=0.3),
        # a language model's training step: loss and gradient over 8192 positions
        _logprobs("logprobs 8192x32768 fused", rows=8192, vocab=32768, gradient="fused", unscored=0.05),
        # round end of a toy run: four replicas
        _sync("sync 4x65536 f32", tensors=4, elements=65536, split=1, workers=4),
        # odd sizes, bf16 parameters, three replicas, the fp32 states averaged too
        _sync("sync 3 packed bf16 average", tensors=37, elements=5_000_011, split=9, packed=True, workers=3, param="bf16", mode="average"),
        # round end of eight ViT-B/16 replicas with working copies, 8-bit states averaged
        _sync("sync 8 vit_b16 e4m3 average", list="vit_b16", workers=8, copy="bf16", states="e4m3", mode="average"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["adamw", "logprobs", "sync"])
    if op == "logprobs":
        vocab = _log_int(rng, 20, 150000)
        return _logprobs(None, rows=_log_int(rng, 1, min(16384, (1 << 28) // vocab)), vocab=vocab, type=rng.choice(["f32", "bf16", "f16"]),
                         top=rng.choice([0, 0, 1, 5, 20]), temperature=rng.choice([1.0, 1.0, 0.7, 1.3]),
                         gradient=rng.choice(["none", "fused", "separate"]), masked=rng.choice([0.0, 0.25, 0.9]),
                         unscored=rng.choice([0.0, 0.3]))
    tensors, elements = _log_int(rng, 1, 400), _log_int(rng, 1000, 80_000_000 if op == "adamw" else 20_000_000)
    states = rng.choice(["f32", "e4m3"])
    packed = states == "f32" and rng.random() < 0.3
    kw = {"tensors": tensors, "elements": elements, "split": rng.randrange(1 << 30), "packed": packed, "states": states,
          "param": rng.choice(["f32", "f32", "bf16", "f16"])}
    kw["copy"] = rng.choice(["none", "bf16", "f16"]) if kw["param"] == "f32" else "none"
    if op == "sync":
        return _sync(None, workers=rng.choice([2, 3, 4, 8, 16]), mode=rng.choice(["keep", "average", "reset"]), **kw)
    # 8-bit states are drawn without clipping: a norm summed in another order may move a value over a code's boundary
    clip = rng.choice([0.0, 1.0]) if states == "f32" else 0.0
    return _adamw(None, grad=rng.choice(["f32", "bf16", "f16"]), clip=clip, step=rng.choice([1, 10, 5000]),
                  lr=rng.choice([8e-4, 8e-3]), **kw)


# ---- inputs ----------------------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _spread(extents, values, total):
    """A value for each tensor, repeated over its extent of a row."""
    return torch.repeat_interleave(values, extents, output_size=total)


def _prepare_list(case, seed):
    sizes, offsets, extents, total = _layout(case)
    K, gen = case["workers"], _generator(seed)
    s = {"case": case, "total": total, "extents": torch.tensor(extents, device=DEV)}
    # vectors (here: small tensors) are exempt from weight decay
    s["decay"] = torch.tensor([0.0 if n < 4096 else 1.0 for n in sizes], device=DEV)
    inside = torch.zeros(total, device=DEV)
    for o, n in zip(offsets, sizes):
        inside[o:o + n] = 1.0

    def normal():
        return torch.randn(K, total, device=DEV, generator=gen).mul_(inside)

    # gradients of one tensor share a magnitude, and different tensors' magnitudes span several decades
    size = _spread(s["extents"], torch.exp2(torch.randn(len(sizes), device=DEV, generator=gen).mul_(3.0).sub_(9.0)), total)
    s["param"] = normal().mul_(0.02).to(TYPES[case["param"]])
    first = case.get("step") == 1
    m = normal().mul_(size).mul_(0.0 if first else 0.3)
    u = normal().abs_().mul_(0.5).add_(0.5).mul_(size).mul_(inside).mul_(0.0 if first else 1.0)
    if case["states"] == "f32":
        s["m"], s["v"] = m, u.square_()
    else:
        s["m"], s["m_scale"] = _to_e4m3(m)
        s["v"], s["v_scale"] = _to_e4m3(u, True)
    del m, u
    if case["op"] == "adamw":
        s["grad"] = normal().mul_(size).to(TYPES[case["grad"]])
    if case["copy"] != "none":
        s["copy"] = s["param"].to(TYPES[case["copy"]])
    if own:
        s["list"] = _own_list(case, s, sizes, offsets)
    return s


def _own_list(case, s, sizes, offsets):
    """The handle a program keeps over its tensors: views of the flat rows, worker by worker."""
    from paper_2310_14423_b200 import binding as B

    def views(name):
        return [row[o:o + n] for row in s[name] for o, n in zip(offsets, sizes)] if name in s else None

    def scales(name):
        return [row[o // BLOCK:-(-(o + n) // BLOCK)] for row in s[name] for o, n in zip(offsets, sizes)] if name in s else None

    K, params = case["workers"], views("param")
    s["workspace"] = torch.empty(B.qsr_list_workspace_bytes([p.numel() for p in params], K), dtype=torch.uint8, device=DEV)
    return B.TensorList(params, views("grad"), views("m"), views("v"), m_scale=scales("m_scale"), v_scale=scales("v_scale"),
                        copies=views("copy"), wd_scale=s["decay"].tolist() * K, workers=K, beta1=0.9, beta2=0.999, eps=1e-8,
                        weight_decay=case.get("decay", 0.0), clip_norm=case.get("clip", 0.0), workspace=s["workspace"],
                        stream=torch.cuda.current_stream().cuda_stream)


def _prepare_logprobs(case, seed):
    gen, R, V = _generator(seed), case["rows"], case["vocab"]
    x = torch.randn(R, V, device=DEV, generator=gen).mul_(2.5)
    # a model that knows something: one token of each row stands out
    y = torch.randint(0, V, (R,), device=DEV, generator=gen)
    x.scatter_add_(1, y[:, None], torch.rand(R, 1, device=DEV, generator=gen) * 14.0)
    if case["masked"] > 0.0:     # a grammar or a list of banned tokens
        x.masked_fill_(torch.rand(R, V, device=DEV, generator=gen) < case["masked"], -math.inf)
    # the scored token is mostly the likely one
    other = torch.randint(0, V, (R,), device=DEV, generator=gen)
    y = torch.where(torch.rand(R, device=DEV, generator=gen) < 0.4, other, y)
    y = torch.where(torch.rand(R, device=DEV, generator=gen) < case["unscored"], torch.full_like(y, -100), y)
    s = {"case": case, "logits": x.to(TYPES[case["type"]]), "tokens": y}
    del x
    s["logprob"], s["entropy"] = torch.empty(R, device=DEV), torch.empty(R, device=DEV)
    k = min(case["top"], V)
    s["top_logprob"] = torch.empty(R, k, device=DEV) if k else None
    s["top_token"] = torch.empty(R, k, device=DEV, dtype=torch.int64) if k else None
    if case["gradient"] != "none":
        s["d_logprob"] = torch.randn(R, device=DEV, generator=gen) if case["gradient"] == "separate" else torch.full((R,), -1.0, device=DEV)
        s["d_entropy"] = torch.full((R,), 0.01, device=DEV) if case["gradient"] == "separate" else None
        s["row_stats"] = torch.empty(R, 2, device=DEV)
        s["d_logits"] = torch.empty_like(s["logits"])
    if own:
        from paper_2310_14423_b200 import binding as B
        s["B"], s["stream"] = B, torch.cuda.current_stream().cuda_stream
    return s


def prepare(case, seed):
    return _prepare_logprobs(case, seed) if case["op"] == "logprobs" else _prepare_list(case, seed)


# ---- one pass --------------------------------------------------------------------------------------------

def run(state):
    return {"adamw": _run_adamw, "sync": _run_sync, "logprobs": _run_logprobs}[state["case"]["op"]](state)


def _held(s):
    return {k: s[k] for k in ("param", "m", "v", "m_scale", "v_scale", "copy") if k in s}


def _to_e4m3(x, floor=False):
    """(codes, scales) of x in blocks of 256: scale = amax / 448 over the block's finite values, codes to nearest even.
    floor: what is positive stays positive."""
    b = x.reshape(-1, BLOCK)
    amax = torch.where(b.isfinite(), b.abs(), 0.0).amax(1, keepdim=True)
    scale = torch.where(amax >= 2.0 ** -100, amax * (1.0 / E4M3_MAX), torch.zeros_like(amax))
    q = b * torch.where(scale > 0, scale.reciprocal(), torch.zeros_like(scale))
    if floor:
        q = torch.where(q > 0, q.clamp_min(E4M3_MIN), q)
    q = q.clamp(-E4M3_MAX, E4M3_MAX)
    return q.to(torch.float8_e4m3fn).view_as(x), scale.view(x.shape[0], -1)


def _from_e4m3(codes, scale):
    return (codes.float().view(-1, BLOCK) * scale.view(-1, 1)).view_as(codes)


def _run_adamw(s):
    c = s["case"]
    if own:
        s["list"].qsr_list_step(c["step"], c["lr"])
        return _held(s)
    n, total = c["step"], s["total"]
    step_size, inv_root = c["lr"] / (1.0 - 0.9 ** n), 1.0 / math.sqrt(1.0 - 0.999 ** n)
    theta, g = s["param"].float(), s["grad"].float()
    if c["clip"] > 0.0:
        norm = g.square().sum(1, keepdim=True).sqrt()
        g = g * (c["clip"] / (norm + 1e-6)).clamp_max(1.0)
    if c["states"] == "f32":
        m, v = s["m"], s["v"]
    else:
        m, v = _from_e4m3(s["m"], s["m_scale"]), _from_e4m3(s["v"], s["v_scale"]).square()
    m = m + 0.1 * (g - m)
    v = v + 0.001 * (g * g - v)
    u = v.sqrt()
    decay = _spread(s["extents"], s["decay"], total) * (c["lr"] * c["decay"])
    theta = theta - (decay * theta + step_size * m / (u * inv_root + 1e-8))
    s["param"].copy_(theta)
    if "copy" in s:
        s["copy"].copy_(theta)
    if c["states"] == "f32":
        s["m"].copy_(m)
        s["v"].copy_(v)
    else:
        for name, x, floor in (("m", m, False), ("v", u, True)):
            codes, scale = _to_e4m3(x, floor)
            s[name].copy_(codes)
            s[name + "_scale"].copy_(scale)
    return _held(s)


def _run_sync(s):
    c = s["case"]
    if own:
        s["list"].qsr_list_sync(c["mode"])
        return _held(s)
    K = c["workers"]
    mean = s["param"].float().sum(0, keepdim=True) / K
    s["param"].copy_(mean.expand_as(s["param"]))
    if "copy" in s:
        s["copy"].copy_(mean.expand_as(s["copy"]))
    if c["mode"] == "reset":
        for name in ("m", "v", "m_scale", "v_scale"):
            if name in s:
                s[name].zero_()
    elif c["mode"] == "average" and c["states"] == "f32":
        for name in ("m", "v"):
            s[name].copy_((s[name].sum(0, keepdim=True) / K).expand_as(s[name]))
    elif c["mode"] == "average":
        m = _from_e4m3(s["m"], s["m_scale"]).sum(0, keepdim=True) / K
        u = (_from_e4m3(s["v"], s["v_scale"]).square().sum(0, keepdim=True) / K).sqrt()
        for name, x, floor in (("m", m, False), ("v", u, True)):
            codes, scale = _to_e4m3(x, floor)
            s[name].copy_(codes.expand_as(s[name]))
            s[name + "_scale"].copy_(scale.expand_as(s[name + "_scale"]))
    return _held(s)


def _run_logprobs(s):
    c = s["case"]
    out = {"logprob": s["logprob"], "entropy": s["entropy"]}
    if c["top"]:
        out |= {"top_logprob": s["top_logprob"], "top_token": s["top_token"]}
    if c["gradient"] != "none":
        out["d_logits"] = s["d_logits"]
    if own:
        B, tau, how = s["B"], 1.0 / c["temperature"], c["gradient"]
        grads = {"d_logprob": s["d_logprob"], "d_entropy": s["d_entropy"], "d_logits": s["d_logits"]} if how != "none" else {}
        B.qsr_token_logprobs(s["logits"], s["tokens"], s["logprob"], entropy=s["entropy"], row_stats=s.get("row_stats"),
                             top_logprob=s["top_logprob"], top_token=s["top_token"], inv_temperature=tau, stream=s["stream"],
                             **(grads if how == "fused" else {}))
        if how == "separate":
            B.qsr_token_logprobs_grad(s["logits"], s["tokens"], s["row_stats"], entropy=s["entropy"], inv_temperature=tau,
                                      stream=s["stream"], **grads)
        return out
    tau, raw, y = 1.0 / c["temperature"], s["logits"], s["tokens"]
    x = raw.float()
    top = x.amax(1, keepdim=True)
    some = top > -math.inf                                    # rows that the mask leaves something of
    z = (x - torch.where(some, top, 0.0)) * tau
    e = z.exp()
    total = e.sum(1, keepdim=True)
    z = z - total.log()                                       # log probabilities (-inf where masked)
    p = e / torch.where(some, total, 1.0)
    plogp = torch.where(p > 0, p * z, 0.0)
    H = -plogp.sum(1, keepdim=True)
    scored = (y >= 0)[:, None]
    at = y.clamp_min(0)[:, None]
    picked = torch.where(some, z.gather(1, at), -math.inf)
    s["logprob"].copy_(torch.where(scored, picked, 0.0)[:, 0])
    s["entropy"].copy_(H[:, 0])
    if c["top"]:
        # one whole number orders value (descending) and index (ascending): no ties are left
        bits = (x + 0.0).view(torch.int32)
        key = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).to(torch.int64) << 32
        key = key + (x.shape[1] - 1 - torch.arange(x.shape[1], device=x.device))
        index = x.shape[1] - 1 - (key.topk(s["top_token"].shape[1], dim=1).values & 0xFFFFFFFF)
        s["top_token"].copy_(index)
        s["top_logprob"].copy_(torch.where(some, z.gather(1, index), -math.inf))
    if c["gradient"] != "none":
        a = torch.where(scored & some, s["d_logprob"][:, None], 0.0)
        d = -a * p
        d.scatter_add_(1, at, a)
        if s["d_entropy"] is not None:
            d = d - s["d_entropy"][:, None] * (plogp + p * H)
        s["d_logits"].copy_(d * tau)
    return out


# ---- what a pass cannot do without -----------------------------------------------------------------------

def work(case):
    if case["op"] == "logprobs":
        R, V, b = case["rows"], case["vocab"], BYTES[case["type"]]
        grad = case["gradient"] != "none"
        k = min(case["top"], V)
        return {"bytes": R * (V * b * (2 if grad else 1) + 16 + 12 * k + (4 if grad else 0)), "flops": R * V * (10.0 if grad else 5.0)}
    n = sum(_sizes(case)) * case["workers"]
    p, q, st = BYTES[case["param"]], BYTES[case["copy"]], BYTES[case["states"]]
    scale = 4.0 / BLOCK if case["states"] == "e4m3" else 0.0
    states = {"keep": 0.0, "average": 4 * (st + scale), "reset": 2 * (st + scale)}[case.get("mode", "average")]
    grad = BYTES[case["grad"]] if case["op"] == "adamw" else 0
    return {"bytes": n * (2 * p + q + grad + states), "flops": n * (25.0 if case["op"] == "adamw" else 3.0)}


# ---- the definitions in 64 bits --------------------------------------------------------------------------

def exact(case, seed):
    global own
    before, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = before
    return {"adamw": _exact_adamw, "sync": _exact_sync, "logprobs": _exact_logprobs}[case["op"]](s)


def _codes64(x, positive):
    """E4M3 codes and scales of 64-bit values by counting in steps of the format: eight steps to a power of two, none
    smaller than 2^-9."""
    b = x.reshape(-1, BLOCK)
    scale = b.abs().amax(1, keepdim=True) / E4M3_MAX
    r = torch.where(scale > 0, b / scale, 0.0)
    _, e = torch.frexp(r)
    unit = torch.exp2((e - 4).clamp_min(-9).double())
    code = torch.round(r / unit) * unit
    if positive:
        code = torch.where((r > 0) & (code == 0), E4M3_MIN, code)
    return code.view_as(x).float().to(torch.float8_e4m3fn), scale.view(x.shape[0], -1)


def _states64(s):
    if s["case"]["states"] == "f32":
        return s["m"].double(), s["v"].double()
    shape = s["m"].shape
    m = s["m"].double().view(-1, BLOCK) * s["m_scale"].double().view(-1, 1)
    u = s["v"].double().view(-1, BLOCK) * s["v_scale"].double().view(-1, 1)
    return m.view(shape), (u * u).view(shape)


def _states_out(out, s, m, v, K):
    if s["case"]["states"] == "f32":
        out["m"], out["v"] = m.expand(K, -1), v.expand(K, -1)
        return out
    for name, x, positive in (("m", m, False), ("v", v.sqrt(), True)):
        codes, scale = _codes64(x, positive)
        out[name], out[name + "_scale"] = codes.expand(K, -1), scale.expand(K, -1)
    return out


def _exact_adamw(s):
    c, K = s["case"], s["case"]["workers"]
    g, n = s["grad"].double(), c["step"]
    if c["clip"] > 0.0:
        g = g * torch.clamp(c["clip"] / (torch.linalg.vector_norm(g, dim=1, keepdim=True) + 1e-6), max=1.0)
    m, v = _states64(s)
    m = 0.9 * m + (1.0 - 0.9) * g
    v = 0.999 * v + (1.0 - 0.999) * g * g
    shrink = torch.repeat_interleave(1.0 - c["lr"] * c["decay"] * s["decay"].double(), s["extents"])
    hat = (m / (1.0 - 0.9 ** n)) / (torch.sqrt(v / (1.0 - 0.999 ** n)) + 1e-8)
    theta = s["param"].double() * shrink - c["lr"] * hat
    out = {"param": theta}
    if "copy" in s:
        out["copy"] = theta
    return _states_out(out, s, m, v, K)


def _exact_sync(s):
    c, K = s["case"], s["case"]["workers"]
    theta = s["param"].double().mean(0, keepdim=True).expand(K, -1)
    out = {"param": theta}
    if "copy" in s:
        out["copy"] = theta
    if c["mode"] == "average":
        m, v = _states64(s)
        return _states_out(out, s, m.mean(0, keepdim=True), v.mean(0, keepdim=True), K)
    for name in ("m", "v", "m_scale", "v_scale"):
        if name in s:
            out[name] = s[name] if c["mode"] == "keep" else torch.zeros_like(s[name])
    return out


def _exact_logprobs(s):
    c, y, V = s["case"], s["tokens"], s["case"]["vocab"]
    keys = ("logprob", "entropy") + (("top_logprob",) if c["top"] else ()) + (("d_logits",) if c["gradient"] != "none" else ())
    parts = {k: [] for k in keys}
    rows = max(1, (1 << 27) // V)
    for at in range(0, y.numel(), rows):
        x = s["logits"][at:at + rows].double() / c["temperature"]
        t = y[at:at + rows]
        lse = torch.logsumexp(x, 1, keepdim=True)
        p = torch.nan_to_num(torch.exp(x - lse), nan=0.0)
        live = ~torch.isneginf(lse)
        H = torch.special.entr(p).sum(1, keepdim=True)
        own_x = x.gather(1, t.clamp_min(0)[:, None])
        lp = torch.where(live, own_x - lse, -math.inf)
        parts["logprob"].append(torch.where(t >= 0, lp[:, 0], 0.0))
        parts["entropy"].append(H[:, 0])
        if c["top"]:
            v = torch.sort(x, dim=1, descending=True).values[:, :min(c["top"], V)]
            parts["top_logprob"].append(torch.where(live, v - lse, -math.inf))
        if c["gradient"] != "none":
            hot = torch.zeros_like(p)
            hot[torch.arange(t.numel(), device=t.device), t.clamp_min(0)] = 1.0
            a = torch.where((t >= 0)[:, None] & live, s["d_logprob"][at:at + rows, None].double(), 0.0)
            d = a * (hot - p)
            if s["d_entropy"] is not None:
                d += s["d_entropy"][at:at + rows, None].double() * (torch.special.entr(p) - p * H)
            parts["d_logits"].append(d / c["temperature"])
    out = {k: torch.cat(v) for k, v in parts.items()}
    if c["top"]:
        out["top_token"] = None
    return out
