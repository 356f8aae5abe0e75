"""Log probabilities of given tokens on the GPU -- values, entropy, alternatives, gradient -- against the definition in
binary64.  Tolerances are sums of roundings (u = 2^-24): the exponent of each term is rounded three times and raised by an
instruction good to 2^-22, at most 256 terms are added one after another, then trees."""
import math

import numpy as np
import pytest
import torch

from paper_2310_14423_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
T = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 2.0 ** -126, "bf16": 2.0 ** -126, "f16": 2.0 ** -25}
LOWEST = {"f32": -3.4028234663852886e38, "bf16": -3.3895313892515355e38, "f16": -65504.0}


def reference(x, y, tau, top, a, b):
    """Everything in binary64, row by row: x [R, V] float64 (of the logits' own values)."""
    R, V = x.shape
    out = {k: [] for k in ("logprob", "entropy", "M", "lnS", "top_token", "top_logprob", "d", "p")}
    for r in range(R):
        row = x[r]
        M = row.max()
        nan = not (M < math.inf)
        if nan:
            M, lnS, lp, p, H = math.nan, math.nan, np.full(V, math.nan), np.full(V, math.nan), math.nan
        elif M == -math.inf:
            lnS, lp, p, H = 0.0, np.full(V, -math.inf), np.zeros(V), 0.0
        else:
            z = tau * (row - M)
            e = np.exp(z)
            lnS = math.log(math.fsum(e)) if V < 5000 else math.log(e.sum())
            lp, p = z - lnS, e / e.sum()
            H = -float(np.where(p > 0, p * np.where(p > 0, lp, 0.0), 0.0).sum())
        own = 0.0 if y[r] < 0 else (lp[y[r]] if y[r] < V else math.nan)
        order = np.lexsort((np.arange(V), -np.where(np.isnan(row), math.inf, row), ~np.isnan(row)))[:top] if top else np.arange(0)
        d = np.zeros(V)
        if not (M == -math.inf):
            ar = 0.0 if y[r] < 0 else (a[r] if y[r] < V else math.nan)
            d = -ar * p - b[r] * p * (np.where(p > 0, lp, 0.0) + H)
            if 0 <= y[r] < V:
                d[y[r]] += ar
        for k, v in (("logprob", own), ("entropy", H), ("M", M), ("lnS", lnS), ("top_token", order), ("top_logprob", lp[order]), ("d", tau * d), ("p", p)):
            out[k].append(v)
    return {k: np.asarray(v) for k, v in out.items()}


def close(got, want, tol):
    """Equal within tol where finite; the same non-finite values elsewhere."""
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    ok = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[~ok & ~np.isnan(want)], want[~ok & ~np.isnan(want)])
    tol = np.broadcast_to(tol, want.shape)
    assert np.all(np.abs(got - want)[ok] <= tol[ok]), (np.max((np.abs(got - want) / tol)[ok]), )


class Call:
    def __init__(self, x, y, kind, stride=None, offset=0, d_offset=0, in_place=False):
        R, V = x.shape
        self.kind, self.R, self.V = kind, R, V
        stride = V if stride is None else stride

        def strided(off):
            flat = torch.full((off + R * stride + 8,), 5.0, device=DEV).to(T[kind])
            return flat, flat.as_strided((R, V), (stride, 1), off)

        self.flat, self.x = strided(offset)
        self.x.copy_(torch.as_tensor(x).to(DEV))
        self.d_flat, self.d = (self.flat, self.x) if in_place else strided(d_offset)
        self.y = torch.as_tensor(np.asarray(y, np.int64)).to(DEV)
        self.x64 = self.x.double().cpu().numpy()
        inside = torch.zeros_like(self.d_flat, dtype=torch.bool)
        inside.as_strided((R, V), (stride, 1), offset if in_place else d_offset).fill_(True)
        self.outside = ~inside

    def forward(self, tau, top=0, a=None, b=None, fused=False):
        R = self.R
        f = lambda *s: torch.full(s, 9.0, device=DEV)      # noqa: E731
        self.logprob, self.entropy, self.stats = f(R), f(R), f(R, 2)
        self.top_lp, self.top = (f(R, top), torch.full((R, top), -7, device=DEV)) if top else (None, None)
        self.a = None if a is None else torch.as_tensor(a, dtype=torch.float32).to(DEV)
        self.b = None if b is None else torch.as_tensor(b, dtype=torch.float32).to(DEV)
        kw = dict(d_logprob=self.a, d_entropy=self.b, d_logits=self.d) if fused else {}
        B.qsr_token_logprobs(self.x, self.y, self.logprob, entropy=self.entropy, row_stats=self.stats, top_logprob=self.top_lp,
                             top_token=self.top, inv_temperature=tau, stream=torch.cuda.current_stream().cuda_stream, **kw)

    def backward(self, tau):
        B.qsr_token_logprobs_grad(self.x, self.y, self.stats, self.d, d_logprob=self.a, d_entropy=self.b, entropy=self.entropy,
                                  inv_temperature=tau, stream=torch.cuda.current_stream().cuda_stream)

    def check(self, tau, top=0, a=None, b=None, gradient=False):
        zero = np.zeros(self.R)
        a32 = zero if a is None else np.asarray(a, np.float32).astype(np.float64)
        b32 = zero if b is None else np.asarray(b, np.float32).astype(np.float64)
        tau32 = float(np.float32(tau))
        w = reference(self.x64, self.y.cpu().numpy(), tau32, top, a32, b32)
        with np.errstate(invalid="ignore", over="ignore"):
            # ln S: relative error of S (256 + 32 additions, exponents' errors weighted by their terms, at most 2^-22 + 8u)
            eS = 300 * U + 2.0 ** -22
            close(self.stats[:, 0].cpu(), w["M"], 0.0)
            close(self.stats[:, 1].cpu(), w["lnS"], eS + 2 * U * np.abs(w["lnS"]))
            z = np.abs(w["logprob"]) + np.abs(w["lnS"])
            close(self.logprob.cpu(), w["logprob"], eS + 8 * U * z)
            close(self.entropy.cpu(), w["entropy"], 2 * eS * (1 + np.abs(w["lnS"]) + np.abs(w["entropy"])))
            if top:
                assert np.array_equal(self.top.cpu().numpy(), w["top_token"])
                close(self.top_lp.cpu(), w["top_logprob"], eS + 8 * U * (np.abs(w["top_logprob"]) + np.abs(w["lnS"])[:, None]))
            if gradient:
                p, H = w["p"], w["entropy"][:, None]
                lp = np.where(p > 0, -np.log(np.maximum(p, 1e-300)), 0.0)
                scale = np.abs(a32)[:, None] + np.abs(b32)[:, None] * (lp + H + 1)
                tol = tau32 * (p * scale * (2 * eS + 8 * U * (lp + np.abs(w["lnS"])[:, None])) + 4 * U * np.abs(a32)[:, None])
                tol = tol + HALF_ULP[self.kind] * np.abs(w["d"]) * (1 if self.kind != "f32" else 4) + TINY[self.kind]
                close(self.d.double().cpu(), w["d"], tol)
                assert bool((self.d_flat[self.outside].float() == 5.0).all())


def draw(R, V, kind, seed=0, spread=3.0, masked=0.0):
    rng = np.random.default_rng(seed)
    x = rng.normal(0, spread, (R, V))
    x[np.arange(R), rng.integers(0, V, R)] += rng.uniform(0, 12, R)
    if masked:
        x[rng.random((R, V)) < masked] = -math.inf
    y = rng.integers(0, V, R)
    y[rng.random(R) < 0.2] = -100
    return x, y, rng.normal(0, 1, R), rng.normal(0, 0.5, R)


SHAPES = [(1, 1), (2, 2), (3, 7), (5, 8), (4, 9), (7, 31), (3, 32), (9, 33), (6, 255), (5, 1000), (33, 1001), (4, 4099), (3, 32768), (2, 50001),
          (1, 131072), (9, 131072), (200, 3001), (2, 300001)]


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("R,V", SHAPES)
def test_forward_top_and_fused_gradient(R, V, kind):
    top = min(V, 20)
    x, y, a, b = draw(R, V, kind, seed=V)
    c = Call(x, y, kind)
    c.forward(1.0, top=top, a=a, b=b, fused=True)
    c.check(1.0, top=top, a=a, b=b, gradient=True)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("R,V", SHAPES)
def test_separate_gradient(R, V, kind):
    x, y, a, b = draw(R, V, kind, seed=V + 1, masked=0.3)
    c = Call(x, y, kind)
    c.forward(0.7, a=a, b=b)
    c.backward(0.7)
    c.check(0.7, a=a, b=b, gradient=True)


@pytest.mark.parametrize("which", ["a", "b", "none"])
def test_gradient_terms_alone(which):
    x, y, a, b = draw(6, 500, "f32")
    a, b = (a if which == "a" else None), (b if which == "b" else None)
    for fused in (True, False):
        c = Call(x, y, "f32")
        c.forward(1.3, a=a, b=b, fused=fused)
        if not fused:
            c.backward(1.3)
        c.check(1.3, a=a, b=b, gradient=True)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("stride,offset,d_offset", [(1040, 0, 0), (1001, 1, 1), (1003, 3, 0), (1007, 5, 2), (4096, 7, 7)])
def test_strides_and_alignment(kind, stride, offset, d_offset):
    x, y, a, b = draw(7, 1001, kind)
    for fused in (True, False):
        c = Call(x, y, kind, stride=stride, offset=offset, d_offset=d_offset)
        c.forward(1.0, top=5, a=a, b=b, fused=fused)
        if not fused:
            c.backward(1.0)
        c.check(1.0, top=5, a=a, b=b, gradient=True)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", [20, 1001, 50001, 131072])
@pytest.mark.parametrize("fused", [True, False])
def test_in_place_gradient(kind, V, fused):
    x, y, a, b = draw(4, V, kind)
    c = Call(x, y, kind, stride=V + 3, offset=1, in_place=True)
    c.forward(1.0, top=3, a=a, b=b, fused=fused)
    if not fused:
        c.backward(1.0)
    c.check(1.0, top=3, a=a, b=b, gradient=True)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", [1, 37, 1000, 60000, 300000])
def test_difficult_rows(kind, V):
    """Masked rows, rows of the type's lowest value, ties, NaN and infinities, tokens out of range, masked tokens."""
    rng = np.random.default_rng(V)
    rows, y = [], []

    def add(row, token):
        rows.append(np.broadcast_to(np.asarray(row, np.float64), (V,)).copy())
        y.append(token)

    base = rng.normal(0, 2, V)
    add(-math.inf, 0)                               # nothing left
    add(-math.inf, -1)
    add(LOWEST[kind], V - 1)                        # masked with the lowest value: uniform
    half = np.where(np.arange(V) % 2 == 0, base, -math.inf)
    add(half, min(V - 1, 1))                        # the token itself is masked (V > 1)
    add(np.where(np.arange(V) % 2 == 0, base, LOWEST[kind]), 0)
    add(np.where(np.arange(V) == V // 2, 1.5, -math.inf), V // 2)        # one token left
    add(0.25, V // 3)                               # all equal: ties go to the lowest index
    add(np.round(base), 0)                          # many ties
    add(np.sort(base), V - 1)
    add(-np.sort(base), 0)
    add(np.where(np.arange(V) == V // 2, math.nan, base), 0)
    add(np.where(np.arange(V) == 0, math.nan, base), 0)
    add(np.where(np.arange(V) == V - 1, math.inf, base), 0)
    add(base, V)                                    # token out of range
    add(base, -1)
    add(np.where(base > 0, 0.0, -0.0), 0)           # zeros of both signs are equal
    add(30.0 * base, int(np.argmax(base)))
    add(1000.0 * base, int(np.argmin(base)))
    x = np.stack(rows)
    a, b = rng.normal(0, 1, len(rows)), rng.normal(0, 1, len(rows))
    top = min(V, B.QSR_MAX_TOP)
    for fused in (True, False):
        c = Call(x, y, kind)
        c.forward(1.0, top=top, a=a, b=b, fused=fused)
        if not fused:
            c.backward(1.0)
        c.check(1.0, top=top, a=a, b=b, gradient=True)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_rows_longer_than_shared_memory(kind):
    x, y, a, b = draw(2, 1_700_003, kind, masked=0.1)
    for fused in (True, False):
        c = Call(x, y, kind, offset=1)
        c.forward(1.0, top=32, a=a, b=b, fused=fused)
        if not fused:
            c.backward(1.0)
        c.check(1.0, top=32, a=a, b=b, gradient=True)


@pytest.mark.parametrize("top", [1, 2, 19, 32])
@pytest.mark.parametrize("V", [64, 777, 40000, 140000])
def test_top_counts(top, V):
    x, y, _, _ = draw(5, V, "bf16", seed=top, spread=1.0)
    c = Call(x, y, "bf16")
    c.forward(1.0, top=top)
    c.check(1.0, top=top)


def test_gradient_against_differences():
    """Central differences of the call's own outputs: f = sum a logprob + b H.  Step h = 2^-6: truncation at most h^2/6 |f'''|
    (|f'''| below 8 here), rounding 2^-18 / h."""
    x, y, a, b = draw(1, 13, "f32", seed=2, spread=1.0)
    y[0] = 4
    h = 2.0 ** -6

    def f(xx):
        c = Call(xx, y, "f32")
        c.forward(1.1)
        return float(a[0] * c.logprob[0].double() + b[0] * c.entropy[0].double())

    c = Call(x, y, "f32")
    c.forward(1.1, a=a, b=b, fused=True)
    d = c.d.double().cpu().numpy()[0]
    for j in range(13):
        step = np.zeros((1, 13))
        step[0, j] = h
        num = (f(x + step) - f(x - step)) / (2 * h)
        assert abs(num - d[j]) <= 8 * h * h / 6 + 2.0 ** -18 / h, (j, num, d[j])


def test_same_bits_every_time_and_on_another_stream():
    x, y, a, b = draw(40, 50001, "bf16")
    runs = []
    for k in range(3):
        s = torch.cuda.Stream() if k == 2 else torch.cuda.current_stream()
        c = Call(x, y, "bf16")
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            c.forward(1.0, top=20, a=a, b=b, fused=True)
            s.synchronize()
        runs.append((c.logprob, c.entropy, c.top, c.top_lp, c.d))
    for other in runs[1:]:
        assert all(torch.equal(p, q) for p, q in zip(runs[0], other))


def test_graph_replay():
    x, y, a, b = draw(4, 131072, "bf16")
    c = Call(x, y, "bf16")
    c.forward(1.0, top=4, a=a, b=b, fused=True)
    want = c.logprob.clone(), c.d.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.forward(1.0, top=4, a=c.a, b=c.b, fused=True)
    c.d.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(c.logprob, want[0]) and torch.equal(c.d, want[1])


def test_offsets_beyond_32_bits():
    """Rows 2^30 elements apart."""
    V, stride, R = 1003, (1 << 30) + 1, 5
    x, y, a, b = draw(R, V, "bf16")
    flat = torch.empty((R - 1) * stride + V, device=DEV, dtype=torch.bfloat16)
    c = Call(x, y, "bf16")
    view = flat.as_strided((R, V), (stride, 1))
    view.copy_(c.x)
    c.x = c.d = view
    c.outside = torch.zeros(1, dtype=torch.bool, device=DEV)
    c.d_flat = torch.zeros(1, device=DEV)
    c.forward(1.0, top=4, a=a, b=b)
    c.backward(1.0)
    c.check(1.0, top=4, a=a, b=b, gradient=True)


def test_no_rows_and_python_refusals():
    f = lambda *s, **k: torch.zeros(*s, device=DEV, **k)      # noqa: E731
    i64 = torch.int64
    B.qsr_token_logprobs(f(0, 5), f(0, dtype=i64), f(0))
    x, y, o = f(3, 5), f(3, dtype=i64), f(3)
    for bad in (dict(logits=f(3, 5, dtype=torch.float64)), dict(logits=f(5, 3).t()), dict(logits=f(15)), dict(logits=torch.zeros(3, 5)),
                dict(tokens=f(3, dtype=torch.int32)), dict(tokens=f(2, dtype=i64)), dict(logprob=f(4)), dict(logprob=f(3, dtype=torch.float64)),
                dict(entropy=f(2)), dict(row_stats=f(3)), dict(top_token=f(3, 2, dtype=i64)), dict(d_logits=f(3, 4)),
                dict(top_token=f(3, 2, dtype=i64), top_logprob=f(3, 3))):
        with pytest.raises(ValueError):
            B.qsr_token_logprobs(**{**dict(logits=x, tokens=y, logprob=o), **bad})
    for kw, status in ((dict(inv_temperature=0.0), B.QSR_EINVAL), (dict(inv_temperature=math.inf), B.QSR_EINVAL),
                       (dict(inv_temperature=math.nan), B.QSR_EINVAL), (dict(inv_temperature=1e-60), B.QSR_EINVAL),
                       (dict(top_token=f(3, 6, dtype=i64), top_logprob=f(3, 6)), B.QSR_ERANGE)):
        with pytest.raises(B.QsrError) as e:
            B.qsr_token_logprobs(x, y, o, **kw)
        assert e.value.status == status
    wide = f(3, 50)
    with pytest.raises(B.QsrError) as e:
        B.qsr_token_logprobs(wide, y, o, top_token=f(3, 33, dtype=i64), top_logprob=f(3, 33))
    assert e.value.status == B.QSR_ERANGE
    with pytest.raises(B.QsrError) as e:
        B.qsr_token_logprobs_grad(x, y, None, f(3, 5), d_logprob=o)
    assert e.value.status == B.QSR_EINVAL
    with pytest.raises(B.QsrError) as e:
        B.qsr_token_logprobs_grad(x, y, f(3, 2), f(3, 5), d_entropy=o)      # entropy is needed
    assert e.value.status == B.QSR_EINVAL


FAR = [-1e9, -1e10, -1e12, -1e15, -1e20, -1e29]


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("V", [37, 1024, 20001, 140000, 300000])
def test_logits_far_from_zero(kind, V):
    """Masks and whole rows of large magnitude, short of the type's lowest value: scattered, over whole threads, warps and
    slices, several of them in one row, and rows whose largest logit is itself far below or above zero."""
    rng = np.random.default_rng(V)
    at, base = np.arange(V), rng.normal(0, 2, V)
    rows, y = [], []

    def add(row, token):
        rows.append(np.broadcast_to(np.asarray(row, np.float64), (V,)).copy())
        y.append(token)

    for far in FAR if V < 50000 else FAR[1::3]:
        add(np.where(rng.random(V) < 0.9, far, base), int(rng.integers(V)))
        add(np.where(at < V - V // 8 - 1, far, base), V - 1)
        add(np.where(at > V // 8, far, base), 0)
        add(np.where(at == V // 2, base, far), V // 2)
        add(far, V // 3)
        add(np.where(at % 3 == 0, far, -math.inf), 0)
        add(np.where(at % 2 == 0, far, 4 * far), 1)
        add(-far, V // 2)
        add(np.where(at == V // 2, -far, base), V // 2)
        add(np.where(at < V // 2, -far, far), 0)
    add(np.where(at < V // 2, base, np.asarray(FAR)[at % len(FAR)]), 0)
    x = np.stack(rows)
    a, b = rng.normal(0, 1, len(rows)), rng.normal(0, 1, len(rows))
    for first in range(0, len(rows), 12):                 # few rows at a time: long ones are shared out over clusters then
        s = slice(first, first + 12)
        for fused in (True, False):
            c = Call(x[s], y[s], kind)
            c.forward(1.0, top=min(V, 5), a=a[s], b=b[s], fused=fused)
            if not fused:
                c.backward(1.0)
            c.check(1.0, top=min(V, 5), a=a[s], b=b[s], gradient=True)


@pytest.mark.parametrize("tau", [1e-9, 0.5, 1e6, 1e9])
@pytest.mark.parametrize("V", [1024, 60000])
def test_temperatures_far_from_one(V, tau):
    """Scaled logits far from zero: ordinary logits and ones that differ by little, about ten and about minus ten."""
    rng = np.random.default_rng(7)
    near = rng.integers(-8, 8, (3, V)) * 2.0 ** -20
    x = np.concatenate([rng.normal(0, 3, (2, V)), 10 + near, near - 10, np.where(rng.random((2, V)) < 0.9, -1e9, rng.normal(0, 3, (2, V)))])
    y, a, b = rng.integers(0, V, len(x)), rng.normal(0, 1, len(x)), rng.normal(0, 1, len(x))
    for fused in (True, False):
        c = Call(x, y, "f32")
        c.forward(tau, top=3, a=a, b=b, fused=fused)
        if not fused:
            c.backward(tau)
        c.check(tau, top=3, a=a, b=b, gradient=True)


@pytest.mark.parametrize("V,stride,at", [(100, 200, 100), (100, 250, 100), (100, 250, 150), (1001, 2003, 1002)])
def test_gradient_in_other_columns_of_the_logits_buffer(V, stride, at):
    x, y, a, b = draw(6, V, "bf16")
    want = Call(x, y, "bf16")
    want.forward(1.0, a=a, b=b, fused=True)
    buffer = torch.full((6, stride), 5.0, device=DEV, dtype=torch.bfloat16)
    for fused in (True, False):
        c = Call(x, y, "bf16")
        buffer[:, :V] = c.x
        c.x, c.d = buffer[:, :V], buffer[:, at:at + V]
        c.forward(1.0, a=a, b=b, fused=fused)
        if not fused:
            c.backward(1.0)
        assert torch.equal(c.x, want.x) and torch.allclose(c.d.float(), want.d.float(), rtol=2.0 ** -7, atol=1e-6)
        used = torch.zeros(stride, dtype=torch.bool, device=DEV)
        used[:V] = used[at:at + V] = True
        assert bool((buffer[:, ~used] == 5.0).all())
