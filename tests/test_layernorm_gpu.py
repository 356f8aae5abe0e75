"""Layer norm forward and backward on the GPU against the formulas in binary64.  Tolerances count roundings (u = 2^-24): a thread adds
at most 8 * 4 elements (8 per 8192 of the row for longer ones), then come trees over lanes and warps."""
import math

import pytest
import torch

from paper_2310_14423_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
T = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 2.0 ** -126, "bf16": 2.0 ** -126, "f16": 2.0 ** -25}
EPS = 1e-5


def stream():
    return torch.cuda.current_stream().cuda_stream


def chain(n):
    """Additions in a row's longest chain."""
    return 64 + 8 * math.ceil(n / 8192)


def matrix(x, kind, pad=0, shift=0):
    """x as the leading columns of rows `pad` longer, `shift` elements behind an allocation's start."""
    R, N = x.shape
    flat = torch.full((R * (N + pad) + shift,), 7.0, device=DEV, dtype=T[kind])
    m = flat[shift:].view(R, N + pad)[:, :N]
    m.copy_(x)
    return m


def untouched(m, pad, shift):
    """Whether what lies around a matrix of `matrix` is as it was."""
    if not (pad or shift):
        return True
    R, N = m.shape
    base = torch.as_strided(m, (R * (N + pad) + shift,), (1,), m.storage_offset() - shift)
    return bool((base[:shift] == 7.0).all()) and bool((base[shift:].view(R, N + pad)[:, N:] == 7.0).all())


def close(got, want, tol):
    got = got.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    ok = torch.isfinite(want)
    assert torch.equal(got[~ok & ~torch.isnan(want)], want[~ok & ~torch.isnan(want)])
    bad = ((got - want).abs() > tol) & ok
    assert not bad.any(), (float(((got - want).abs() / tol)[ok].max()), int(bad.sum()))


def inputs(R, N, kind, wkind, seed=0, offset=0.5):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    n = lambda *s: torch.randn(*s, device=DEV, generator=g)        # noqa: E731
    x = (n(R, N) * (1 + 10 * (torch.rand(N, device=DEV, generator=g) < 0.05)) + offset * n(R, 1)).to(T[kind])
    return x, n(R, N).to(T[kind]), (1 + 0.3 * n(N)).to(T[wkind]), (0.1 * n(N)).to(T[wkind])


def forward64(x, w, b, eps=EPS):
    x = x.double()
    N = x.shape[1]
    mean = x.mean(1, keepdim=True)
    var = (x - mean).square().mean(1, keepdim=True)
    rstd = (var + eps).rsqrt()
    hat = (x - mean) * rstd
    w = torch.ones(N, device=DEV, dtype=torch.float64) if w is None else w.double()
    b = torch.zeros(N, device=DEV, dtype=torch.float64) if b is None else b.double()
    y = hat * w + b
    d_mean = (chain(N) + 1) * U * x.abs().mean(1, keepdim=True)
    d_var = (chain(N) + 4) * U * var + d_mean.square()
    r_rel = 0.5 * d_var / (var + eps) + 3 * U
    tol = (hat * w).abs() * (r_rel + 4 * U) + w.abs() * rstd * d_mean + 2 * U * y.abs()
    return mean, rstd, y, d_mean, r_rel * rstd, tol


def backward64(x, dy, mean, rstd, w):
    x, dy, mean, rstd = x.double(), dy.double(), mean.double()[:, None], rstd.double()[:, None]
    R, N = x.shape
    w = torch.ones(N, device=DEV, dtype=torch.float64) if w is None else w.double()
    hat = (x - mean) * rstd
    d = dy * w
    c1, c2 = d.mean(1, keepdim=True), (d * hat).mean(1, keepdim=True)
    dx = rstd * (d - c1 - hat * c2)
    e1 = (chain(N) + 3) * U * d.abs().mean(1, keepdim=True)
    e2 = (chain(N) + 6) * U * (d * hat).abs().mean(1, keepdim=True)
    tol = rstd * (e1 + hat.abs() * e2 + 5 * U * (d.abs() + c1.abs() + (hat * c2).abs()))
    # a thread adds the rows of its block, a block its groups of threads (256 at most), then 8 threads the blocks' sums
    depth = min(R, 8 * (R // 296 + 1)) + 256 + 48
    return dx, (dy * hat).sum(0), dy.sum(0), tol, (depth + 3) * U * (dy * hat).abs().sum(0), depth * U * dy.abs().sum(0)


def rounded(tol, want, kind):
    return tol * (1 + HALF_ULP[kind]) + HALF_ULP[kind] * want.abs() + TINY[kind]


SHAPES = [(1, 1), (3, 2), (2, 8), (5, 7), (300, 9), (17, 64), (129, 100), (64, 255), (33, 256), (40, 257), (700, 768), (5, 1000), (65, 1024), (9, 1025),
          (31, 4097), (12, 8192), (5, 8193), (6, 12345), (3, 32768), (4, 32769), (2, 70001)]


@pytest.mark.parametrize("kind,wkind", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f16", "f16")])
@pytest.mark.parametrize("R,N", SHAPES)
def test_forward(R, N, kind, wkind):
    x, _, w, b = inputs(R, N, kind, wkind, R + N)
    y, mean, rstd = torch.empty_like(x), torch.empty(R, device=DEV), torch.empty(R, device=DEV)
    B.qsr_layer_norm(x, y, weight=w, bias=b, mean=mean, rstd=rstd, eps=EPS, stream=stream())
    m64, r64, y64, dm, dr, tol = forward64(x, w, b)
    close(mean, m64[:, 0], dm[:, 0] + U * m64[:, 0].abs())
    close(rstd, r64[:, 0], dr[:, 0])
    close(y, y64, rounded(tol, y64, kind))


@pytest.mark.parametrize("kind,wkind", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f16", "f16")])
@pytest.mark.parametrize("R,N", SHAPES)
def test_backward(R, N, kind, wkind):
    x, dy, w, _ = inputs(R, N, kind, wkind, R + N + 1)
    m64, r64 = forward64(x, None, None)[:2]
    mean, rstd = m64[:, 0].float(), r64[:, 0].float()
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(w)
    ws = torch.empty(B.qsr_layer_norm_workspace_bytes(R, N), dtype=torch.uint8, device=DEV)
    B.qsr_layer_norm_grad(x, dy, mean, rstd, d_x=dx, weight=w, d_weight=dw, d_bias=db, workspace=ws, stream=stream())
    dx64, dw64, db64, tx, tw, tb = backward64(x, dy, mean, rstd, w)
    close(dx, dx64, rounded(tx, dx64, kind))
    close(dw, dw64, rounded(tw, dw64, wkind))
    close(db, db64, rounded(tb, db64, wkind))
    # the same bits again, and without the other outputs
    dx2, dw2 = torch.empty_like(x), torch.empty_like(w)
    ws.fill_(255)
    B.qsr_layer_norm_grad(x, dy, mean, rstd, weight=w, d_weight=dw2, workspace=ws, stream=stream())
    B.qsr_layer_norm_grad(x, dy, mean, rstd, d_x=dx2, weight=w, stream=stream())
    assert torch.equal(dw2, dw) and torch.equal(dx2, dx)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("pad,shift", [(0, 1), (3, 0), (8, 0), (5, 3)])
@pytest.mark.parametrize("R,N", [(7, 40), (10, 1001), (4, 4100), (3, 33000)])
def test_strides_and_alignment(R, N, pad, shift, kind):
    x, dy, w, b = inputs(R, N, kind, "f32", 3)
    w, b = matrix(w[None], "f32", 0, 1)[0], matrix(b[None], "f32", 0, 3)[0]
    mean, rstd = torch.empty(R, device=DEV), torch.empty(R, device=DEV)
    xs, dys, y, dx = matrix(x, kind, pad, shift), matrix(dy, kind, pad + 1, 0), matrix(torch.zeros_like(x), kind, pad, shift), matrix(torch.zeros_like(x), kind, 0, shift)
    B.qsr_layer_norm(xs, y, weight=w, bias=b, mean=mean, rstd=rstd, eps=EPS, stream=stream())
    _, _, y64, _, _, tol = forward64(x, w, b)
    close(y, y64, rounded(tol, y64, kind))
    dw, db = torch.empty_like(w), torch.empty_like(b)
    ws = torch.empty(B.qsr_layer_norm_workspace_bytes(R, N), dtype=torch.uint8, device=DEV)
    B.qsr_layer_norm_grad(xs, dys, mean, rstd, d_x=dx, weight=w, d_weight=dw, d_bias=db, workspace=ws, stream=stream())
    dx64, dw64, db64, tx, tw, tb = backward64(x, dy, mean, rstd, w)
    close(dx, dx64, rounded(tx, dx64, kind))
    close(dw, dw64, tw + U * dw64.abs())
    close(db, db64, tb + U * db64.abs())
    assert untouched(y, pad, shift) and untouched(dx, 0, shift)


@pytest.mark.parametrize("R,N", [(50, 768), (3, 9001), (2, 40000)])
def test_in_place(R, N):
    x, dy, w, b = inputs(R, N, "bf16", "bf16", 5)
    mean, rstd = torch.empty(R, device=DEV), torch.empty(R, device=DEV)
    y, dx, dw = torch.empty_like(x), torch.empty_like(x), torch.empty_like(w)
    ws = torch.empty(B.qsr_layer_norm_workspace_bytes(R, N), dtype=torch.uint8, device=DEV)
    B.qsr_layer_norm(x, y, weight=w, bias=b, mean=mean, rstd=rstd, stream=stream())
    B.qsr_layer_norm_grad(x, dy, mean, rstd, d_x=dx, weight=w, d_weight=dw, workspace=ws, stream=stream())
    for over in ("x", "dy"):
        a, d, dw2 = x.clone(), dy.clone(), torch.empty_like(w)
        B.qsr_layer_norm_grad(a, d, mean, rstd, d_x=a if over == "x" else d, weight=w, d_weight=dw2, workspace=ws, stream=stream())
        assert torch.equal(a if over == "x" else d, dx) and torch.equal(dw2, dw)
    a = x.clone()
    B.qsr_layer_norm(a, a, weight=w, bias=b, stream=stream())
    assert torch.equal(a, y)


def test_without_weight_and_bias():
    x, dy, w, b = inputs(20, 300, "f32", "f32", 6)
    y, mean, rstd = torch.empty_like(x), torch.empty(20, device=DEV), torch.empty(20, device=DEV)
    for ww, bb in ((None, None), (w, None), (None, b)):
        B.qsr_layer_norm(x, y, weight=ww, bias=bb, mean=mean, rstd=rstd, stream=stream())
        _, _, y64, _, _, tol = forward64(x, ww, bb)
        close(y, y64, rounded(tol, y64, "f32"))
    dx = torch.empty_like(x)
    B.qsr_layer_norm_grad(x, dy, mean, rstd, d_x=dx, stream=stream())
    dx64, _, _, tx, _, _ = backward64(x, dy, mean, rstd, None)
    close(dx, dx64, rounded(tx, dx64, "f32"))


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("N", [5, 768, 5000, 40000])
def test_rows_far_from_zero_and_constant_rows(kind, N):
    """Rows whose mean is large against their spread, and rows of one value (variance zero)."""
    x, _, w, b = inputs(6, N, kind, "f32", 7)
    x = (x.float() + torch.tensor([0.0, 100.0, -1000.0, 4096.0, 0.0, 0.0], device=DEV)[:, None]).to(T[kind])
    x[4] = 3.0
    x[5] = 0.0
    y = torch.empty_like(x)
    B.qsr_layer_norm(x, y, weight=w, bias=b, stream=stream())
    _, _, y64, _, _, tol = forward64(x, w, b)
    close(y, y64, rounded(tol, y64, kind))


def test_values_that_are_not_finite_stay_in_their_rows():
    x, dy, w, b = inputs(9, 500, "bf16", "f32", 8)
    clean, mean, rstd = torch.empty_like(x), torch.empty(9, device=DEV), torch.empty(9, device=DEV)
    B.qsr_layer_norm(x, clean, weight=w, bias=b, mean=mean, rstd=rstd, stream=stream())
    dx0, dx = torch.empty_like(x), torch.empty_like(x)
    B.qsr_layer_norm_grad(x, dy, mean, rstd, d_x=dx0, weight=w, stream=stream())
    x[2, 10], x[5, 499], y = math.inf, math.nan, torch.empty_like(x)
    B.qsr_layer_norm(x, y, weight=w, bias=b, mean=mean, rstd=rstd, stream=stream())
    rows = [r for r in range(9) if r not in (2, 5)]
    assert torch.equal(y[rows], clean[rows]) and torch.isnan(y[5]).all() and torch.isnan(y[2]).all()
    B.qsr_layer_norm_grad(x, dy, mean, rstd, d_x=dx, weight=w, stream=stream())
    assert torch.equal(dx[rows], dx0[rows]) and torch.isnan(dx[5]).all()


def test_gradient_against_differences():
    """The gradient of sum(c * y) in fp32 against central differences of the formula in binary64."""
    R, N, h = 3, 33, 1e-5
    x, c, w, b = inputs(R, N, "f32", "f32", 9)
    mean, rstd, y = torch.empty(R, device=DEV), torch.empty(R, device=DEV), torch.empty_like(x)
    B.qsr_layer_norm(x, y, weight=w, bias=b, mean=mean, rstd=rstd, stream=stream())
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
    ws = torch.empty(B.qsr_layer_norm_workspace_bytes(R, N), dtype=torch.uint8, device=DEV)
    B.qsr_layer_norm_grad(x, c, mean, rstd, d_x=dx, weight=w, d_weight=dw, d_bias=db, workspace=ws, stream=stream())
    value = lambda X, W, Bb: float((c.double() * forward64(X, W, Bb)[2]).sum())             # noqa: E731
    X, W, Bb = x.double(), w.double(), b.double()
    for args, grad in ((0, dx), (1, dw), (2, db)):
        flat = [X, W, Bb][args].view(-1)
        for i in range(0, flat.numel(), 7):
            keep = float(flat[i])
            flat[i] = keep + h
            up = value(X, W, Bb)
            flat[i] = keep - h
            down = value(X, W, Bb)
            flat[i] = keep
            # third derivatives of a row are below 100 here: h^2 * 100 / 6, and fp32 roundings
            assert abs((up - down) / (2 * h) - float(grad.view(-1)[i])) < 2e-5 * (1 + abs(float(grad.view(-1)[i])))


def test_no_rows():
    x, w = torch.empty(0, 10, device=DEV), torch.ones(10, device=DEV)
    none = torch.empty(0, device=DEV)
    B.qsr_layer_norm(x, x, weight=w, mean=none, rstd=none, stream=stream())
    dw, db = torch.full_like(w, 3.0), torch.full_like(w, 3.0)
    ws = torch.empty(B.qsr_layer_norm_workspace_bytes(0, 10), dtype=torch.uint8, device=DEV)
    B.qsr_layer_norm_grad(x, x, none, none, weight=w, d_weight=dw, d_bias=db, workspace=ws, stream=stream())
    assert not dw.any() and not db.any()


def test_captured_and_on_a_stream_of_its_own():
    x, dy, w, b = inputs(200, 768, "bf16", "bf16", 10)
    y, mean, rstd = torch.empty_like(x), torch.empty(200, device=DEV), torch.empty(200, device=DEV)
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
    ws = torch.empty(B.qsr_layer_norm_workspace_bytes(200, 768), dtype=torch.uint8, device=DEV)

    def both():
        B.qsr_layer_norm(x, y, weight=w, bias=b, mean=mean, rstd=rstd, stream=stream())
        B.qsr_layer_norm_grad(x, dy, mean, rstd, d_x=dx, weight=w, d_weight=dw, d_bias=db, workspace=ws, stream=stream())

    both()
    first = [t.clone() for t in (y, dx, dw, db)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        both()
    for t in (y, dx, dw, db):
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(first, (y, dx, dw, db)))
    x.mul_(2.0)                        # the graph reads what is there at the replay
    graph.replay()
    _, _, y64, _, _, tol = forward64(x, w, b)
    close(y, y64, rounded(tol, y64, "bf16"))


@pytest.mark.parametrize("kind,wkind", [("f32", "f32"), ("bf16", "f32"), ("f16", "f16")])
@pytest.mark.parametrize("R,N", [(4800, 1032), (2368, 2048), (2367, 2045), (2400, 3001), (2369, 4096), (1200, 4101), (592, 8192), (600, 8193), (296, 16384), (592, 16389), (300, 12000)])
def test_many_wide_rows(R, N, kind, wkind):
    """Enough rows for blocks that stay, and a few less; buffers as below; in place."""
    x, _, w, b = inputs(R, N, kind, wkind, R + N)
    pad = -N % 8

    def wide(m):
        flat = torch.full((R * (N + pad) - pad,), math.nan, device=DEV, dtype=T[kind])
        out = flat.as_strided((R, N), (N + pad, 1))
        out.copy_(m)
        return out

    xs, y, mean, rstd = wide(x), wide(torch.zeros_like(x)), torch.empty(R, device=DEV), torch.empty(R, device=DEV)
    B.qsr_layer_norm(xs, y, weight=w, bias=b, mean=mean, rstd=rstd, eps=EPS, stream=stream())
    for rows in (slice(0, R // 2), slice(R // 2, R)):
        m64, r64, y64, dm, dr, tol = forward64(x[rows], w, b)
        close(mean[rows], m64[:, 0], dm[:, 0] + U * m64[:, 0].abs())
        close(rstd[rows], r64[:, 0], dr[:, 0])
        close(y[rows], y64, rounded(tol, y64, kind))
    xs[R // 3, N - 1] = math.nan
    B.qsr_layer_norm(xs, xs, weight=w, bias=b, eps=EPS, stream=stream())
    rows = torch.arange(R, device=DEV) != R // 3
    assert torch.equal(xs[rows], y[rows]) and torch.isnan(xs[R // 3]).all()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("R,N", [(1, 3080), (2, 3136), (148, 3081), (149, 4096), (297, 4100), (445, 5003), (300, 6144), (900, 3500), (450, 6145), (297, 8185), (151, 8192)])
def test_wide_rows_in_aligned_buffers(R, N, kind):
    """Rows that a block takes alone, several for each block, in buffers whose other columns are not numbers, and which end with the last row."""
    x, dy, w, _ = inputs(R, N, kind, kind, R + N)
    m64, r64 = forward64(x, None, None)[:2]
    mean, rstd = m64[:, 0].float(), r64[:, 0].float()
    pad = -N % 8

    def wide(m):
        flat = torch.full((R * (N + pad) - pad,), math.nan, device=DEV, dtype=T[kind])
        out = flat.as_strided((R, N), (N + pad, 1))
        out.copy_(m)
        return out

    xs, dys, dx = wide(x), wide(dy), wide(torch.zeros_like(x))
    dw, db = torch.empty_like(w), torch.empty_like(w)
    ws = torch.empty(B.qsr_layer_norm_workspace_bytes(R, N), dtype=torch.uint8, device=DEV)
    B.qsr_layer_norm_grad(xs, dys, mean, rstd, d_x=dx, weight=w, d_weight=dw, d_bias=db, workspace=ws, stream=stream())
    dx64, dw64, db64, tx, tw, tb = backward64(x, dy, mean, rstd, w)
    close(dx, dx64, rounded(tx, dx64, kind))
    close(dw, dw64, rounded(tw, dw64, kind))
    close(db, db64, rounded(tb, db64, kind))
    dw2 = torch.empty_like(w)
    B.qsr_layer_norm_grad(xs, dys, mean, rstd, weight=w, d_weight=dw2, workspace=ws, stream=stream())
    assert torch.equal(dw2, dw)
    for over in (wide(x), wide(dy)):
        a, d = (over, dys) if torch.equal(over, xs) else (xs, over)
        B.qsr_layer_norm_grad(a, d, mean, rstd, d_x=over, weight=w, stream=stream())
        assert torch.equal(over, dx)
    if R > 2:
        xs[R // 2, N - 1] = math.nan
        dx2 = wide(torch.zeros_like(x))
        B.qsr_layer_norm_grad(xs, dys, mean, rstd, d_x=dx2, weight=w, stream=stream())
        rows = torch.arange(R, device=DEV) != R // 2
        assert torch.equal(dx2[rows], dx[rows]) and torch.isnan(dx2[R // 2]).all()
