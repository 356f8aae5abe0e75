"""Steps by orthogonalised momentum on the GPU against the formulas in binary64, with a bound on the iteration's error that is
carried along with the binary64 iterates.

One iteration maps singular values by p(s) = a s + b s^3 + c s^5, and to first order a perturbation of an iterate grows at most by the
largest of (p(s) - p(t)) / (s - t), (p(s) + p(t)) / (s + t) and p(s) / s over its singular values.  Added to it, in the 2-norm of all entries:
the roundings of X, A and C where they are held (E relative to each entry), and those of the three products (G relative to the
product of absolute values).  E = 2^-11 for fp16, 2^-22 for a sum of two, which also leaves out products of 2^-22; the tensor cores
add 16 products and the accumulator at a time and may cut off the result, 2^-23 each: `sums` / 16 times with one product,
at most 12 times with three before fp32 registers take over (2^-24 each)."""
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
a, b, c = 3.4445, -4.7750, 2.0315


def growth(s):
    """The largest divided difference of p over the singular values s."""
    x, y = s[:, None], s[None, :]
    even = x * x + x * y + y * y                                    # (x^3 - y^3) / (x - y)
    fifth = x ** 4 + x ** 3 * y + x * x * y * y + x * y ** 3 + y ** 4
    odd_even = x * x - x * y + y * y                                # (x^3 + y^3) / (x + y)
    odd_fifth = x ** 4 - x ** 3 * y + x * x * y * y - x * y ** 3 + y ** 4
    return max(float((a + b * even + c * fifth).abs().max()), float((a + b * odd_even + c * odd_fifth).abs().max()),
               float((a + b * s ** 2 + c * s ** 4).abs().max()))



def stream():
    return torch.cuda.current_stream().cuda_stream


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def orthogonal64(u, iterations, eps, products):
    """(X, bound on the 2-norm of the entries' error) for one matrix in binary64, rounded where X, A and C are held in fp16."""
    X = u / (torch.linalg.vector_norm(u) + eps)
    tall = X.shape[0] > X.shape[1]
    X = X.T if tall else X
    m, n = X.shape
    # With one product the reference rounds where the kernels do, at the same powers of two.  What is left are entries that lie nearer to
    # a boundary than the products' error G (below 2^-17 of them, 2^-7 of a step) and fall to its other side: one in 2^6, each a
    # step off, which is 2^-3 of a step in the mean over many entries and up to a whole one over few.
    e = 2.0 ** -11 * min(1.0, 0.25 + 4.0 / math.sqrt(m * n)) if products == 1 else 2.0 ** -22
    scale = 2.0 ** min(15, math.floor(0.5 * math.log2(m * n)))
    held = (lambda M, at: (M * at).half().double() / at) if products == 1 else (lambda M, at: M)
    gamma = (lambda k: (k / 16 + 1) * 2.0 ** -23) if products == 1 else (lambda k: 12 * 2.0 ** -23 + (k / 64 + 2) * 2.0 ** -24 + 2.0 ** -22)
    norm = lambda M: float(torch.linalg.vector_norm(M))                # noqa: E731
    grain = 2.0 ** -25 * 2                                             # fp16's smallest step against entries of about one
    X = held(X, scale)
    err = e * norm(X) + 8 * U * norm(X) + grain
    eye = torch.eye(m, device=DEV, dtype=torch.float64)
    for _ in range(iterations):
        A = held(X @ X.T, 2.0 ** 14)
        singular = torch.linalg.eigvalsh(A).clamp_min(0.0).sqrt()
        two = float(singular[-1]) * 1.01
        d_A = e * norm(A) + gamma(n) * norm(X.abs() @ X.T.abs())
        C = held(a * eye + b * A + c * A @ A, 2.0 ** 14)
        d_C = (abs(b) + 2 * c * two * two) * d_A + c * gamma(m) * norm(A.abs() @ A.abs()) + 4 * U * norm(abs(b) * A.abs() + 4 * eye)
        new = held(C @ X, scale) if _ + 1 < iterations else C @ X
        local = d_C * two + (e + gamma(m)) * norm(C.abs() @ X.abs()) + e * norm(new) + grain
        # the perturbation so far goes through this iteration; that of A and C is local
        err = growth(singular) * err + local
        X = new
    return (X.T if tall else X), 1.05 * err


class Case:
    """K workers' matrices of the given shapes with their operands, and the list over them."""

    def __init__(self, shapes, workers=1, param="f32", grad="bf16", copy=None, shift=0, seed=0, **kw):
        g = gen(seed)
        self.shapes, self.param, self.copy_kind, self.K = shapes, param, copy, workers

        def make(kind, size):
            out = []
            for _ in range(workers):
                for r, cc in shapes:
                    flat = torch.empty(r * cc + shift, device=DEV, dtype=T[kind])
                    out.append(flat[shift:].view(r, cc))
                    out[-1].copy_(torch.randn(r, cc, device=DEV, generator=g) * size)
            return out

        self.p, self.g, self.m = make(param, 0.1), make(grad, 1e-3), make("f32", 1e-3)
        self.c = [x.to(T[copy]) for x in self.p] if copy else None
        self.kw = dict(beta=0.95, nesterov=True, weight_decay=0.1, eps=1e-7, iterations=5, products=1) | kw
        self.scale = [1.0 + 0.5 * i for i in range(len(self.p))]
        self.wd = [float(i % 2) for i in range(len(self.p))]
        self.ws = torch.full((B.qsr_muon_workspace_bytes([x.shape for x in self.p], workers, self.kw["products"]),), 255, dtype=torch.uint8, device=DEV)
        self.list = B.MuonList(self.p, self.g, self.m, copies=self.c, wd_scale=self.wd, update_scale=self.scale, workers=workers, workspace=self.ws,
                               stream=stream(), **self.kw)

    def step_and_compare(self, lr=0.02, grad_scale=1.0):
        before = [(x.double(), g.float() * grad_scale, m.clone()) for x, g, m in zip(self.p, self.g, self.m)]
        self.list.qsr_muon_step(lr, grad_scale)
        self.list.qsr_muon_check()
        kw = self.kw
        beta = float(torch.tensor(kw["beta"], dtype=torch.float32))
        omb = float(torch.tensor(1.0 - kw["beta"], dtype=torch.float32))
        for i, (theta, g, m) in enumerate(before):
            if theta.numel() == 0:
                continue
            g, m = g.double(), m.double()
            want = m + omb * (g - m)
            tol = 2 * U * ((g - m).abs() + want.abs()) + TINY["f32"]
            assert not ((self.m[i].double() - want).abs() > tol).any()
            held = self.m[i].double()                      # the direction is taken from the momentum as it is held
            u = g + beta * (held - g) if kw["nesterov"] else held
            X, err = orthogonal64(u, kw["iterations"], kw["eps"], kw["products"])
            s = lr * self.scale[i]
            new = theta - lr * kw["weight_decay"] * self.wd[i] * theta - s * X
            kind = self.param
            off = float(torch.linalg.vector_norm(self.p[i].double() - new))
            bound = s * err * (1 + HALF_ULP[kind]) + (HALF_ULP[kind] + 4 * U) * float(torch.linalg.vector_norm(new.abs() + (s * X).abs())) + TINY[kind] * theta.numel()
            assert off <= bound, (i, tuple(theta.shape), off / bound)
            assert err < 0.5 * float(torch.linalg.vector_norm(X))      # the bound says something
            if self.c is not None:
                if kind == "f32":
                    assert torch.equal(self.c[i], self.p[i].to(self.c[i].dtype))
                ck = self.copy_kind
                assert not ((self.c[i].double() - self.p[i].double()).abs() > (HALF_ULP[ck] + HALF_ULP[kind]) * 1.01 * new.abs().clamp_min(float(err * s)) + TINY[ck] * 2).any()


SHAPES = [(1, 1), (1, 5), (7, 1), (2, 2), (1, 640), (63, 65), (64, 64), (65, 63), (128, 128), (100, 300), (300, 100), (129, 257), (256, 256), (257, 128),
          (512, 260), (320, 700), (64, 512), (512, 65), (63, 500), (129, 64), (128, 512), (130, 300), (600, 513)]


@pytest.mark.parametrize("products", [1, 3])
@pytest.mark.parametrize("shape", SHAPES)
def test_one_matrix(shape, products):
    Case([shape], products=products).step_and_compare()


@pytest.mark.parametrize("param,grad,copy,products", [("f32", "bf16", "bf16", 3), ("f32", "f32", "f16", 1), ("bf16", "bf16", None, 1), ("f16", "f16", None, 1),
                                                      ("bf16", "f32", "f32", 3), ("f32", "f16", None, 3)])
def test_types_and_several_matrices(param, grad, copy, products):
    x = Case([(70, 200), (200, 70), (0, 5), (64, 256), (600, 650), (256, 65)], workers=2, param=param, grad=grad, copy=copy, products=products)
    x.step_and_compare()
    x.step_and_compare(lr=0.01, grad_scale=0.5)
    assert x.list.qsr_muon_launch_count() == 2 * (1 + 18)


@pytest.mark.parametrize("products", [1, 3])
@pytest.mark.parametrize("shape", [(768, 768), (768, 2304), (2304, 768), (1023, 2047), (1537, 77), (1300, 1100), (2600, 2500)])
def test_larger_matrices(shape, products):
    Case([shape], products=products, copy="bf16").step_and_compare()


@pytest.mark.parametrize("kw", [dict(nesterov=False), dict(iterations=1), dict(iterations=2), dict(iterations=6), dict(beta=0.0), dict(weight_decay=0.0), dict(eps=0.0),
                                dict(eps=1.0)])
def test_settings(kw):
    Case([(150, 90), (90, 150)], products=3, **kw).step_and_compare()


@pytest.mark.parametrize("param,copy", [("f32", "bf16"), ("bf16", None)])
@pytest.mark.parametrize("shift", [1, 3, 8])
def test_unaligned(param, copy, shift):
    x = Case([(96, 200), (201, 96), (33, 130)], param=param, copy=copy, shift=shift, products=3)
    x.step_and_compare()


def test_many_small_matrices():
    Case([(5 + i % 40, 3 + 7 * i % 50) for i in range(300)], products=3).step_and_compare()


@pytest.mark.parametrize("products", [1, 3])
def test_low_rank_and_badly_scaled(products):
    x = Case([(200, 300), (200, 300), (200, 300)], products=products, nesterov=False, beta=0.0, grad="f32")
    x.g[0].copy_(torch.randn(200, 2, device=DEV, generator=gen(1)) @ torch.randn(2, 300, device=DEV, generator=gen(2)))
    x.g[1].mul_(1e15)
    x.g[2].zero_()
    x.g[2][17, 200] = 1e-3            # a single element
    x.step_and_compare()


def test_zeros_have_no_update():
    for eps in (1e-7, 0.0):
        x = Case([(70, 90)], weight_decay=0.0, eps=eps)
        x.g[0].zero_()
        x.m[0].zero_()
        before = x.p[0].clone()
        x.list.qsr_muon_step(0.1)
        assert torch.equal(x.p[0], before) and not x.m[0].any()


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_values_that_are_not_finite_stay_in_their_matrix(value):
    clean = Case([(70, 90), (130, 60), (64, 64)], products=3, grad="f32")
    dirty = Case([(70, 90), (130, 60), (64, 64)], products=3, grad="f32")
    dirty.g[1][100, 3] = value
    for x in (clean, dirty):
        x.list.qsr_muon_step(0.1)
    assert torch.equal(clean.p[0], dirty.p[0]) and torch.equal(clean.p[2], dirty.p[2])
    assert torch.isnan(dirty.p[1]).all()


def test_the_same_bits_again():
    runs = []
    for _ in range(2):
        x = Case([(300, 500), (77, 1000)], products=3, copy="bf16")
        for _ in range(3):
            x.list.qsr_muon_step(0.02)
        runs.append(x)
    for name in ("p", "m", "c"):
        assert all(torch.equal(s, t) for s, t in zip(getattr(runs[0], name), getattr(runs[1], name)))


@pytest.mark.parametrize("param,copy", [("f32", "bf16"), ("bf16", None)])
@pytest.mark.parametrize("mode", ["keep", "average", "reset"])
@pytest.mark.parametrize("workers", [1, 3, 4])
def test_round_end(mode, workers, param, copy):
    x = Case([(33, 70), (0, 9), (200, 101)], workers=workers, param=param, copy=copy)
    p0, m0 = [t.clone() for t in x.p], [t.clone() for t in x.m]
    x.list.qsr_muon_sync(mode)
    n = len(x.shapes)

    def mean(ts, j):
        total = ts[j].float()
        for k in range(1, workers):
            total = total + ts[k * n + j].float()
        return total / torch.full_like(total, workers)        # a division by a Python number is a product with its rounded reciprocal
    for k in range(workers):
        for j in range(n):
            i, value = k * n + j, mean(p0, j)
            assert torch.equal(x.p[i], value.to(x.p[i].dtype))
            if copy:
                assert torch.equal(x.c[i], value.to(x.c[i].dtype))
            want = {"keep": m0[i], "average": mean(m0, j), "reset": torch.zeros_like(m0[i])}[mode]
            assert torch.equal(x.m[i], want)


def test_new_gradients():
    x, y = Case([(70, 90), (90, 70)], seed=1), Case([(70, 90), (90, 70)], seed=1)
    other = [torch.randn_like(g) for g in x.g]
    x.list.qsr_muon_set_grads(other)
    for g, o in zip(y.g, other):
        g.copy_(o)
    x.list.qsr_muon_step(0.1)
    y.list.qsr_muon_step(0.1)
    assert all(torch.equal(s, t) for s, t in zip(x.p, y.p))


def test_without_gradients_a_step_is_refused():
    p, m = torch.zeros(8, 8, device=DEV), torch.zeros(8, 8, device=DEV)
    ws = torch.empty(B.qsr_muon_workspace_bytes([(8, 8)]), dtype=torch.uint8, device=DEV)
    x = B.MuonList([p], None, [m], workspace=ws, stream=stream())
    with pytest.raises(B.QsrError) as e:
        x.qsr_muon_step(0.1)
    assert e.value.status == B.QSR_ESTATE
    x.qsr_muon_set_grads([torch.ones(8, 8, device=DEV)])
    x.qsr_muon_step(0.1)
    x.qsr_muon_check()


def test_captured_and_replayed():
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        x, y = Case([(200, 300), (64, 30)], products=3, seed=3), Case([(200, 300), (64, 30)], products=3, seed=3)
        x.list.qsr_muon_step(0.02)                     # outside a graph first
        y.list.qsr_muon_step(0.02)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            x.list.qsr_muon_step(0.02)
            with pytest.raises(B.QsrError) as e:
                x.list.qsr_muon_set_grads(x.g)
            assert e.value.status == B.QSR_ESTATE
        for _ in range(3):
            x.g[0].mul_(-1.1)
            y.g[0].mul_(-1.1)
            graph.replay()
            y.list.qsr_muon_step(0.02)
        side.synchronize()
    assert all(torch.equal(s, t) for s, t in zip(x.p + x.m, y.p + y.m))


def test_two_lists_at_once():
    """Two lists with their own workspaces on two streams."""
    alone = [Case([(500, 700)] * 4, products=3, seed=s) for s in (1, 2)]
    for x in alone:
        for _ in range(5):
            x.list.qsr_muon_step(0.02)
    torch.cuda.synchronize()
    together, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for s, st in zip((1, 2), streams):
        with torch.cuda.stream(st):
            together.append(Case([(500, 700)] * 4, products=3, seed=s))
    torch.cuda.synchronize()
    for _ in range(5):
        for x in together:
            x.list.qsr_muon_step(0.02)
    torch.cuda.synchronize()
    for x, y in zip(alone, together):
        assert all(torch.equal(s, t) for s, t in zip(x.p, y.p))


def short64(u, iterations, short, products):
    """What orthogonal64 gives, with the last `short` iterations on A alone: A <- C (C A), P <- C P and one product P X at the end, rounded
    where the kernels round."""
    X = u / torch.linalg.vector_norm(u)
    tall = X.shape[0] > X.shape[1]
    X = X.T if tall else X
    m, n = X.shape
    e = 2.0 ** -11 * min(1.0, 0.25 + 4.0 / math.sqrt(m * n)) if products == 1 else 2.0 ** -22
    scale = 2.0 ** min(15, math.floor(0.5 * math.log2(m * n)))
    held = (lambda M, at: (M * at).half().double() / at) if products == 1 else (lambda M, at: M)
    gamma = (lambda k: (k / 16 + 1) * 2.0 ** -23) if products == 1 else (lambda k: 12 * 2.0 ** -23 + (k / 64 + 2) * 2.0 ** -24 + 2.0 ** -22)
    norm = lambda M: float(torch.linalg.vector_norm(M))                # noqa: E731
    two = lambda M: float(torch.linalg.matrix_norm(M, 2))              # noqa: E731
    grain = 2.0 ** -25 * 2
    tile = torch.arange(m, device=DEV) // 256
    above = tile[:, None] <= tile[None, :]                            # of a symmetric matrix, the 256 x 256 tiles that are held
    both = lambda M: torch.where(above, M, M.T)                        # noqa: E731
    eye = torch.eye(m, device=DEV, dtype=torch.float64)
    X = held(X, scale)
    err = e * norm(X) + 8 * U * norm(X) + grain
    terms = []                                                         # errors of the products C_j ... C_first, times X
    for k in range(iterations):
        on_x = k <= iterations - short
        if on_x:
            A = held(X @ X.T, 2.0 ** 14)
            d_A = e * norm(A) + gamma(n) * norm(X.abs() @ X.T.abs())
        t = torch.linalg.eigvalsh(A).clamp_min(0.0)
        top, singular = float(t[-1]) * 1.02, t.sqrt()
        # C = f(A): a change of A changes it by at most f's largest divided difference, |b + c (t + t')|
        to_C = max(abs(b), abs(b + 2 * c * top))
        own = c * gamma(m) * norm(A.abs() @ A.abs()) + 4 * U * norm(abs(b) * A.abs() + 4 * eye)
        C = both(held(a * eye + b * A + c * A @ A, 2.0 ** 14))
        own += e * norm(C)
        d_C = to_C * d_A + own
        err *= growth(singular)                                       # X's, through what remains
        if k < iterations - short:
            new = held(C @ X, scale)
            err += d_C * math.sqrt(top) + (e + gamma(m)) * norm(C.abs() @ X.abs()) + e * norm(new) + grain
            X = new
            continue
        if on_x:
            P, at = C, 2.0 ** 14
            terms = [d_C]
        else:
            # what was wrong in P passes C; P's own rounding, C's error times P
            at /= 4
            new = both(held(C @ P, at))
            # with C times P times X taken by its parts: P's earlier errors grow by at most C's norm
            terms = [x * two(C) for x in terms] + [d_C * two(P @ X) / max(two(X), 1e-30), e * norm(new) + gamma(m) * norm(C.abs() @ P.abs())]
            P = new
        if k + 1 < iterations:
            CA = both(held(C @ A, 2.0 ** 14))
            A_next = both(held(C @ CA, 2.0 ** 14))
            d_CA = e * norm(CA) + gamma(m) * norm(C.abs() @ A.abs())
            # A' = q(A), q(t) = t f(t)^2, by q's largest divided difference over A's eigenvalues; then what this step rounds
            grid = t[:, None], t[None, :]
            q = lambda x: x * (a + b * x + c * x * x) ** 2             # noqa: E731
            slope = lambda x: (a + b * x + c * x * x) ** 2 + 2 * x * (a + b * x + c * x * x) * (b + 2 * c * x)     # noqa: E731
            apart = (grid[0] - grid[1]).abs() > 1e-4
            divided = torch.where(apart, (q(grid[0]) - q(grid[1])) / torch.where(apart, grid[0] - grid[1], 1.0), slope((grid[0] + grid[1]) / 2))
            to_A = float(divided.abs().max()) * 1.01
            d_A = to_A * d_A + own * (two(CA) + two(C) * top) + two(C) * d_CA + e * norm(A_next) + gamma(m) * norm(C.abs() @ CA.abs())
            A = A_next
    err += sum(terms) * two(X) + gamma(m) * norm(P.abs() @ X.abs())
    X = P @ X
    return (X.T if tall else X), 1.05 * err


def spread(shape, rank, seed):
    """Entries of a matrix of low rank over weak noise, or a normal one."""
    r, k = shape
    if rank == 0:
        return torch.randn(r, k, device=DEV, generator=gen(seed))
    low = torch.randn(r, rank, device=DEV, generator=gen(seed)) @ torch.randn(rank, k, device=DEV, generator=gen(seed + 1))
    return low + 0.01 * torch.randn(r, k, device=DEV, generator=gen(seed + 2))


@pytest.mark.parametrize("products", [1, 3])
@pytest.mark.parametrize("shape,iterations,rank", [((300, 640), 5, 0), ((640, 300), 5, 0), ((130, 2000), 4, 0), ((2000, 130), 4, 0), ((520, 1100), 6, 0),
                                                   ((65, 5000), 8, 0), ((700, 1500), 5, 0), ((1500, 700), 16, 0), ((300, 900), 5, 20), ((900, 300), 5, 3)])
def test_long_matrices(shape, iterations, rank, products):
    """Sides that differ by two or more and four iterations or more: the last three (of four, two) on m x m matrices."""
    g = spread(shape, rank, 5)
    p, m = torch.zeros(shape, device=DEV), torch.zeros(shape, device=DEV)
    ws = torch.empty(B.qsr_muon_workspace_bytes([shape], 1, products), dtype=torch.uint8, device=DEV)
    x = B.MuonList([p], [g], [m], beta=0.0, nesterov=False, eps=0.0, iterations=iterations, products=products, update_scale=[1.0], workspace=ws, stream=stream())
    x.qsr_muon_step(1.0)
    x.qsr_muon_check()
    assert x.qsr_muon_launch_count() == 3 + 3 * iterations + 1
    short = min(3, iterations - 2)
    want, err = short64(g.double(), iterations, short, products)
    off, size = float(torch.linalg.vector_norm(p.double() + want)), float(torch.linalg.vector_norm(want))
    assert off <= err + U * size
    if iterations <= (8 if products == 3 else 6) and (products == 3 or rank == 0):
        assert err < 0.5 * size                                       # the bound says something; it grows with each iteration


def test_long_matrices_beside_others():
    """A list's matrices go through the same launches, long or not, and each is what it is alone."""
    shapes = [(300, 640), (500, 600), (700, 300), (30, 20), (640, 1400)]
    for products in (1, 3):
        together = Case(shapes, products=products, seed=9)
        alone = []
        for i in range(len(shapes)):
            ws = torch.empty(B.qsr_muon_workspace_bytes([shapes[i]], 1, products), dtype=torch.uint8, device=DEV)
            p, m = together.p[i].clone(), together.m[i].clone()
            x = B.MuonList([p], [together.g[i]], [m], wd_scale=[together.wd[i]], update_scale=[together.scale[i]], workspace=ws, stream=stream(), **together.kw)
            for _ in range(2):
                x.qsr_muon_step(0.02)
            x.qsr_muon_check()
            alone.append((p, m))
        for _ in range(2):
            together.list.qsr_muon_step(0.02)
        together.list.qsr_muon_check()
        for (p, m), q, mm in zip(alone, together.p, together.m):
            assert torch.equal(p, q) and torch.equal(m, mm)


def test_offsets_beyond_32_bits():
    """512 copies of one 2048 x 2048 matrix below one another, 2^31 elements: the orthogonal factor of a stack is the stack of the
    factors over sqrt(512), up to the polynomial, which sees the same A."""
    n, side = 512, 2048
    y = torch.randn(side, side, device=DEV, generator=gen(1)).bfloat16()
    g = y.repeat(n, 1)
    p, m = torch.zeros(n * side, side, device=DEV, dtype=torch.bfloat16), torch.zeros(n * side, side, device=DEV)
    ws = torch.empty(B.qsr_muon_workspace_bytes([p.shape]), dtype=torch.uint8, device=DEV)
    x = B.MuonList([p], [g], [m], beta=0.0, update_scale=[n ** 0.5], workspace=ws, stream=stream())
    x.qsr_muon_step(1.0)
    x.qsr_muon_check()
    want, err = orthogonal64(y.double(), 5, 0.0, 1)
    for part in (0, 255, 511):
        got = -p[part * side:(part + 1) * side].double()
        assert float(torch.linalg.vector_norm(got - want)) <= err + 2.0 ** -8 * float(torch.linalg.vector_norm(want))
    assert torch.equal(m[-side:], y.float())


@pytest.mark.parametrize("products", [1, 3])
@pytest.mark.parametrize("shape", [(64, 64), (60, 200), (300, 200), (500, 130), (1, 7)])
def test_the_size_of_a_gradient_does_not_matter(shape, products):
    """Without eps, a gradient times a power of two has the same update, bit for bit, as long as fp32 holds its elements: from 2^-140 (whole numbers
    times that; the norm's reciprocal is beyond fp32) to 2^120."""
    g0 = torch.randint(-8, 9, shape, device=DEV, generator=gen(7)).float()
    g0.view(-1)[0] = 5.0
    theta = torch.randn(shape, device=DEV, generator=gen(8))
    results = []
    for power in (0, -140, -127, -100, -62, 61, 100, 120):
        p, m, g = theta.clone(), torch.zeros(shape, device=DEV), torch.ldexp(g0.double(), torch.tensor(power, device=DEV)).float()
        ws = torch.empty(B.qsr_muon_workspace_bytes([shape], 1, products), dtype=torch.uint8, device=DEV)
        x = B.MuonList([p], [g], [m], beta=0.0, nesterov=False, eps=0.0, products=products, workspace=ws, stream=stream())
        x.qsr_muon_step(0.1)
        x.qsr_muon_check()
        assert torch.equal(m, g)
        results.append(p)
    assert not torch.equal(results[0], theta)
    assert all(torch.equal(r, results[0]) for r in results)


def plain64(u, iterations):
    X = u / torch.linalg.vector_norm(u)
    X = X.T if u.shape[0] > u.shape[1] else X
    for _ in range(iterations):
        A = X @ X.T
        X = a * X + (b * A + c * A @ A) @ X
    return X.T if u.shape[0] > u.shape[1] else X


def held64(u, iterations):
    """The iterations in binary64 with X, A and C in fp16, all of them on X."""
    held = lambda M, at: (M * at).half().double() / at                 # noqa: E731
    X = u / torch.linalg.vector_norm(u)
    X = X.T if u.shape[0] > u.shape[1] else X
    m, n = X.shape
    scale, eye = 2.0 ** min(15, math.floor(0.5 * math.log2(m * n))), torch.eye(m, device=DEV, dtype=torch.float64)
    X = held(X, scale)
    for _ in range(iterations):
        A = held(X @ X.T, 2.0 ** 14)
        X = held(held(a * eye + b * A + c * A @ A, 2.0 ** 14) @ X, scale)
    return X.T if u.shape[0] > u.shape[1] else X


@pytest.mark.parametrize("products", [1, 3])
@pytest.mark.parametrize("shape,iterations,rank", [((300, 900), 5, 20), ((900, 300), 5, 3), ((300, 577), 5, 60), ((300, 577), 5, 100), ((256, 1024), 6, 20), ((700, 1500), 5, 0),
                                                   ((130, 2000), 5, 10), ((130, 2000), 4, 3), ((150, 600), 4, 40), ((300, 576), 5, 60)])
def test_long_matrices_are_as_near_as_others(shape, iterations, rank, products):
    """Low rank over weak noise, whose small singular values five iterations raise by hundreds, and with them whatever was rounded.  The last
    iterations of long matrices go through A, which holds those values by their squares; that may not show.  With one product the roundings
    are those of the iterations on X in fp16 (emulated here; another set of them gives within a few per cent the same), and three
    more of A and C: half as much again is allowed, and as much again with four iterations, which raise small values less and so
    leave these a larger share.  With three products they are 2^-22 instead of fp32's 2^-24: four times what fp32 products leave."""
    u = spread(shape, rank, 11)
    p, m = torch.zeros(shape, device=DEV), torch.zeros(shape, device=DEV)
    ws = torch.empty(B.qsr_muon_workspace_bytes([shape], 1, products), dtype=torch.uint8, device=DEV)
    x = B.MuonList([p], [u], [m], beta=0.0, nesterov=False, eps=0.0, iterations=iterations, products=products, update_scale=[1.0], workspace=ws, stream=stream())
    x.qsr_muon_step(1.0)
    x.qsr_muon_check()
    want = plain64(u.double(), iterations)
    off = lambda X: float(torch.linalg.vector_norm(X.double() - want) / torch.linalg.vector_norm(want))       # noqa: E731
    limit = (1.5 if iterations > 4 else 2.0) * off(held64(u.double(), iterations)) if products == 1 else 4.0 * off(plain64(u, iterations))
    assert off(-p) <= limit


def cut64(u, iterations):
    """The iterations in binary64 with X, A and C as sums of two fp16 numbers, and every product too small by what three products may cut off at
    most: all errors in one direction, whereas those of the kernels fall both ways where sums are rounded."""
    def held(M, at):
        hi = (M * at).half().double()
        return (hi + (M * at - hi).half().double()) / at

    def product(L, R):
        P = L @ R
        return P - torch.sign(P) * (12 * 2.0 ** -23 + (L.shape[1] / 64 + 2) * 2.0 ** -24 + 2.0 ** -22) * (L.abs() @ R.abs())

    X = u / torch.linalg.vector_norm(u)
    X = X.T if u.shape[0] > u.shape[1] else X
    m, n = X.shape
    scale, eye = 2.0 ** min(15, math.floor(0.5 * math.log2(m * n))), torch.eye(m, device=DEV, dtype=torch.float64)
    X = held(X, scale)
    for _ in range(iterations):
        A = held(product(X, X.T), 2.0 ** 14)
        X = held(product(held(a * eye + b * A + c * product(A, A), 2.0 ** 14), X), scale)
    return X.T if u.shape[0] > u.shape[1] else X


@pytest.mark.parametrize("products", [1, 3])
@pytest.mark.parametrize("shape,iterations", [((1500, 700), 16), ((128, 128), 16), ((700, 900), 12), ((300, 900), 9)])
def test_many_iterations(shape, iterations, products):
    """The polynomial does not converge, so that each iteration raises what was rounded before: compared with the same roundings in binary64 (half
    as much again, since others than those give within a few per cent the same), or with the most that can be cut off."""
    u = spread(shape, 0, 13)
    p, m = torch.zeros(shape, device=DEV), torch.zeros(shape, device=DEV)
    ws = torch.empty(B.qsr_muon_workspace_bytes([shape], 1, products), dtype=torch.uint8, device=DEV)
    x = B.MuonList([p], [u], [m], beta=0.0, nesterov=False, eps=0.0, iterations=iterations, products=products, update_scale=[1.0], workspace=ws, stream=stream())
    x.qsr_muon_step(1.0)
    x.qsr_muon_check()
    want = plain64(u.double(), iterations)
    off = lambda X: float(torch.linalg.vector_norm(X.double() - want) / torch.linalg.vector_norm(want))       # noqa: E731
    limit = 1.5 * off(held64(u.double(), iterations)) if products == 1 else off(cut64(u.double(), iterations))
    assert off(-p) <= limit < 0.05
