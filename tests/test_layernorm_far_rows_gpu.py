"""Layer norm of rows far from zero, and of rows of one value: nothing of the mean's rounding, which grows with the mean and not with the row's
spread, is left in the result."""
import pytest
import torch

from paper_2310_14423_b200 import binding as B
from test_layernorm_gpu import DEV, EPS, U, chain, close, inputs, rounded, stream
from test_layernorm_loops_gpu import laid_out

pytestmark = pytest.mark.gpu


def bounds(x, w, b):
    """The formula in binary64, and what fp32 may be off: first a mean, off by d0; what is left of x then, a, has a mean of its own that is taken off
    too where the row is further from zero than four standard deviations (64 where x has 16 bits, whose own roundings are that much
    larger), off by (chain + 4) u mean(a); each subtraction rounds by u a."""
    limit = 4.04 if x.dtype == torch.float32 else 64.7                  # nearer rows may or may not be corrected
    x, w, b = x.double(), w.double(), b.double()
    N = x.shape[1]
    mean = x.mean(1, keepdim=True)
    off = x - mean
    var = off.square().mean(1, keepdim=True)
    rstd = (var + EPS).rsqrt()
    y = off * rstd * w + b
    d0 = (chain(N) + 1) * U * x.abs().mean(1, keepdim=True)
    a = off.abs() + d0
    far = mean.abs() * rstd > limit
    d1 = torch.where(far, (chain(N) + 4) * U * a.mean(1, keepdim=True), d0)
    d_var = (chain(N) + 6) * U * (var + d1.square()) + d1.square() + 4 * U * (off.abs() * a).mean(1, keepdim=True)
    r_rel = 0.5 * d_var / (var + EPS) + 3 * U
    tol = (off * rstd * w).abs() * (r_rel + 4 * U) + w.abs() * rstd * (d1 + 2 * U * a) + 2 * U * y.abs()
    return mean, rstd, y, d1, r_rel * rstd, tol


# the kernels: a warp and a block a row, rows of any length; warps and blocks that stay
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("how", ["aligned", "odd"])
@pytest.mark.parametrize("R,N", [(40, 5), (40, 100), (40, 768), (40, 1000), (40, 2045), (40, 5000), (40, 8192), (16, 40000), (16, 17000), (9600, 768), (9501, 1000), (40000, 60),
                                 (2400, 2045), (600, 8193), (300, 12000)])
def test_rows_far_from_zero(R, N, how, kind):
    x, _, w, b = inputs(R, N, "f32", "f32", R + N)
    level = torch.tensor([0.0, 3.0, -10.0, 100.0, 1000.0, -4096.3, 30000.7, 1e6], device=DEV).repeat(-(-R // 8))[:R, None]
    x = x + level
    x[1::3] = level[1::3] + 1e-3 * torch.arange(x[1::3].shape[0], device=DEV)[:, None]        # one value all along
    x = x.to({"f32": torch.float32, "bf16": torch.bfloat16}[kind])
    xs, y, mean, rstd = laid_out(x, how), laid_out(torch.zeros_like(x), how), torch.empty(R, device=DEV), torch.empty(R, device=DEV)
    B.qsr_layer_norm(xs, y, weight=w, bias=b, mean=mean, rstd=rstd, eps=EPS, stream=stream())
    m64, r64, y64, dm, dr, tol = bounds(x, w, b)
    close(mean, m64[:, 0], dm[:, 0] + U * m64[:, 0].abs())
    close(rstd, r64[:, 0], dr[:, 0])
    close(y, y64, rounded(tol, y64, kind))
    B.qsr_layer_norm(xs, xs, weight=w, bias=b, eps=EPS, stream=stream())
    assert torch.equal(xs, y)                                         # in place


def test_more_far_rows_than_a_block_remembers():
    """1184 blocks that stay take 256 rows and more each, all of them far from zero."""
    R, N = 1184 * 260 + 7, 1032
    x, _, w, b = inputs(64, N, "f32", "f32", 1)
    x = (x + torch.linspace(50.0, 900.0, 64, device=DEV)[:, None]).bfloat16()
    _, _, y64, _, _, tol = bounds(x, w, b)
    many = x.repeat(-(-R // 64), 1)[:R]
    mean, rstd = torch.empty(R, device=DEV), torch.empty(R, device=DEV)
    B.qsr_layer_norm(many, many, weight=w, bias=b, mean=mean, rstd=rstd, eps=EPS, stream=stream())
    close(many[:64], y64, rounded(tol, y64, "bf16"))
    for t in (many, mean, rstd):
        assert torch.equal(t[64:], t[:-64])                           # rows 64 apart are the same


@pytest.mark.parametrize("R,N", [(10, 1000), (10, 777), (10, 5003), (10, 20001), (9600, 999), (2400, 2047)])
def test_a_row_of_one_value_is_the_bias(R, N):
    """What is left of the value after its mean (chain u of it at most) has a mean that is off by chain u of itself: (chain u)^2 |x| rstd in all."""
    value = torch.linspace(-1000.0, 1000.0, R, device=DEV)[:, None]
    x = laid_out(value.expand(R, N).contiguous(), "aligned")
    w, b, y = torch.full((N,), 1.5, device=DEV), torch.linspace(-1.0, 1.0, N, device=DEV), laid_out(torch.zeros(R, N, device=DEV), "aligned")
    B.qsr_layer_norm(x, y, weight=w, bias=b, eps=EPS, stream=stream())
    tol = 1.5 * EPS ** -0.5 * ((chain(N) + 4) * U) ** 2 * 1000.0 + 2 * U
    assert float((y - b).abs().max()) <= tol
