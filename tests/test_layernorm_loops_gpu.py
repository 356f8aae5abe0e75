"""Layer norm over so many rows that a warp, a group of threads or a block takes several, one after the other: rows loaded ahead, pointers moved on,
buffers in turn, sums over rows that stay in registers.  Compared with binary64; tolerances as in test_layernorm_gpu, but for the sums over
rows, whose longest chain of additions is counted here."""
import math

import pytest
import torch

from paper_2310_14423_b200 import binding as B
from test_layernorm_gpu import DEV, EPS, T, U, backward64, close, forward64, inputs, rounded, stream

pytestmark = pytest.mark.gpu
MULTIPROCESSORS = 148


def laid_out(x, how):
    """x in a buffer whose other elements are not numbers: rows aligned to eight elements ("aligned"; the buffer ends with the last row), or of
    an odd stride behind an odd start ("odd")."""
    R, N = x.shape
    stride, shift = (N + -N % 8, 0) if how == "aligned" else (N + 1 + N % 2, 1)
    flat = torch.full((shift + (R - 1) * stride + N,), math.nan, device=DEV, dtype=x.dtype)
    out = flat.as_strided((R, N), (stride, 1), shift)
    out.copy_(x)
    return out


def column_chain(R, N):
    """Additions that a column's sum goes through at most: a group of threads adds its rows, a block its groups, sixteen threads the blocks' sums
    one after the other (ten each, at most), and then these.  Groups are as launch_backward makes them; rows longer than 8192 have blocks
    of 256 granules instead."""
    granules = -(-N // 8)
    if granules > 1024:
        blocks, groups = min(max(1, 2 * MULTIPROCESSORS // -(-granules // 256)), R, MULTIPROCESSORS), 1
    else:
        lanes = 1 << (granules - 1).bit_length() if granules <= 32 else -(-granules // 32) * 32
        groups = max(1, 512 // lanes if lanes <= 32 else min(768 // lanes, 15))
        blocks = min(-(-R // groups), MULTIPROCESSORS)
    return -(-R // (blocks * groups)) + groups + -(-blocks // 16) + 16


# 592 blocks of 256 threads stay from two rows for each group of threads on: 9472 rows for a warp a row, more for narrower rows
MANY = [(9471, 768), (9472, 255), (9473, 768), (12544, 768), (9501, 1000), (9600, 1024), (30000, 257), (19000, 100), (40000, 64), (151553, 16), (303105, 5), (310000, 8)]


@pytest.mark.parametrize("kind,wkind", [("f32", "f32"), ("bf16", "f32"), ("f16", "f16")])
@pytest.mark.parametrize("how", ["aligned", "odd"])
@pytest.mark.parametrize("R,N", MANY)
def test_forward_over_many_rows(R, N, how, kind, wkind):
    x, _, w, b = inputs(R, N, kind, wkind, R + N)
    xs, y, mean, rstd = laid_out(x, how), laid_out(torch.zeros_like(x), how), torch.empty(R, device=DEV), torch.empty(R, device=DEV)
    around = y.as_strided((R - 1, y.stride(0) - N), (y.stride(0), 1), y.storage_offset() + N)
    B.qsr_layer_norm(xs, y, weight=w, bias=b, mean=mean, rstd=rstd, eps=EPS, stream=stream())
    m64, r64, y64, dm, dr, tol = forward64(x, w, b)
    close(mean, m64[:, 0], dm[:, 0] + U * m64[:, 0].abs())
    close(rstd, r64[:, 0], dr[:, 0])
    close(y, y64, rounded(tol, y64, kind))
    assert torch.isnan(around).all()                                  # nothing but the rows was written
    dirty = [R // 3, R - 1]
    xs[dirty[0], N - 1], xs[dirty[1], 0] = math.nan, math.inf
    B.qsr_layer_norm(xs, xs, weight=w, bias=b, eps=EPS, stream=stream())      # in place, and what is not finite stays in its row
    clean = torch.ones(R, dtype=torch.bool, device=DEV)
    clean[dirty] = False
    assert torch.equal(xs[clean], y[clean]) and torch.isnan(xs[dirty]).all()
    bare = torch.empty(R, N, device=DEV, dtype=T[kind])
    B.qsr_layer_norm(x, bare, eps=EPS, stream=stream())              # without weight, bias and statistics
    _, _, y64, _, _, tol = forward64(x, None, None)
    close(bare, y64, rounded(tol, y64, kind))


# several rows for each group of threads, an uneven number; wide rows that a block takes; rows of more than 8192
SEVERAL = [(3700, 768), (12544, 768), (7500, 256), (4000, 1000), (2000, 1025), (1000, 3000), (20000, 100), (40000, 40), (240000, 7), (76000, 1), (450, 4097), (460, 6200), (450, 8185),
           (300, 8193), (299, 16385), (200, 33000)]


@pytest.mark.parametrize("kind,wkind", [("f32", "f32"), ("bf16", "f32"), ("f16", "f16")])
@pytest.mark.parametrize("how", ["aligned", "odd"])
@pytest.mark.parametrize("R,N", SEVERAL)
def test_backward_over_several_rows_each(R, N, how, kind, wkind):
    x, dy, w, _ = inputs(R, N, kind, wkind, R + N + 1)
    m64, r64 = forward64(x, None, None)[:2]
    mean, rstd = m64[:, 0].float(), r64[:, 0].float()
    xs, dys, dx = laid_out(x, how), laid_out(dy, how), laid_out(torch.zeros_like(x), how)
    around = dx.as_strided((R - 1, dx.stride(0) - N), (dx.stride(0), 1), dx.storage_offset() + N)
    dw, db = torch.empty_like(w), torch.empty_like(w)
    ws = torch.full((B.qsr_layer_norm_workspace_bytes(R, N),), 255, dtype=torch.uint8, device=DEV)
    B.qsr_layer_norm_grad(xs, dys, mean, rstd, d_x=dx, weight=w, d_weight=dw, d_bias=db, workspace=ws, stream=stream())
    dx64, dw64, db64, tx, _, _ = backward64(x, dy, mean, rstd, w)
    close(dx, dx64, rounded(tx, dx64, kind))
    hat = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    depth = column_chain(R, N)
    close(dw, dw64, rounded((depth + 3) * U * (dy.double() * hat).abs().sum(0), dw64, wkind))      # a subtraction and two products more
    close(db, db64, rounded(depth * U * dy.double().abs().sum(0), db64, wkind))
    assert torch.isnan(around).all()
    # the sums by themselves, one by one, and the rows by themselves: the same bits
    dw2, db2, dx2 = torch.empty_like(w), torch.empty_like(w), laid_out(torch.zeros_like(x), how)
    ws.fill_(255)
    B.qsr_layer_norm_grad(xs, dys, mean, rstd, weight=w, d_weight=dw2, workspace=ws, stream=stream())
    B.qsr_layer_norm_grad(xs, dys, mean, rstd, weight=w, d_bias=db2, workspace=ws, stream=stream())
    B.qsr_layer_norm_grad(xs, dys, mean, rstd, d_x=dx2, weight=w, stream=stream())
    assert torch.equal(dw2, dw) and torch.equal(db2, db) and torch.equal(dx2, dx)
    # in place of either operand, rows loaded ahead included
    for over in ("x", "dy"):
        a, d = laid_out(x, how) if over == "x" else xs, laid_out(dy, how) if over == "dy" else dys
        B.qsr_layer_norm_grad(a, d, mean, rstd, d_x=a if over == "x" else d, weight=w, d_weight=dw2, d_bias=db2, workspace=ws, stream=stream())
        assert torch.equal(a if over == "x" else d, dx) and torch.equal(dw2, dw) and torch.equal(db2, db)
    # a row that is not finite: no other row, and the sums of its columns
    row = 2 * R // 3
    xs[row, N - 1] = math.nan
    B.qsr_layer_norm_grad(xs, dys, mean, rstd, d_x=dx2, weight=w, d_weight=dw2, d_bias=db2, workspace=ws, stream=stream())
    clean = torch.arange(R, device=DEV) != row
    assert torch.equal(dx2[clean], dx[clean]) and torch.isnan(dx2[row]).all()
    assert torch.isnan(dw2[N - 1]) and torch.equal(dw2[:N - 1], dw[:N - 1]) and torch.equal(db2, db)


@pytest.mark.parametrize("R,N,stride", [((1 << 21) + 1001, 760, 1032), (300_001, 8184, 8192), (66_001, 33000, 33001)])
def test_offsets_beyond_32_bits(R, N, stride):
    """Matrices of more than 2^31 elements: their last rows are what they are by themselves (the warps, blocks and sums that take them
    are others, but a row's arithmetic is the same)."""
    last = 700
    x, dy, w, b = inputs(last, N, "bf16", "f32", 5)
    big = lambda: torch.empty(R * stride, device=DEV, dtype=torch.bfloat16).as_strided((R, N), (stride, 1))        # noqa: E731
    xs, out = big(), big()
    xs.zero_()
    xs[-last:] = x
    mean, rstd = torch.empty(R, device=DEV), torch.empty(R, device=DEV)
    B.qsr_layer_norm(xs, out, weight=w, bias=b, mean=mean, rstd=rstd, eps=EPS, stream=stream())
    m64, r64, y64, dm, dr, tol = forward64(x, w, b)
    close(mean[-last:], m64[:, 0], dm[:, 0] + U * m64[:, 0].abs())
    close(rstd[-last:], r64[:, 0], dr[:, 0])
    close(out[-last:], y64, rounded(tol, y64, "bf16"))
    assert torch.equal(out[0], b.bfloat16()) and torch.equal(out[R // 2], b.bfloat16())
    dys = xs                                                          # gradients by themselves: x and d_y may be one matrix
    dw, db = torch.empty_like(w), torch.empty_like(w)
    ws = torch.empty(B.qsr_layer_norm_workspace_bytes(R, N), dtype=torch.uint8, device=DEV)
    B.qsr_layer_norm_grad(xs, dys, mean, rstd, d_x=out, weight=w, d_weight=dw, d_bias=db, workspace=ws, stream=stream())
    dx64, dw64, db64, tx, _, _ = backward64(x, x, mean[-last:], rstd[-last:], w)
    close(out[-last:], dx64, rounded(tx, dx64, "bf16"))
    hat = (x.double() - mean[-last:].double()[:, None]) * rstd[-last:].double()[:, None]
    depth = last + 512 + 26                                           # all other rows add zeros
    close(dw, dw64, rounded((depth + 3) * U * (x.double() * hat).abs().sum(0), dw64, "f32"))
    close(db, db64, rounded(depth * U * x.double().abs().sum(0), db64, "f32"))
    assert not out[0].any() and not out[R // 2].any()
