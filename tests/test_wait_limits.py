"""Waits inside kernels that have a limit: what is reported, and what is left behind, where one runs out."""
import os
import re

import pytest
import torch

import paper_2310_14423_b200
from paper_2310_14423_b200 import binding as B

DEV = "cuda:0"
CSRC = os.path.join(os.path.dirname(paper_2310_14423_b200.__file__), "csrc")


def body(source, kernel):
    """Text of a kernel's definition."""
    text = open(os.path.join(CSRC, source)).read()
    return re.search(r"\n" + kernel + r"\(.*?\n}\n", text, re.S).group(0)


def test_the_product_kernel_looks_for_waits_that_ran_out_when_all_its_warps_are_done():
    """A warp may give up after every other one has finished, so the flag is read behind the barrier that all of them reach."""
    text = body("muon.cu", "product_kernel")
    assert text.count("*p.late = 1u") == 1
    assert text.rindex("pair_sync();") < text.index("*p.late = 1u")


@pytest.fixture
def no_patience():
    B.qsr_debug_copy_patience(0)
    yield
    B.qsr_debug_copy_patience(-1)


# widths with one row at a time and two, whole granules and not; one row for each block, several, and more than its ring holds
@pytest.mark.gpu
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("R,N", [(1, 3136), (300, 4096), (2000, 4101), (450, 8192), (149, 8185)])
def test_no_number_passes_for_a_gradient_where_a_wait_ran_out(R, N, kind, no_patience):
    pad = -N % 8
    rows = lambda: torch.randn(R, N + pad, device=DEV).to(kind)[:, :N]             # noqa: E731; aligned, whatever the width
    x, dy, w = rows(), rows(), torch.randn(N, device=DEV)
    mean, rstd = x.float().mean(1), 1.0 / x.float().std(1, correction=0)
    ws = torch.empty(B.qsr_layer_norm_workspace_bytes(R, N), dtype=torch.uint8, device=DEV)

    def gradients(with_dx):
        dx, dw, db = rows(), torch.zeros_like(w), torch.zeros_like(w)
        B.qsr_layer_norm_grad(x, dy, mean, rstd, d_x=dx if with_dx else None, weight=w, d_weight=dw, d_bias=db, workspace=ws,
                              stream=torch.cuda.current_stream().cuda_stream)
        return (dx, dw, db) if with_dx else (dw, db)

    for with_dx in (True, False):
        assert all(torch.isnan(t).all() for t in gradients(with_dx))
    B.qsr_debug_copy_patience(-1)
    assert all(torch.isfinite(t).all() for t in gradients(True))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("R,N", [(2400, 2048), (2400, 3001), (5000, 1032), (600, 8192), (296, 16384)])
def test_no_number_passes_for_a_row_where_a_wait_ran_out(R, N, kind, no_patience):
    pad = -N % 8
    x = torch.randn(R, N + pad, device=DEV).to(kind)[:, :N]

    def forward():
        y, mean, rstd = torch.zeros(R, N + pad, device=DEV, dtype=kind)[:, :N], torch.zeros(R, device=DEV), torch.zeros(R, device=DEV)
        B.qsr_layer_norm(x, y, mean=mean, rstd=rstd, stream=torch.cuda.current_stream().cuda_stream)
        return y, mean, rstd

    assert all(torch.isnan(t).all() for t in forward())
    B.qsr_debug_copy_patience(-1)
    assert all(torch.isfinite(t).all() for t in forward())
