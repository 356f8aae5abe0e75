"""The embedding lookup and its gradient on the GPU.  A lookup is one product and one rounding, compared bit for bit; a gradient is a
sum in fp32 of as many terms as the token occurs, then one product and one rounding."""
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


def stream():
    return torch.cuda.current_stream().cuda_stream


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def draw(R, V, seed, how="zipf"):
    g = gen(seed)
    if how == "zipf":
        t = (torch.exp(torch.rand(R, device=DEV, generator=g, dtype=torch.float64) * math.log(V + 1.0)) - 1.0).long().clamp_(0, V - 1)
        return torch.where(torch.rand(R, device=DEV, generator=g) < 0.1, torch.full_like(t, -1), t)
    if how == "same":
        return torch.full((R,), V - 1, device=DEV, dtype=torch.int64)
    if how == "absent":
        return torch.full((R,), -5, device=DEV, dtype=torch.int64)
    if how == "outside":                   # some beyond the vocabulary, far beyond, and the extremes of the type
        t = torch.randint(0, V, (R,), device=DEV, generator=g)
        t[::3] = V
        t[1::7] = 1 << 40
        t[2::11] = torch.iinfo(torch.int64).min
        return t
    return torch.randint(0, V, (R,), device=DEV, generator=g)


def around(R, N, kind, pad=0, shift=0, value=7.0):
    flat = torch.full((R * (N + pad) + shift,), value, device=DEV, dtype=T[kind])
    return flat, flat[shift:].view(R, N + pad)[:, :N]


@pytest.mark.parametrize("table,out", [("f32", "bf16"), ("bf16", "bf16"), ("f16", "f32"), ("f32", "f32"), ("bf16", "f16")])
@pytest.mark.parametrize("R,V,N", [(1, 1, 1), (5, 3, 7), (8, 100, 8), (33, 10, 64), (64, 1000, 129), (300, 50, 768), (9, 7, 1024), (3, 4, 5001)])
def test_lookup(R, V, N, table, out):
    w = torch.randn(V, N, device=DEV, generator=gen(1)).to(T[table])
    for how, scale in (("zipf", 1.0), ("uniform", 27.7), ("outside", -0.3)):
        t = draw(R, V, R + N, how)
        y = torch.full((R, N), 5.0, device=DEV, dtype=T[out])
        B.qsr_embed(w, t, y, scale=scale, stream=stream())
        want = w.float()[t.clamp(0, V - 1)] * torch.tensor(scale, dtype=torch.float32, device=DEV)
        want = torch.where((t >= 0)[:, None], want, 0.0)
        want = torch.where((t >= V)[:, None], math.nan, want).to(T[out])
        assert torch.equal(torch.isnan(y), torch.isnan(want)) and torch.equal(y.nan_to_num(), want.nan_to_num())


def check_grad(d, t, V, scale, kind, accumulate=False, into=None, lay=(0, 0)):
    R, N = d.shape
    g0 = torch.randn(V, N, device=DEV, generator=gen(9)).to(T[kind])
    flat, out = around(V, N, kind, *lay)
    out.copy_(g0)
    before = flat.clone()
    ws = torch.full((B.qsr_embed_workspace_bytes(R, V, N),), 255, dtype=torch.uint8, device=DEV)
    B.qsr_embed_grad(d, t, out, scale=scale, accumulate=accumulate, workspace=ws, stream=stream())
    some = (t >= 0) & (t < V)
    want = torch.zeros(V, N, device=DEV, dtype=torch.float64).index_put_((t[some],), d[some].double(), accumulate=True)
    size = torch.zeros(V, N, device=DEV, dtype=torch.float64).index_put_((t[some],), d[some].double().abs(), accumulate=True)
    count = torch.bincount(t[some], minlength=V).double()[:, None]
    s32 = float(torch.tensor(scale, dtype=torch.float32))
    want, tol = want * s32, (count + 8) * U * size * abs(s32)
    if accumulate:
        want = want + g0.double()
        tol = tol + 2 * U * want.abs()
    tol = tol * 1.01 + HALF_ULP[kind] * want.abs() + TINY[kind]
    assert not (((out.double() - want).abs() > tol).any()), float(((out.double() - want).abs() / tol).max())
    if accumulate:
        assert torch.equal(out[count[:, 0] == 0], g0[count[:, 0] == 0])
    else:
        assert not out[count[:, 0] == 0].any()
    result = out.clone()
    out.fill_(7.0)
    flat2 = before.clone()
    flat2[lay[1]:].view(V, N + lay[0])[:, :N].fill_(7.0)
    assert torch.equal(flat, flat2)               # nothing around the rows was written
    out.copy_(g0)
    ws.fill_(0)
    B.qsr_embed_grad(d, t, out, scale=scale, accumulate=accumulate, workspace=ws, stream=stream())
    assert torch.equal(out, result)               # the same bits again
    return result


@pytest.mark.parametrize("kind,out", [("f32", "bf16"), ("bf16", "bf16"), ("f16", "f32"), ("f32", "f16")])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("R,V,N", [(1, 1, 1), (2, 5, 8), (8, 3, 7), (33, 1000, 40), (700, 20, 129), (2048, 1000, 128), (5000, 4, 64), (1000, 300, 1030), (20011, 5003, 24)])
def test_gradient(R, V, N, kind, out, accumulate):
    d = torch.randn(R, N, device=DEV, generator=gen(R)).to(T[out])
    for how, scale in (("zipf", 1.0), ("uniform", 11.3)):
        check_grad(d, draw(R, V, R + V, how), V, scale, kind, accumulate)


@pytest.mark.parametrize("how", ["same", "absent", "outside"])
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient_of_unusual_tokens(how, accumulate):
    for R, V, N in ((1, 9, 16), (64, 5, 24), (1000, 70, 33), (9000, 3, 16)):
        d = torch.randn(R, N, device=DEV, generator=gen(R)).bfloat16()
        check_grad(d, draw(R, V, R, how), V, 2.0, "f32", accumulate)


@pytest.mark.parametrize("V", [1 << 10, (1 << 10) + 1, (1 << 20) - 1, 1 << 20, (1 << 21) + 5])
def test_vocabularies_of_several_digits(V):
    R, N = 5000, 1
    t = draw(R, V, 3, "uniform")
    t[:10] = torch.arange(V - 10, V, device=DEV)
    t[10:20] = V - 1
    check_grad(torch.randn(R, N, device=DEV, generator=gen(4)), t, V, 1.0, "f32")


def test_many_rows():
    """More rows than the sort's blocks take at 2048 each, and runs over hundreds of chunks."""
    R, V, N = 700_001, 900, 8
    check_grad(torch.randn(R, N, device=DEV, generator=gen(4)).bfloat16(), draw(R, V, 5), V, 1.0, "f32")


def test_rows_are_added_in_order():
    """A sum whose value depends on the order: large terms that cancel around small ones.  In row order within a chunk the
    small ones between them are lost or kept just as fp32 addition does it."""
    d = torch.tensor([2.0 ** 24, 1.0, -2.0 ** 24, 1.0, 3.0], device=DEV)[:, None].repeat(1, 3).contiguous()
    t = torch.tensor([2, 2, 2, 2, 0], device=DEV)
    got = torch.empty(4, 3, device=DEV)
    ws = torch.empty(B.qsr_embed_workspace_bytes(5, 4, 3), dtype=torch.uint8, device=DEV)
    B.qsr_embed_grad(d, t, got, workspace=ws, stream=stream())
    assert got[:, 0].tolist() == [3.0, 0.0, 1.0, 0.0]


@pytest.mark.parametrize("pad,shift", [(0, 1), (3, 0), (8, 8), (5, 3)])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_strides_and_alignment(pad, shift, kind):
    R, V, N = 500, 60, 100
    _, d = around(R, N, "bf16", pad + 1, shift)
    d.copy_(torch.randn(R, N, device=DEV, generator=gen(2)))
    t = draw(R, V, 6)
    for accumulate in (False, True):
        check_grad(d, t, V, 0.5, kind, accumulate, lay=(pad, shift))
    _, w = around(V, N, kind, pad, shift)
    w.copy_(torch.randn(V, N, device=DEV, generator=gen(3)))
    flat, y = around(R, N, "f32", pad, shift)
    B.qsr_embed(w, t, y, stream=stream())
    want = torch.where((t >= 0)[:, None], w.float()[t.clamp_min(0)], 0.0)
    assert torch.equal(y, want)
    y.fill_(7.0)
    assert bool((flat == 7.0).all())


def test_values_that_are_not_finite_stay_in_their_tokens():
    d = torch.randn(300, 40, device=DEV, generator=gen(1))
    t = draw(300, 10, 1, "uniform")
    d[7, 3], d[9, 4] = math.nan, math.inf
    t[7], t[9] = 2, 5
    got = torch.empty(10, 40, device=DEV)
    ws = torch.empty(B.qsr_embed_workspace_bytes(300, 10, 40), dtype=torch.uint8, device=DEV)
    B.qsr_embed_grad(d, t, got, workspace=ws, stream=stream())
    bad = ~torch.isfinite(got)
    assert bad.sum() == 2 and math.isnan(got[2, 3]) and math.isinf(got[5, 4])


def test_no_rows():
    none, t = torch.empty(0, 12, device=DEV), torch.empty(0, device=DEV, dtype=torch.int64)
    g = torch.full((5, 12), 3.0, device=DEV)
    ws = torch.empty(B.qsr_embed_workspace_bytes(0, 5, 12), dtype=torch.uint8, device=DEV)
    B.qsr_embed(g, t, none, stream=stream())
    B.qsr_embed_grad(none, t, g, accumulate=True, workspace=ws, stream=stream())
    assert bool((g == 3.0).all())
    B.qsr_embed_grad(none, t, g, workspace=ws, stream=stream())
    assert not g.any()


def test_offsets_beyond_32_bits():
    """A table of more than 2^32 bytes and 2^31 elements: its last rows."""
    V, N = (1 << 21) + 100, 1024
    w = torch.zeros(V, N, device=DEV, dtype=torch.bfloat16)
    w[-3:] = torch.randn(3, N, device=DEV, generator=gen(1)).bfloat16()
    t = torch.tensor([V - 1, V - 3, 0, V - 2], device=DEV)
    y = torch.empty(4, N, device=DEV, dtype=torch.bfloat16)
    B.qsr_embed(w, t, y, stream=stream())
    assert torch.equal(y, w[t])
    B.qsr_embed_grad(y, t, w.fill_(1.0), workspace=torch.empty(B.qsr_embed_workspace_bytes(4, V, N), dtype=torch.uint8, device=DEV), stream=stream())
    assert torch.equal(w[t], y) and int(torch.count_nonzero(w[1:-3])) == 0


def test_captured_and_replayed_with_other_tokens():
    R, V, N = 3000, 500, 96
    d = torch.randn(R, N, device=DEV, generator=gen(1)).bfloat16()
    t, g = draw(R, V, 1), torch.empty(V, N, device=DEV)
    ws = torch.empty(B.qsr_embed_workspace_bytes(R, V, N), dtype=torch.uint8, device=DEV)
    B.qsr_embed_grad(d, t, g, workspace=ws, stream=stream())
    first = g.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        B.qsr_embed_grad(d, t, g, workspace=ws, stream=stream())
    g.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(g, first)
    t.copy_(draw(R, V, 2))
    graph.replay()
    second = g.clone()
    B.qsr_embed_grad(d, t, g, workspace=ws, stream=stream())
    assert torch.equal(g, second) and not torch.equal(first, second)


@pytest.mark.parametrize("kind,out", [("f32", "bf16"), ("bf16", "f16"), ("f16", "f32")])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("R,V,N", [(1, 2048, 3), (15, 3, 9), (16, 2049, 9), (17, 40, 64), (32, 1, 65), (33, 70000, 8), (257, 5000, 200), (4095, 6, 70), (4096, 300, 130), (4097, 300, 130),
                                   (4096, 1 << 21, 2), (600, (1 << 21) + 1, 2), (8192, 5000, 128), (8193, 5000, 128),
                                   (8192, 3, 129), (16384, 30011, 64), (16383, 9, 33), (16385, 700, 64)])
def test_gradient_of_few_rows(R, V, N, kind, out, accumulate):
    """One launch for up to 4096 rows, or 16384 parts of 64 columns, and 2^21 tokens; the others sort."""
    d = torch.randn(R, N, device=DEV, generator=gen(R)).to(T[out])
    for how in ("zipf", "uniform", "same", "absent", "outside"):
        check_grad(d, draw(R, V, R + V, how), V, 0.75, kind, accumulate)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("R,V,N", [(20000, 30011, 64), (20000, 20000, 513), (70000, 70001, 24), (5000, (1 << 21) + 9, 8)])
def test_sorted_gradient_in_a_graph_before_a_copy(R, V, N, accumulate):
    """Rows that are sorted, none of whose tokens has rows in two chunks, so that nothing is joined: what follows the gradient in a graph finds it
    complete.  All tokens different (positions, say): every sum is one product; padding alone: nothing is added."""
    d = torch.randn(R, N, device=DEV, generator=gen(R)).bfloat16()
    start = torch.randn(V, N, device=DEV, generator=gen(V)) if accumulate else None
    for t in (torch.randperm(V, device=DEV, generator=gen(1))[:R], torch.full((R,), -1, device=DEV)):
        g, copy = torch.zeros(V, N, device=DEV), torch.empty(V, N, device=DEV)
        ws = torch.empty(B.qsr_embed_workspace_bytes(R, V, N), dtype=torch.uint8, device=DEV)
        B.qsr_embed_grad(d, t, g, scale=0.5, accumulate=accumulate, workspace=ws, stream=stream())
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            if accumulate:
                g.copy_(start)
            else:
                g.fill_(3.0)
            B.qsr_embed_grad(d, t, g, scale=0.5, accumulate=accumulate, workspace=ws, stream=stream())
            copy.copy_(g)
        for _ in range(20):
            d.mul_(-1.0).add_(0.25)
            want = start.clone() if accumulate else torch.zeros(V, N, device=DEV)
            some = t >= 0
            want[t[some]] += 0.5 * d[some].float()
            graph.replay()
            assert torch.equal(copy, want) and torch.equal(g, want)


@pytest.mark.parametrize("accumulate", [False, True])
def test_rows_beyond_32_bits(accumulate):
    """Looked-up rows of more than 2^31 elements; of the gradient, which sorts them, those with a token are the last ones."""
    R, V, N = (1 << 21) + 1001, 4000, 1024
    w = torch.randn(V, N, device=DEV, generator=gen(1)).bfloat16()
    t = torch.full((R,), -1, device=DEV)
    t[-3000:] = torch.randint(0, V, (3000,), device=DEV, generator=gen(2))
    y = torch.empty(R, N, device=DEV, dtype=torch.bfloat16)
    B.qsr_embed(w, t, y, stream=stream())
    assert torch.equal(y[-3000:], w[t[-3000:]]) and not y[0].any() and not y[R // 2].any() and not y[-3001].any()
    y[:-3000] = math.nan                                              # of rows without a token nothing is added
    g = torch.randn(V, N, device=DEV, generator=gen(3))
    want = (g.double() if accumulate else torch.zeros(V, N, device=DEV, dtype=torch.float64)).index_add_(0, t[-3000:], y[-3000:].double())
    size = (g.double().abs() if accumulate else torch.zeros_like(want)).index_add_(0, t[-3000:], y[-3000:].double().abs())
    ws = torch.empty(B.qsr_embed_workspace_bytes(R, V, N), dtype=torch.uint8, device=DEV)
    B.qsr_embed_grad(y, t, g, accumulate=accumulate, workspace=ws, stream=stream())
    count = torch.bincount(t[-3000:], minlength=V).double()[:, None]
    assert not ((g.double() - want).abs() > (count + 10) * U * size).any()
