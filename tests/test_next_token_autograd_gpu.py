"""The next-token example's functions as autograd knows them: gradients are returned and not left somewhere, hooks run, what is written over
between the passes is noticed, and a second derivative is refused."""
import pytest
import torch

from paper_2310_14423_b200 import next_token

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def embedding():
    table = torch.randn(9, 16, device=DEV, generator=torch.Generator(DEV).manual_seed(1)).requires_grad_()
    tokens = torch.tensor([3, 0, 3, 8], device=DEV)
    d_out = torch.arange(64, device=DEV, dtype=torch.float32).view(4, 16)
    want = torch.zeros(9, 16, device=DEV).index_add_(0, tokens, d_out)
    return table, tokens, d_out, want


def test_the_tables_gradient_is_returned():
    table, tokens, d_out, want = embedding()
    table.grad = torch.full_like(table, 7.0)
    got, = torch.autograd.grad(next_token.Embedding.apply(table, tokens), table, d_out)
    assert torch.equal(got, want) and bool((table.grad == 7.0).all())
    next_token.Embedding.apply(table, tokens).backward(d_out)
    assert torch.equal(table.grad, want + 7.0)                        # added to what is there, in place
    fresh = table.detach().clone().requires_grad_()
    next_token.Embedding.apply(fresh, tokens).backward(d_out)          # and made where nothing is
    assert torch.equal(fresh.grad, want)


def test_two_uses_of_a_table_and_hooks():
    table, tokens, d_out, want = embedding()
    seen = []
    table.register_hook(lambda g: seen.append(g.clone()) or 2.0 * g)
    (next_token.Embedding.apply(table, tokens) + next_token.Embedding.apply(table, tokens.flip(0))).backward(d_out)
    both = want + torch.zeros_like(want).index_add_(0, tokens.flip(0), d_out)
    assert len(seen) == 1 and torch.equal(seen[0], both) and torch.equal(table.grad, 2.0 * both)


def test_tokens_written_over_between_the_passes_are_noticed():
    table, tokens, d_out, _ = embedding()
    out = next_token.Embedding.apply(table, tokens)
    tokens[0] = 1
    with pytest.raises(RuntimeError):
        out.backward(d_out)
    assert table.grad is None


def test_second_derivatives_are_refused():
    table, tokens, d_out, _ = embedding()
    weight, bias = torch.ones(16, device=DEV, requires_grad=True), torch.zeros(16, device=DEV, requires_grad=True)
    d_out.requires_grad_()
    for out, leaf in ((next_token.Embedding.apply(table, tokens), table), (next_token.LayerNorm.apply(table, weight, bias), weight)):
        d = d_out if out.shape == d_out.shape else torch.ones_like(out, requires_grad=True)
        first, = torch.autograd.grad(out, leaf, d, create_graph=True)
        with pytest.raises(RuntimeError):
            torch.autograd.grad(first.square().sum(), d)
