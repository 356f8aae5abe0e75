"""The operators of a training step together: embedding, layer norm, log probabilities, and steps by AdamW and by orthogonalised momentum
with their round ends, as the next-token example's "normed" model uses them."""
import pytest
import torch

from paper_2310_14423_b200 import binding as B
from paper_2310_14423_b200 import next_token
from paper_2310_14423_b200 import workloads as W

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("states,state_sync,width", [("f32", "keep", 64), ("e4m3", "average", 64), ("f32", "reset", 200)])
def test_the_normed_model_runs(states, state_sync, width):
    r = next_token.train(workers=3, steps=40, vocab=101, width=width, rows=16, length=16, states=states, state_sync=state_sync, model="normed")
    assert r["replicas_equal"] and r["loss"] == r["loss"]
    w = W.Workload("next_token", 3, W.flat_layout(1), W.OPT_ADAMW, T=40, T_warmup=2, eta_max=8e-3, alpha=0.0175, H_base=4, weight_decay=0.05)
    starts, _ = B.qsr_config_schedule(B.make_config(w))
    assert r["rounds"] == len(starts)
    sync = r["rounds"] * (2 if state_sync == "reset" else 1)
    assert r["launches"] == 2 * 40 + sync
    assert r["matrix_launches"] == 40 * (1 if width == 64 else 18) + sync      # a small matrix's step is one launch


def test_gradients_of_the_whole_model():
    """All gradients in fp32 against the same model in binary64.  No chain of additions is longer than 400 (rows, vocabulary, width),
    400 * 2^-24 = 2.4e-5 of the terms' size; four products and a norm in a row and what cancels in them leave two orders of magnitude."""
    V, N, R = 90, 48, 300
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    n = lambda *s: torch.randn(*s, device=DEV, generator=g)                    # noqa: E731
    weights = [n(V, N), 1 + 0.2 * n(N), 0.2 * n(N), n(N, N) * N ** -0.5, 0.1 * n(N), n(N, V) * N ** -0.5]
    tokens, targets = (torch.randint(0, V, (R,), device=DEV, generator=g) for _ in range(2))
    mine = [w.clone().requires_grad_() for w in weights]
    mine[0].grad = torch.zeros_like(weights[0])
    logits = next_token.normed_logits_of(mine, tokens)
    logprob, d_logits = torch.empty(R, device=DEV), torch.empty_like(logits)
    B.qsr_token_logprobs(logits.detach(), targets, logprob, d_logprob=torch.full((R,), -1.0 / R, device=DEV), d_logits=d_logits,
                         stream=torch.cuda.current_stream().cuda_stream)
    logits.backward(gradient=d_logits)
    embed, nw, nb, hidden, bias, head = want = [w.double().requires_grad_() for w in weights]
    h = torch.nn.functional.layer_norm(embed[tokens], (N,), nw, nb, 1e-5)
    out = torch.nn.functional.gelu(h @ hidden + bias) @ head
    torch.nn.functional.cross_entropy(out, targets).backward()
    assert torch.allclose(logprob.double(), out.log_softmax(1).gather(1, targets[:, None])[:, 0], rtol=0, atol=2.4e-3)
    for a, b in zip(mine, want):
        assert float(torch.linalg.vector_norm(a.grad.double() - b.grad)) <= 2.4e-3 * float(torch.linalg.vector_norm(b.grad))


def test_a_step_of_the_whole_model_in_a_graph():
    """Forward, backward and both optimizers' steps captured once and replayed: the same bits as without a graph."""
    V, N, R, lr = 64, 32, 100, 1e-2
    results = []
    for captured in (False, True):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            s = stream.cuda_stream
            g = torch.Generator(device=DEV)
            g.manual_seed(5)
            n = lambda *sz: torch.randn(*sz, device=DEV, generator=g)          # noqa: E731
            table, w, b, hidden = n(V, N), 1 + 0.1 * n(N), 0.1 * n(N), n(N, V) * N ** -0.5
            tokens, targets = (torch.randint(0, V, (R,), device=DEV, generator=g) for _ in range(2))
            e = lambda *sz: torch.empty(*sz, device=DEV)                       # noqa: E731
            x, y, mean, rstd, dx, dy, dw, db, dt, dh = e(R, N), e(R, N), e(R), e(R), e(R, N), e(R, N), e(N), e(N), e(V, N), e(N, V)
            logits, d_logits, lp, dlp = e(R, V), e(R, V), e(R), torch.full((R,), -1.0 / R, device=DEV)
            ws = torch.empty(max(B.qsr_embed_workspace_bytes(R, V, N), B.qsr_layer_norm_workspace_bytes(R, N)), dtype=torch.uint8, device=DEV)
            z = lambda t: torch.zeros_like(t)                                  # noqa: E731
            space = torch.empty(B.qsr_list_workspace_bytes([table.numel(), N, N]), dtype=torch.uint8, device=DEV)
            rest = B.TensorList([table, w, b], [dt, dw, db], [z(table), z(w), z(b)], [z(table), z(w), z(b)], workspace=space, stream=s)
            more = torch.empty(B.qsr_muon_workspace_bytes([(N, V)], 1, 3), dtype=torch.uint8, device=DEV)
            matrix = B.MuonList([hidden], [dh], [z(hidden)], products=3, workspace=more, stream=s)

            def step():
                B.qsr_embed(table, tokens, x, stream=s)
                B.qsr_layer_norm(x, y, weight=w, bias=b, mean=mean, rstd=rstd, stream=s)
                torch.matmul(y, hidden, out=logits)
                B.qsr_token_logprobs(logits, targets, lp, d_logprob=dlp, d_logits=d_logits, stream=s)
                torch.matmul(d_logits, hidden.t(), out=dy)
                torch.matmul(y.t(), d_logits, out=dh)
                B.qsr_layer_norm_grad(x, dy, mean, rstd, d_x=dx, weight=w, d_weight=dw, d_bias=db, workspace=ws, stream=s)
                B.qsr_embed_grad(dx, tokens, dt, workspace=ws, stream=s)
                rest.qsr_list_step(1, lr)
                matrix.qsr_muon_step(lr)

            step()
            stream.synchronize()
            if captured:
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=stream):
                    step()
                for _ in range(3):
                    graph.replay()
            else:
                for _ in range(3):
                    step()
            stream.synchronize()
            results.append([t.clone() for t in (table, w, b, hidden, lp)])
    assert all(torch.equal(p, q) for p, q in zip(*results))
