"""Local AdamW with the Quadratic Synchronization Rule (Algorithm 2 of arXiv 2310.14423) on a small next-token model: the
tensor lists and the token log probabilities of this library, as a training program uses them.

K replicas of an embedding - GELU layer - head model learn a seeded first-order Markov chain.  torch does the model's matrix
products and their backward pass; the library does the rest of the step: the loss and its gradient with respect to the logits
(one call), the clipped AdamW step over all replicas' tensors (states in fp32 or 8 bits, bf16 working copies written along),
the round lengths and learning rates, and the averaging at the end of each round.

The "normed" model has a layer norm behind the embedding.  The library then does the lookup and its gradient, the norm and its gradients
too, and the hidden matrix is stepped by its orthogonalised momentum while AdamW steps the rest.

    python -m paper_2310_14423_b200.next_token --workers 4 --steps 400 --states e4m3
    python -m paper_2310_14423_b200.next_token --model normed
"""
from __future__ import annotations

import argparse
import math
import sys
from typing import Dict, List

import torch
from torch.autograd.function import once_differentiable

from . import binding as B
from . import workloads as W

DEV = "cuda"


class Chain:
    """A first-order Markov chain over `vocab` tokens whose transitions are softmax(1.5 * normal) (seeded)."""

    def __init__(self, vocab: int, seed: int):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        self.p = torch.softmax(1.5 * torch.randn(vocab, vocab, device=DEV, generator=g), 1)
        self.generator = g

    def batch(self, rows: int, length: int):
        """(tokens, the token after each): two int64 vectors of rows * length."""
        x = torch.randint(0, self.p.shape[0], (rows,), device=DEV, generator=self.generator)
        steps = [x]
        for _ in range(length):
            x = torch.multinomial(self.p[x], 1, generator=self.generator)[:, 0]
            steps.append(x)
        s = torch.stack(steps, 1)
        return s[:, :-1].reshape(-1).contiguous(), s[:, 1:].reshape(-1).contiguous()

    def entropy_rate(self) -> float:
        """Conditional entropy under the stationary distribution: the least loss any model can reach."""
        q = torch.full((1, self.p.shape[0]), 1.0 / self.p.shape[0], device=DEV)
        for _ in range(200):
            q = q @ self.p
        return float((q[0] * torch.special.entr(self.p).sum(1)).sum())


def logits_of(weights: List[torch.Tensor], tokens: torch.Tensor) -> torch.Tensor:
    embed, hidden, bias, head = weights
    h = torch.nn.functional.gelu(embed[tokens] @ hidden + bias)
    return h @ head


class Embedding(torch.autograd.Function):
    """Rows of a table."""

    @staticmethod
    def forward(ctx, table, tokens):
        out = torch.empty(tokens.numel(), table.shape[1], device=table.device, dtype=table.dtype)
        B.qsr_embed(table, tokens, out, stream=torch.cuda.current_stream().cuda_stream)
        ctx.save_for_backward(tokens)
        ctx.shape = table.shape
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, d_out):
        tokens, = ctx.saved_tensors
        d_table = torch.empty(ctx.shape, device=d_out.device, dtype=d_out.dtype)
        workspace = torch.empty(B.qsr_embed_workspace_bytes(tokens.numel(), *ctx.shape), dtype=torch.uint8, device=d_out.device)
        B.qsr_embed_grad(d_out.contiguous(), tokens, d_table, workspace=workspace, stream=torch.cuda.current_stream().cuda_stream)
        return d_table, None


class LayerNorm(torch.autograd.Function):
    """Layer norm of the rows of a matrix with weight and bias."""

    @staticmethod
    def forward(ctx, x, weight, bias):
        y, mean, rstd = torch.empty_like(x), torch.empty(x.shape[0], device=x.device), torch.empty(x.shape[0], device=x.device)
        B.qsr_layer_norm(x, y, weight=weight, bias=bias, mean=mean, rstd=rstd, stream=torch.cuda.current_stream().cuda_stream)
        ctx.save_for_backward(x, weight, mean, rstd)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, d_y):
        x, weight, mean, rstd = ctx.saved_tensors
        d_x, d_weight, d_bias = torch.empty_like(x), torch.empty_like(weight), torch.empty_like(weight)
        workspace = torch.empty(B.qsr_layer_norm_workspace_bytes(*x.shape), dtype=torch.uint8, device=x.device)
        B.qsr_layer_norm_grad(x, d_y.contiguous(), mean, rstd, d_x=d_x, weight=weight, d_weight=d_weight, d_bias=d_bias, workspace=workspace,
                              stream=torch.cuda.current_stream().cuda_stream)
        return d_x, d_weight, d_bias


def normed_logits_of(weights: List[torch.Tensor], tokens: torch.Tensor) -> torch.Tensor:
    embed, norm_weight, norm_bias, hidden, bias, head = weights
    h = LayerNorm.apply(Embedding.apply(embed, tokens), norm_weight, norm_bias)
    return torch.nn.functional.gelu(h @ hidden + bias) @ head


MODELS = {"plain": logits_of, "normed": normed_logits_of}


def train(workers: int = 4, steps: int = 400, vocab: int = 1000, width: int = 128, rows: int = 64, length: int = 32, states: str = "e4m3",
          state_sync: str = "keep", eta_max: float = 8e-3, alpha: float = 0.0175, h_base: int = 4, clip: float = 1.0, seed: int = 1,
          model: str = "plain", muon_lr: float = 2.5, log=None) -> Dict[str, float]:
    """One run; returns the last held-out loss, the chain's entropy rate, rounds and kernel launches.  muon_lr: the hidden matrix's
    learning rate in the "normed" model, in units of AdamW's."""
    stream = torch.cuda.current_stream().cuda_stream
    torch.manual_seed(seed)
    w = W.Workload("next_token", workers, W.flat_layout(1), W.OPT_ADAMW, T=steps, T_warmup=max(1, steps // 20), eta_max=eta_max, alpha=alpha,
                   H_base=h_base, weight_decay=0.05, state_sync=state_sync)
    cfg = B.make_config(w)
    chain = Chain(vocab, seed)

    shapes = [(vocab, width), (width, width), (width,), (width, vocab)]
    first = [torch.randn(s, device=DEV) * (0.02 if len(s) == 1 or s[0] == vocab else s[0] ** -0.5) for s in shapes]
    if model == "normed":
        shapes[1:1] = [(width,), (width,)]
        first[1:1] = [torch.ones(width, device=DEV), torch.zeros(width, device=DEV)]
    forward = MODELS[model]
    params = [x.clone() for _ in range(workers) for x in first]
    copies = [x.to(torch.bfloat16).requires_grad_() for x in params]
    for c in copies:
        c.grad = torch.zeros_like(c)                    # kept and zeroed, so that the list's addresses stay valid
    f8 = torch.float8_e4m3fn
    kind = f8 if states == "e4m3" else torch.float32
    zeros = lambda: [torch.zeros(p.shape, device=DEV, dtype=torch.uint8).view(f8) if kind is f8 else torch.zeros_like(p) for p in params]  # noqa: E731
    scales = lambda: [torch.zeros((p.numel() + 255) // 256, device=DEV) for p in params] if kind is f8 else None                         # noqa: E731
    norms = torch.zeros(workers, device=DEV)
    # the hidden matrix goes to the list of matrices in the normed model, everything else to the list of tensors
    hidden = [i for i in range(len(params)) if model == "normed" and i % len(shapes) == 3]
    rest = [i for i in range(len(params)) if i not in hidden]
    every = lambda a, which=rest: None if a is None else [a[i] for i in which]                                                          # noqa: E731
    workspace = torch.empty(B.qsr_list_workspace_bytes([params[i].numel() for i in rest], workers), dtype=torch.uint8, device=DEV)
    tensors = B.TensorList(every(params), [copies[i].grad for i in rest], every(zeros()), every(zeros()), m_scale=every(scales()),
                           v_scale=every(scales()), copies=[copies[i].detach() for i in rest],
                           wd_scale=[0.0 if params[i].dim() == 1 else 1.0 for i in rest], workers=workers,
                           beta1=w.beta1, beta2=w.beta2, eps=w.eps, weight_decay=w.weight_decay, clip_norm=clip, grad_norm=norms,
                           workspace=workspace, stream=stream)
    matrices = None
    if hidden:
        space = torch.empty(B.qsr_muon_workspace_bytes([(width, width)] * workers, workers, 3), dtype=torch.uint8, device=DEV)
        matrices = B.MuonList(every(params, hidden), [copies[i].grad for i in hidden], [torch.zeros(width, width, device=DEV) for _ in hidden],
                              copies=[copies[i].detach() for i in hidden], workers=workers, weight_decay=w.weight_decay, products=3,
                              workspace=space, stream=stream)
    n = rows * length
    logprob = torch.empty(n, device=DEV)
    d_logprob = torch.full((n,), -1.0 / n, device=DEV)   # loss: the mean of -logprob
    d_logits = torch.empty(n, vocab, device=DEV, dtype=torch.bfloat16)
    held_x, held_y = chain.batch(64, 32)

    def weights(k: int) -> List[torch.Tensor]:
        return copies[k * len(shapes):(k + 1) * len(shapes)]

    def held_out() -> float:
        with torch.no_grad():
            x = forward(weights(0), held_x)
            out = torch.empty(held_y.numel(), device=DEV)
            B.qsr_token_logprobs(x, held_y, out, stream=stream)
            return -float(out.mean())

    t = rounds = origin = 0
    start = loss = held_out()
    while t < steps:
        H = B.qsr_config_round_length(cfg, t)
        for h in range(H):
            for c in copies:
                c.grad.zero_()
            for k in range(workers):
                tokens, targets = chain.batch(rows, length)
                logits = forward(weights(k), tokens)
                B.qsr_token_logprobs(logits, targets, logprob, d_logprob=d_logprob, d_logits=d_logits, stream=stream)
                logits.backward(gradient=d_logits)
            lr = B.qsr_config_learning_rate(cfg, t + h)
            tensors.qsr_list_step(t + h + 1 - origin, lr)
            if matrices:
                matrices.qsr_muon_step(muon_lr * lr)
        t += H
        rounds += 1
        tensors.qsr_list_sync(state_sync)
        if matrices:
            matrices.qsr_muon_sync(state_sync)
        if state_sync == W.STATE_RESET:
            origin = t
        if log:
            loss = held_out()
            log(f"round {rounds}: t = {t}, H = {H}, lr = {B.qsr_config_learning_rate(cfg, t - 1):.2e}, gradient norm {float(norms[0]):.3f}, "
                f"held-out loss {loss:.4f}")
    loss = held_out()
    if matrices:
        matrices.qsr_muon_check()

    # serving form: one row, its most likely continuations
    with torch.no_grad():
        x = forward(weights(0), held_x[:1])
        lp, ent = torch.empty(1, device=DEV), torch.empty(1, device=DEV)
        top_lp, top = torch.empty(1, 5, device=DEV), torch.empty(1, 5, device=DEV, dtype=torch.int64)
        B.qsr_token_logprobs(x, held_y[:1], lp, entropy=ent, top_logprob=top_lp, top_token=top, stream=stream)
    if log:
        true = torch.log(chain.p[held_x[0], top[0]])
        log("after token %d: " % int(held_x[0]) + ", ".join("%d (%.2f, chain %.2f)" % (int(i), float(a), float(b))
                                                             for i, a, b in zip(top[0], top_lp[0], true)) + f"; entropy {float(ent[0]):.3f}")
    same = all(torch.equal(a, b) for k in range(1, workers) for a, b in zip(params[:len(shapes)], params[k * len(shapes):]))
    return {"start": start, "loss": loss, "entropy_rate": chain.entropy_rate(), "rounds": rounds, "launches": tensors.qsr_list_launch_count(),
            "matrix_launches": matrices.qsr_muon_launch_count() if matrices else 0,
            "replicas_equal": same, "uniform": math.log(vocab)}


def main() -> int:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--steps", type=int, default=400)
    ap.add_argument("--vocab", type=int, default=1000)
    ap.add_argument("--width", type=int, default=128)
    ap.add_argument("--states", choices=("f32", "e4m3"), default="e4m3")
    ap.add_argument("--state-sync", choices=("keep", "average", "reset"), default="keep")
    ap.add_argument("--model", choices=tuple(MODELS), default="plain")
    ap.add_argument("--seed", type=int, default=1)
    a = ap.parse_args()
    r = train(workers=a.workers, steps=a.steps, vocab=a.vocab, width=a.width, states=a.states, state_sync=a.state_sync, seed=a.seed, model=a.model,
              log=print)
    print(f"held-out loss {r['loss']:.4f} (start {r['start']:.4f}, entropy rate of the chain {r['entropy_rate']:.4f}), {r['rounds']} rounds, "
          f"{r['launches']} list launches")
    return 0


if __name__ == "__main__":
    sys.exit(main())
