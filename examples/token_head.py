"""Train a token encoder's head, serve it in 8 bits, and search the tokens that it makes.

The head is a layer norm and a projection to the 128 columns of the search engine, on top of the hidden states
of an encoder (synthetic ones here: what tells passages apart lies in a few directions, under a larger part that
does not). It is trained with the library's layer norm and AdamW (8-bit moments) so that a query's sum of token
maxima is larger for its passage than for the others of a batch; then the projection is quantised, passages and
queries go through the int8 head, and `build_index` and `search_async` find the passages again.

    python examples/token_head.py [--steps 150]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2501_17788_amd as warp  # noqa: E402

WIDTH, DIM = 768, 128
DOCS, DOC_TOKENS, QUERY_TOKENS, BATCH = 1024, 24, 8, 64
SIGNAL = 64  # directions that tell tokens apart


class Data:
    """Hidden states [docs, tokens, WIDTH] bfloat16 of passages and of queries that repeat some of their tokens."""

    def __init__(self, seed: int):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def randn(*shape):
            return torch.randn(*shape, generator=g, device="cuda")

        self.generator = g
        self.basis = randn(SIGNAL, WIDTH) / WIDTH ** 0.5
        self.noise_basis = randn(160, WIDTH) / WIDTH ** 0.5
        self.signal = randn(DOCS, DOC_TOKENS, SIGNAL)
        self.randn = randn
        self.passages = self.hidden(self.signal)
        self.queries = self.hidden(self.signal[:, :QUERY_TOKENS] + 0.1 * randn(DOCS, QUERY_TOKENS, SIGNAL))

    def hidden(self, signal):
        noise = self.randn(*signal.shape[:-1], 160) @ self.noise_basis
        return (signal @ self.basis + 1.2 * noise).bfloat16()


def head(hidden, weight, bias, projection):
    """Unit tokens [..., DIM] of hidden states, for training."""
    y = warp.layer_norm(hidden, weight, bias)[0]
    return torch.nn.functional.normalize(y.float() @ projection.t(), dim=-1)


def train(data: Data, steps: int):
    weight, bias = torch.ones(WIDTH, device="cuda"), torch.zeros(WIDTH, device="cuda")
    projection = torch.randn(DIM, WIDTH, generator=data.generator, device="cuda") / WIDTH ** 0.5
    params = [p.requires_grad_() for p in (weight, bias, projection)]
    opt = warp.AdamW(params, lr=5e-3, weight_decay=0.01, bits=8)
    losses = []
    for step in range(steps):
        docs = torch.randint(0, DOCS, (BATCH,), generator=data.generator, device="cuda")
        q, d = (head(h[docs], *params) for h in (data.queries, data.passages))
        similarity = (q.reshape(-1, DIM) @ d.reshape(-1, DIM).t()).view(BATCH, QUERY_TOKENS, BATCH, DOC_TOKENS)
        scores = similarity.amax(3).sum(1)
        loss = torch.nn.functional.cross_entropy(8 * scores, torch.arange(BATCH, device="cuda"))
        grads = torch.autograd.grad(loss, params)
        opt.step([g.contiguous() for g in grads])
        losses.append(loss.detach())
        if step % 50 == 49:
            print(f"step {step + 1}: loss {torch.stack(losses[-50:]).mean().item():.3f}", flush=True)
    return [p.detach() for p in params]


def encode(hidden, weight, bias, projection: warp.QuantizedRows):
    """Unit tokens [..., DIM] float32 of hidden states through the int8 head."""
    rows = warp.layer_norm_int8(hidden, weight, bias)
    tokens = warp.linear_int8(rows, projection, dtype=torch.float32)
    return torch.nn.functional.normalize(tokens, dim=-1).view(*hidden.shape[:-1], DIM)


def find(data: Data, weight, bias, projection) -> float:
    """The share of queries whose passage a search puts first."""
    quantised = warp.quantize_rows(projection)
    tokens = encode(data.passages, weight, bias, quantised).view(-1, DIM)
    queries = encode(data.queries, weight, bias, quantised)
    sample = torch.arange(tokens.shape[0]).numpy()
    built = warp.build_index(tokens, torch.arange(DOCS, device="cuda").repeat_interleave(DOC_TOKENS), DOCS,
                             warp.initial_centroids(tokens, sample, 256), sample, 4, 4, tokens.shape[0])
    with warp.Index.from_device(built["centroids"], built["offsets"], built["doc_ids"], built["codes"], 4,
                                built["weights"], DOCS) as index:
        ids = index.search_async(queries.contiguous(), 32, warp.t_prime_policy(tokens.shape[0]), 10)[0]
        index.sync()
        return (ids[:, 0] == torch.arange(DOCS, device="cuda")).float().mean().item()


def main(argv=None) -> tuple[float, float]:
    parser = argparse.ArgumentParser()
    parser.add_argument("--steps", type=int, default=150)
    args = parser.parse_args(argv)
    before = find(Data(0), *train(Data(0), 0))
    data = Data(0)
    params = train(data, args.steps)
    after = find(data, *params)
    exact = head(data.queries, *params)
    close = (exact * encode(data.queries, *params[:2], warp.quantize_rows(params[2]))).sum(-1).min().item()
    print(f"passage found first: {before:.1%} with the untrained head, {after:.1%} after {args.steps} steps; "
          f"smallest cosine of a token in 8 bits with its exact one {close:.4f}", flush=True)
    return before, after


if __name__ == "__main__":
    main()
