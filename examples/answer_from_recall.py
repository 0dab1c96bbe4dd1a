"""Answer from recalled chunks: the serving calls together, on one MI355X.

    python examples/answer_from_recall.py [--chunks 16] [--layers 4] [--steps 8]

One request recalls cached video chunks and decodes an answer over them:

1. ``rehydrate``      rebuilds every chunk at its place in the context;
2. ``page_tables``    gives the request pages for the whole context;
3. ``append_paged8``  keeps the rebuilt rows in 8 bits, with the pages' key sums;
4. ``page_tables``, ``append_paged8``, ``attend_paged``
                      the question's tokens, causal over the context;
5. every answer token: the same, with ``select_pages`` and attention over the
   selected pages alone, captured once in a HIP graph and replayed.

The library has no model: queries, keys and values of new tokens are seeded
random rows that stand for a layer's projections.
"""

from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2606_23581_amd as km  # noqa: E402

KV_HEADS, GROUP, DIM, PAGE, RANK = 8, 8, 128, 16, 16


class Request:
    """One request's cache and the calls that grow and read it."""

    def __init__(self, layers: int, most_tokens: int, keep: int, device):
        self.layers, self.keep, self.device = layers, keep, device
        self.most = -(-most_tokens // PAGE) * PAGE
        pages = self.most // PAGE
        self.cache = km.Cache8.allocate(layers, pages + 8, PAGE, KV_HEADS, DIM, device)
        self.table = torch.full((1, pages), -1, dtype=torch.int32, device=device)
        self.free = torch.randperm(pages + 8, device=device).to(torch.int32)
        i32 = dict(dtype=torch.int32, device=device)
        self.begin, self.end, self.base = torch.zeros(1, **i32), torch.zeros(1, **i32), torch.zeros(2, **i32)
        self.before, self.tokens = torch.zeros(1, **i32), torch.zeros(1, **i32)
        self.sel = torch.zeros((1, KV_HEADS, keep), **i32)
        self.count = torch.zeros((1, KV_HEADS), **i32)
        self.status = torch.zeros(1, **i32)

    def grow(self, n: int) -> None:
        """n more tokens: their pages (the lengths stay on the device)."""
        self.before.copy_(self.tokens)
        self.tokens.add_(n)
        self.begin.copy_(self.end)
        km.page_tables(self.before, self.tokens, self.free, self.table, page_size=PAGE,
                       n_pool_pages=self.cache.k.shape[1], free_begin=self.begin, free_end=self.end,
                       token_base=self.base, status=self.status)

    def append(self, k, v, table=None, tokens_before=None) -> None:
        """Rows [chunks, layers, n, KV heads, dim] behind the tokens that are there."""
        c = self.cache
        km.append_paged8(k, v, c.k, c.v, c.k_scale, c.v_scale, self.table if table is None else table,
                         tokens_before=tokens_before, k_sum=c.k_sum, k_sum_scale=c.k_sum_scale, status=self.status)

    def attend(self, layer: int, q, out, selected: bool = False) -> None:
        """The last q.shape[0] tokens' queries over the cache; ``selected``: over the chosen pages."""
        c, kw = self.cache, {}
        if selected:
            km.select_pages(q, c.k_sum[layer], c.k_sum_scale[layer], self.table, self.tokens, self.sel, self.count,
                            n_keys=self.most, page_size=PAGE, n_first=1, n_last=2, status=self.status)
            kw = dict(sel=self.sel, sel_count=self.count)
        km.attend_paged(q, out=out, page_table=self.table, kv_tokens=self.tokens, n_queries=q.shape[0],
                        n_keys=self.most, status=self.status, **c.layer(layer), **kw)


def recall(chunks: int, tokens: int, layers: int, gen, device):
    """Cached chunks rebuilt at contiguous places: K, V [chunks, layers, tokens, heads, dim]."""
    def rows(*shape, std=1.0):
        return (torch.randn(shape, generator=gen, device=device) * std).to(torch.bfloat16)

    shape = (chunks, layers, tokens, KV_HEADS, DIM)
    k, v = rows(*shape), rows(*shape)
    u = rows(2, chunks, layers, KV_HEADS, tokens, RANK, std=0.1)
    w = rows(2, chunks, layers, KV_HEADS, RANK, DIM, std=0.1)
    at = torch.zeros((chunks, 3), dtype=torch.int32, device=device)
    at[:, 0] = torch.arange(chunks, device=device) * tokens
    k_out, v_out = torch.empty_like(k), torch.empty_like(v)
    km.rehydrate(k, k_out, v_in=v, v_out=v_out, rope=km.RopeSpec(theta=1e6, rope_dim=DIM), chunk_pos=at,
                 u_k=u[0], w_k=w[0], u_v=u[1], w_v=w[1])
    return k_out, v_out


def answer(chunks=16, tokens=256, layers=4, question=64, steps=8, keep=32, seed=0, device="cuda", graph=True):
    """Runs the whole; returns the outputs of the question and of every answer token by layer."""
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)

    def rows(*shape):
        return torch.randn(shape, generator=gen, device=device).to(torch.bfloat16)

    r = Request(layers, chunks * tokens + question + steps, keep, device)
    k, v = recall(chunks, tokens, layers, gen, device)
    r.grow(chunks * tokens)
    # each chunk fills pages of its own: its row of the table is a piece of the request's
    r.append(k, v, table=r.table[:, :chunks * tokens // PAGE].reshape(chunks, tokens // PAGE))

    r.grow(question)
    k, v = rows(2, 1, layers, question, KV_HEADS, DIM)
    r.append(k, v, tokens_before=r.before)
    out_q = torch.empty((layers, question, KV_HEADS * GROUP, DIM), dtype=torch.bfloat16, device=device)
    for l in range(layers):
        r.attend(l, rows(question, KV_HEADS * GROUP, DIM), out_q[l])

    new = torch.empty((2, 1, layers, 1, KV_HEADS, DIM), dtype=torch.bfloat16, device=device)
    q = torch.empty((layers, 1, KV_HEADS * GROUP, DIM), dtype=torch.bfloat16, device=device)
    out = torch.empty_like(q)

    def step():
        r.grow(1)
        r.append(new[0], new[1], tokens_before=r.before)
        for l in range(layers):
            r.attend(l, q[l], out[l], selected=True)

    captured = None
    if graph:
        captured = torch.cuda.CUDAGraph()
        with torch.cuda.graph(captured):
            step()
    answers = []
    for _ in range(steps):
        new.copy_(rows(*new.shape))
        q.copy_(rows(*q.shape))
        if captured is not None:
            captured.replay()
        else:
            step()
        answers.append(out.clone())
    torch.cuda.synchronize()
    if int(r.status):
        raise RuntimeError(f"status {int(r.status)}: pages ran out or a table is wrong")
    return out_q, torch.stack(answers), r


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--chunks", type=int, default=16)
    ap.add_argument("--tokens", type=int, default=256, help="tokens of a chunk, a multiple of 16")
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--question", type=int, default=64)
    ap.add_argument("--steps", type=int, default=8)
    ap.add_argument("--keep", type=int, default=32, help="pages that an answer token attends to")
    a = ap.parse_args()
    out_q, answers, r = answer(a.chunks, a.tokens, a.layers, a.question, a.steps, a.keep)
    print(f"question {tuple(out_q.shape)}, answers {tuple(answers.shape)}, {int(r.tokens)} tokens in the cache, "
          f"{int(r.count.max())} of {int(r.tokens + PAGE - 1) // PAGE} pages attended to")


if __name__ == "__main__":
    main()
