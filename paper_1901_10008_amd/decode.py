"""Decoder layers of several tenants' models, step after step: the framework's products and the operators over paged caches
as a serving loop uses them.

    python -m paper_1901_10008_amd.decode [--tenants 4] [--layers 2] [--prompt 500] [--children 4] [--steps 32]

Every tenant has weights, pages and sequences of its own.  A layer is, for all tenants at once,

    sk_launch        queries, keys and values out of the hidden states: one product per tenant, all in one launch
    sk_attn_append   norms and rotation of their heads, keys and values to their pages
    sk_attn_launch   attention over the pages
    sk_launch        the products with the output weights, one launch

and the hidden states take up the result (a torch addition).  First the prompts, all rows at once; then every tenant's prompt is
forked into `children` continuations, which share its pages until they write to them, and each gets a token a step.  There is no
vocabulary: a step's input is the last hidden state of the sequence, scaled to unit size.
"""
from __future__ import annotations

import argparse
import math
import time

import torch

from . import (SK_GEMM, make_attn_problem, make_page_arrays, sk_attn_append, sk_attn_launch, sk_attn_plan_create, sk_launch, sk_pages_apply, sk_pages_create,
               sk_pages_fork, sk_pages_resize, sk_pages_state, sk_plan_create, sk_problem)

DTYPE = torch.bfloat16


def _product(a, b, c):
    """C = A . B^T as an operator of a plan."""
    p = sk_problem()
    p.op, p.dtype = SK_GEMM, 1
    p.M, p.K, p.N = a.shape[0], a.shape[1], b.shape[0]
    p.A, p.B, p.C = a.data_ptr(), b.data_ptr(), c.data_ptr()
    p.deadline_ms = math.inf
    return p


class Tenant:
    """One model: weights, pages, the account of its sequences."""

    def __init__(self, hidden, heads, layers, sequences, most_tokens, page=16, window=0, sinks=0, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def normal(*shape, scale=1.0):
            return (torch.randn(shape, generator=g, device="cuda") * scale).to(DTYPE)

        self.hidden, (self.hq, self.hkv, self.d), self.layers = hidden, heads, layers
        self.page, self.window, self.sinks, self.sequences = page, window, sinks, sequences
        self.columns = -(-most_tokens // page)
        self.pages = sequences * self.columns
        self.w_qkv = [normal((self.hq + 2 * self.hkv) * self.d, hidden, scale=hidden ** -0.5) for _ in range(layers)]
        self.w_out = [normal(hidden, self.hq * self.d, scale=(self.hq * self.d) ** -0.5) for _ in range(layers)]
        self.q_norm = [1 + normal(self.d, scale=0.1) for _ in range(layers)]
        self.k_norm = [1 + normal(self.d, scale=0.1) for _ in range(layers)]
        self.cache = torch.zeros((layers, 2, self.pages, self.hkv, page, self.d), dtype=DTYPE, device="cuda")
        one = self.cache[0, 0].numel() * 2
        self.arrays = make_page_arrays([(self.cache.data_ptr() + i * one, one // self.pages) for i in range(2 * layers)])
        half = self.d // 2
        angle = torch.arange(self.columns * page, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
        self.cos, self.sin = angle.cos().float().contiguous(), angle.sin().float().contiguous()
        self.table = torch.full((sequences, self.columns), -1, dtype=torch.int32, device="cuda")
        self.lengths = torch.zeros(sequences, dtype=torch.int32, device="cuda")
        self.first_row = torch.zeros(sequences + 1, dtype=torch.int32, device="cuda")
        self.account = sk_pages_create(self.pages, page, sequences, self.columns)


class Step:
    """The launches of a step in which every tenant has so many rows: planned once, used for every such step."""

    def __init__(self, tenants, rows, most_new):
        self.tenants, self.rows = tenants, rows
        new = lambda *shape: torch.zeros(shape, dtype=DTYPE, device="cuda")  # noqa: E731
        self.x = [new(n, t.hidden) for t, n in zip(tenants, rows)]
        self.qkv = [new(n, (t.hq + 2 * t.hkv) * t.d) for t, n in zip(tenants, rows)]
        self.q = [new(n, t.hq, t.d) for t, n in zip(tenants, rows)]
        self.out = [new(n, t.hq * t.d) for t, n in zip(tenants, rows)]
        self.y = [new(n, t.hidden) for t, n in zip(tenants, rows)]
        self.layers = []
        for layer in range(tenants[0].layers):
            into = sk_plan_create([_product(x, t.w_qkv[layer], c) for t, x, c in zip(tenants, self.x, self.qkv)])
            attend = sk_attn_plan_create([make_attn_problem(
                dtype="bf16", q_heads=t.hq, kv_heads=t.hkv, head_dim=t.d, page_tokens=t.page, num_pages=t.pages, sequences=t.sequences,
                pages_per_sequence=t.columns, rows=n, max_new=most_new, window=t.window, sinks=t.sinks, rotary_dim=t.d, positions=t.cos.shape[0], eps=1e-6,
                k=t.cache[layer, 0].data_ptr(), v=t.cache[layer, 1].data_ptr(), page_table=t.table.data_ptr(), lengths=t.lengths.data_ptr(),
                first_row=t.first_row.data_ptr(), qkv=qkv.data_ptr(), q_weight=t.q_norm[layer].data_ptr(), k_weight=t.k_norm[layer].data_ptr(),
                cos=t.cos.data_ptr(), sin=t.sin.data_ptr(), q=q.data_ptr(), out=out.data_ptr())
                for t, n, qkv, q, out in zip(tenants, rows, self.qkv, self.q, self.out)])
            out_of = sk_plan_create([_product(out, t.w_out[layer], y) for t, out, y in zip(tenants, self.out, self.y)])
            self.layers.append((into, attend, out_of))

    def run(self, stream):
        """self.x in, self.x out."""
        for into, attend, out_of in self.layers:
            sk_launch(into, stream)
            sk_attn_append(attend, stream)
            sk_attn_launch(attend, stream)
            sk_launch(out_of, stream)
            for x, y in zip(self.x, self.y):
                x += y

    def close(self):
        for plans in self.layers:
            for p in plans:
                p.close()


def grow(t, sequences, tokens, rows, stream):
    """Room for the sequences' tokens, and the step's numbers: `rows` new rows of each sequence."""
    sk_pages_resize(t.account, sequences, tokens)
    sk_pages_apply(t.account, t.arrays, t.table.data_ptr(), stream)
    held = [sk_pages_state(t.account, s)[0] for s in range(t.sequences)]
    first = [0]
    for n in rows:
        first.append(first[-1] + n)
    t.lengths.copy_(torch.tensor(held, dtype=torch.int32))
    t.first_row.copy_(torch.tensor(first, dtype=torch.int32))


def unit(x):
    return (x.float() / x.float().square().mean(-1, keepdim=True).sqrt().clamp(min=1e-6)).to(DTYPE)


def serve(tenants, prompts, children, steps, stream, seen=None):
    """Prompts (hidden states per tenant), a fork into `children` continuations, then `steps` tokens for each.  Returns the continuations' last hidden
    states per tenant, seconds of the prompts and of a step.  seen(step) is called behind each step, 0 for the prompts."""
    first = Step(tenants, [p.shape[0] for p in prompts], max(p.shape[0] for p in prompts))
    for t, x, p in zip(tenants, first.x, prompts):
        x.copy_(p)
        grow(t, [0], [p.shape[0]], [p.shape[0]] + [0] * (t.sequences - 1), stream)
    torch.cuda.synchronize()
    begin = time.perf_counter()
    first.run(stream)
    torch.cuda.synchronize()
    prompt_s = time.perf_counter() - begin
    if seen:
        seen(0)
    for t in tenants:
        sk_pages_fork(t.account, 0, range(1, children))
    each = Step(tenants, [children] * len(tenants), 1)
    for t, x, last in zip(tenants, each.x, first.x):
        x.copy_(last[-1:].expand(children, -1))
    begin = time.perf_counter()
    for n in range(steps):
        for t, x, p in zip(tenants, each.x, prompts):
            x.copy_(unit(x))
            grow(t, list(range(children)), [p.shape[0] + n + 1] * children, [1] * children + [0] * (t.sequences - children), stream)
        each.run(stream)
        if seen:
            seen(n + 1)
    torch.cuda.synchronize()
    step_s = (time.perf_counter() - begin) / max(steps, 1)
    last = [x.clone() for x in each.x]
    torch.cuda.synchronize()
    first.close()
    each.close()
    return last, prompt_s, step_s


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("tenants", 4), ("layers", 2), ("prompt", 500), ("children", 4), ("steps", 32)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args(argv)
    kinds = [(768, (12, 12, 64), 0, 0), (2048, (16, 4, 128), 0, 0), (1024, (16, 4, 80), 256, 4)]
    tenants = [Tenant(h, heads, a.layers, a.children, a.prompt + 64 + a.steps, window=w, sinks=s, seed=i)
               for i, (h, heads, w, s) in ((i, kinds[i % len(kinds)]) for i in range(a.tenants))]
    g = torch.Generator(device="cuda").manual_seed(99)
    prompts = [unit(torch.randn((a.prompt + 7 * i, t.hidden), generator=g, device="cuda")) for i, t in enumerate(tenants)]
    stream = torch.cuda.current_stream().cuda_stream
    last, prompt_s, step_s = serve(tenants, prompts, a.children, a.steps, stream)
    rows = sum(p.shape[0] for p in prompts)
    print(f"{a.tenants} tenants, {a.layers} layers: prompts of {rows} rows {prompt_s * 1e3:.2f} ms; {a.children} continuations of each, {a.steps} steps, "
          f"{step_s * 1e3:.3f} ms a step")
    for i, (t, x) in enumerate(zip(tenants, last)):
        free, _ = sk_pages_state(t.account)
        print(f"  tenant {i}: {t.hq}/{t.hkv} heads of {t.d}, {t.pages - free} pages for {a.children} sequences of {t.lengths[0].item()} tokens, "
              f"last hidden states of size {x.float().square().mean().sqrt().item():.3f}")


if __name__ == "__main__":
    main()
