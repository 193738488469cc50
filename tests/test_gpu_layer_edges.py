"""Norms, mixture-of-experts layers and verification where their arithmetic and their rules of choice end: arguments far from 0, numbers of rows and vocabularies at
both ends, the types' lowest values."""
import copy
import threading

import pytest
import torch

import paper_1901_10008_amd as sk
import layer_harness as H

pytestmark = pytest.mark.gpu

ACTS = ["none", "sigmoid", "silu", "tanh", "gelu", "relu"]


def far_from_zero():
    """Finite arguments of all sizes, many of them where e^-t passes the largest number of 32 bits: t = -88.8, which is z = -44.4 (tanh) and about -10 (gelu)."""
    line = lambda a, b, n: torch.linspace(a, b, n, device="cuda", dtype=torch.float64)  # noqa: E731
    z = torch.cat([line(-1e4, 1e4, 801), line(-120, -80, 641), line(-60, -40, 321), line(-16, -9, 449), line(80, 120, 161), line(9, 60, 205)])
    return torch.cat([z, torch.tensor([s * v for v in (1e5, 1e8, 1e15, 1e25, 1e30) for s in (1, -1)], device="cuda", dtype=torch.float64)])


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_gates_far_from_zero(act, dtype):
    z = far_from_zero().to(H.TORCH[dtype])
    z = z[torch.isfinite(z)]
    n = H.Norm(dtype=dtype, stream="f32", dim=z.numel(), rows=1, gate="one", act=act, residual=False, next=False, bs=1.0)
    n.gate = z
    u, z = n.block.double(), z.double()
    y, _ = H.activated(act, z)
    # As in the harness; but an argument t of the exponential counts up to 200, since 1 / (1 + e^-t) is 0 or 1 to 2^-126 beyond, and what fp32 arithmetic may take as 0
    # (below 2^-126) is multiplied by z.
    t = {"tanh": 2 * z, "gelu": 1.6 * (z + 0.045 * z ** 3)}.get(act, z).abs().clamp(max=200)
    tol = 4 * H.E * (10 + t) * y.abs() + 2.0 ** -126 * (1 + z.abs()) if act not in ("none", "relu") else torch.zeros_like(z)
    with sk.sk_norm_plan_create([n.problem()], keepalive=n) as plan:
        sk.sk_norm_launch(plan, H.stream_handle())
        torch.cuda.synchronize()
    # (three roundings behind it: the product, the scale of 1, the output)
    H.check(n.residual_out, u * y, u.abs() * tol + 3 * H.E * (u * y).abs() + H.TINY["f32"], f"{act} {dtype}")


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_experts_activations_far_from_zero(act, gated, dtype):
    """What goes into the activations is spread over +- 100 and over +- 1000: every row meets what lies beyond the exponential's range."""
    for spread in (40.0, 400.0):
        m = H.Moe(rows=19, dim=64, ffn=48, act=act, dtype=dtype, gated=gated, shared=40, top_k=3, seed=int(spread))
        for w in [m.gate_b if gated else m.up_b, m.s[0] if gated else m.s[1]]:
            w.mul_(spread)
        H.run_moe([m], f"{act} {spread}")


def check_many(v, label):
    """As H.check_verify, with the reference on the host: so many short rows are many small steps."""
    host = copy.copy(v)
    for name, x in vars(v).items():
        if torch.is_tensor(x):
            setattr(host, name, x.cpu())
    tokens, accepted = host.reference()
    with sk.sk_verify_plan_create([v.problem()], keepalive=v) as plan:
        for turn in range(2):
            v.tokens.fill_(-9), v.accepted.fill_(-9)
            sk.sk_verify_launch(plan, H.stream_handle())
            torch.cuda.synchronize()
            assert v.accepted.tolist() == accepted, f"{label} launch {turn}: accepted"
            assert v.tokens.tolist() == tokens, f"{label} launch {turn}: tokens"


@pytest.mark.parametrize("vocab", [1, 3, 7, 8, 9, 513])
@pytest.mark.parametrize("draft,rows", [("logits", 3001), ("certain", 6001), ("none", 6001)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_rows_of_short_vocabularies(vocab, draft, rows, dtype):
    """So many rows that longer ones go in chunks of several pieces; padded with NaN, so that what is read beside a row is seen."""
    counts = [3] * (rows // 3) + [rows % 3]
    check_many(H.Verify(dtype=dtype, vocab=vocab, counts=counts, draft=draft, spread=0.7, pad=4, seed=vocab + rows), f"{vocab} {draft} {dtype}")


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("temperature", [1.0, 0.7, 1e-3, 1e30, 0.0])
def test_logits_of_the_types_lowest_value(dtype, temperature):
    """A usual mask: the lowest finite value.  Rows of it alone are uniform, whole chunks, pieces and lanes of it beside other logits count (almost) nothing."""
    lowest = torch.finfo(H.TORCH[dtype]).min
    for draft in ("logits", "certain"):
        v = H.Verify(dtype=dtype, vocab=5000, counts=(2,) * 12 + (1, 1), draft=draft, temperature=temperature, seed=21)
        v.accept_random.uniform_(0.0, 1e-3, generator=H.generator(5))  # a p of 1/5000 is accepted one time in five
        for row, (first, last) in enumerate([(0, 5000), (0, 5000), (0, 512), (512, 1024), (100, 4900), (0, 4999), (1, 5000), (8, 16), (2048, 5000), (3, 4096)]):
            v.logits[row, first:last] = lowest
        v.logits[10, :] = lowest
        v.logits[10, 4000:] = -float("inf")
        v.logits[24:26, :] = lowest
        if v.draft_logits is not None:
            for row, (first, last) in {0: (0, 5000), 2: (0, 5000), 4: (0, 5000), 12: (0, 5000), 14: (17, 4500), 16: (512, 5000)}.items():
                v.draft_logits[row, first:last] = lowest
        H.check_verify([v], f"{draft} {temperature}")


def test_many_rows_of_the_lowest_value_in_larger_chunks():
    v = H.Verify(dtype="f32", vocab=4500, counts=(1,) * 3001, draft="none", seed=22)
    v.logits[::2] = torch.finfo(torch.float32).min
    v.logits[1::4, 700:] = torch.finfo(torch.float32).min
    check_many(v, "lowest")


@pytest.mark.parametrize("used", [-2 ** 31, -2 ** 31 + 1, -2 ** 31 + 511, -2 ** 31 + 512, -2 ** 31 + 1023, -513, -1, 2 ** 31 - 1])
def test_numbers_of_rows_at_the_ends_of_their_type(used):
    """A layer of more rows than are routed together: none of its parts has rows that the number does not give."""
    m = H.Moe(rows=1100, dim=32, experts=4, top_k=2, ffn=16, shared=8, used=used)
    H.run_moe([m], f"{used}")
    H.check_norms([H.Norm(dim=100, rows=7, used=used), H.Norm(dim=64, rows=2100, used=used)], f"{used}")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rows", [1, 5, 12, 40, 100])
@pytest.mark.parametrize("ffn", [16, 264, 1032])
def test_nothing_is_rounded_between_the_products(dtype, rows, ffn):
    """Whole numbers of up to 20 bits between the products, in pairs that differ by at most 63, and the second products take their differences: any rounding to fewer than 20 bits
    is seen.  All sums of 32 bits are exact (16 numbers below 2^19 times +-1)."""
    g = torch.Generator().manual_seed(rows + ffn)
    m = H.Moe(dtype=dtype, rows=rows, dim=64, ffn=ffn, experts=3, top_k=1, gated=False, act="none", shared=ffn, normalize=1)
    m.x.copy_(torch.randint(1, 64, (rows, 64), generator=g))

    def weights(up, down):  # (of an expert) the number at place 2 p + 1 is that at 2 p with one weight of x less by 1
        w = torch.randint(64, 128, (ffn, 64), generator=g)
        w[1::2] = w[::2]
        pairs = torch.arange(0, ffn, 2)
        w[pairs + 1, torch.randint(0, 64, (len(pairs),), generator=g)] -= 1
        up.copy_(w)
        down.zero_()
        for d in range(64):
            for p in torch.randperm(ffn // 2, generator=g)[:4].tolist():
                sign = 1 if p % 2 else -1
                down[d, 2 * p], down[d, 2 * p + 1] = sign, -sign

    for e in range(3):
        up, down = torch.empty((ffn, 64)), torch.empty((64, ffn))
        weights(up, down)
        m.up_b[e], m.down_b[e] = up.to(m.up_b.dtype), down.to(m.up_b.dtype)
    up, down = torch.empty((ffn, 64)), torch.empty((64, ffn))
    weights(up, down)
    m.s[1].copy_(up), m.s[2].copy_(down)
    with sk.sk_moe_plan_create([m.problem()], keepalive=m) as plan:
        sk.sk_moe_launch(plan, H.stream_handle())
        torch.cuda.synchronize()
    want = m.reference()[0]
    assert (want == want.round()).all() and float(want.abs().max()) <= 8 * 63  # eight pairs: those of the routed and of the shared expert
    assert torch.equal(m.out, want.to(m.out.dtype))  # (rounded once: what is above 256 may be odd)


@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("rows", [3, 14, 60])
def test_f16_between_the_products_beyond_its_range(gated, rows):
    """Numbers of 10^5 to 10^9 between the products, and of 2^-24 and less, where the outputs are ordinary."""
    large = H.Moe(dtype="f16", rows=rows, dim=64, ffn=48, shared=24, act="silu", gated=gated, experts=3, top_k=2, seed=1)
    small = H.Moe(dtype="f16", rows=rows, dim=64, ffn=48, shared=24, act="none", gated=gated, experts=3, top_k=2, seed=2)
    for m, first, second in ((large, 2.0 ** 13 if gated else 2.0 ** 14, 2.0 ** -20 if gated else 2.0 ** -10), (small, 2.0 ** -10 if gated else 2.0 ** -17, 2.0 ** 12)):
        for w in (m.gate_b, m.up_b, m.s[0], m.s[1]):
            if w is not None:
                w.mul_(first)
        for w in (m.down_b, m.s[2]):
            w.mul_(second)
        m.x.mul_(2.0 if m is large else 2.0 ** -5 if not gated else 2.0 ** -3)
    H.run_moe([large], "large")
    H.run_moe([small], "small")


@pytest.mark.parametrize("rows", [1, 30, 600])
def test_experts_over_their_input(rows):
    """out is x: nothing of it is written before all of it has been read, by tenants whose x is another's out too."""
    ms = [H.Moe(rows=rows, dim=64, ffn=40, experts=6, top_k=2, shared=16, pad=8, seed=s) for s in (1, 2)]
    wants = [m.reference() for m in ms]
    problems = [m.problem() for m in ms]
    problems[0].out, problems[1].out = ms[1].x.data_ptr(), ms[0].x.data_ptr()
    with sk.sk_moe_plan_create(problems, keepalive=ms) as plan:
        sk.sk_moe_launch(plan, H.stream_handle())
        torch.cuda.synchronize()
    for (out, tol, ids, w), m, at in zip(wants, ms, (ms[1].x, ms[0].x)):
        H.check(at, out, tol)
        assert torch.equal(m.ids.long(), ids)


def test_norms_launched_by_several_threads_at_once():
    n = H.Norm(dim=700, rows=40, post=1, stream="f32", gate="rows", act="silu")
    (r, y), (tr, ty) = n.reference()
    streams, failed = [torch.cuda.Stream() for _ in range(4)], []
    torch.cuda.synchronize()

    def work(plan, stream):
        try:
            for _ in range(200):
                sk.sk_norm_launch(plan, stream.cuda_stream)
        except Exception as e:  # noqa: BLE001
            failed.append(e)

    plan = sk.sk_norm_plan_create([n.problem()], keepalive=n)
    threads = [threading.Thread(target=work, args=(plan, s)) for s in streams]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    plan.close()  # (waits for all of them)
    assert not failed and all(s.query() for s in streams)
    H.check(n.residual_out, r, tr)
    H.check(n.next, y, ty)


@pytest.mark.parametrize("dim,rows", [(2056, 10000), (200, 100000), (768, 30000), (5000, 5000), (12000, 2000)])
def test_loads_and_stores_past_the_caches_give_the_same_bits(dim, rows):
    """A launch of more than 160 MiB, which goes past the caches, and its rows in launches that do not."""
    make = lambda: H.Norm(dim=dim, rows=rows, kind="layer", post=1, stream="f32", gate="rows", act="sigmoid", biases=True, seed=3)  # noqa: E731
    a, b = make(), make()
    assert rows * dim * (3 * 2 + 2 * 4) > 160 << 20
    with sk.sk_norm_plan_create([a.problem()], keepalive=a) as plan:
        sk.sk_norm_launch(plan, H.stream_handle())
        torch.cuda.synchronize()
    step = rows // 4 if dim > 2048 else max(2048, rows // 8)  # (of up to 2048 elements as many rows as give a plan of the same form)
    for at in range(0, rows, step):
        p, n = b.problem(), min(step, rows - at)
        if dim <= 2048 and n < 2048:
            at, n = rows - 2048, 2048
        p.rows = n
        for name, x in (("block", b.block), ("gate", b.gate), ("residual", b.residual), ("residual_out", b.residual_out), ("next", b.next)):
            setattr(p, name, x[at:].data_ptr())
        assert n * dim * (3 * 2 + 2 * 4) <= 160 << 20
        with sk.sk_norm_plan_create([p], keepalive=b) as plan:
            sk.sk_norm_launch(plan, H.stream_handle())
            torch.cuda.synchronize()
    assert torch.equal(a.residual_out, b.residual_out) and torch.equal(a.next, b.next)
    (r, y), (tr, ty) = a.reference()
    H.check(a.next, y, ty)


@pytest.mark.parametrize("rows,experts,top_k", [(512, 512, 32), (600, 33, 32), (65, 512, 32), (512, 3, 1), (2000, 128, 8)])
def test_most_choices(rows, experts, top_k):
    """More pairs of a row and an expert than the router keeps at hand, and as many as there can be."""
    H.run_moe([H.Moe(rows=rows, dim=16, ffn=8, experts=experts, top_k=top_k, scoring="sigmoid", bias=True, seed=rows), H.Moe(rows=3, dim=16, ffn=8, seed=1)], f"{rows} {experts}/{top_k}")


@pytest.mark.parametrize("dim,ffn", [(1 << 20, 8), (8, 1 << 20), (8200, 9000)])
def test_longest_rows_of_experts(dim, ffn):
    H.run_moe([H.Moe(rows=34, dim=dim, ffn=ffn, experts=2, top_k=1, shared=8, seed=1)], f"{dim} x {ffn}")


def test_two_layers_on_two_streams():
    ms = [H.Moe(rows=40, dim=256, ffn=128, experts=8, top_k=2, shared=64, seed=s) for s in (1, 2)]
    streams = [torch.cuda.Stream() for _ in ms]
    plans = [sk.sk_moe_plan_create([m.problem()], keepalive=m) for m in ms]
    torch.cuda.synchronize()
    for _ in range(50):
        for plan, stream in zip(plans, streams):
            sk.sk_moe_launch(plan, stream.cuda_stream)
    torch.cuda.synchronize()
    for m, plan in zip(ms, plans):
        H.check_moe(m)
        plan.close()


@pytest.mark.parametrize("counts,vocab,draft", [((1200,), 40, "logits"), ((700, 1, 700), 30, "certain"), ((3,) * 5000, 9, "certain"), ((2, 0, 1), 1 << 20, "logits"), ((300, 300), 2049, "logits")])
def test_long_and_many_sequences(counts, vocab, draft):
    v = H.Verify(dtype="f32", vocab=vocab, counts=counts, draft=draft, seed=31)
    if draft == "logits":
        v.draft_logits.copy_(v.logits)  # (all but a few are accepted)
        v.draft_logits[-3:] += H.randn(H.generator(1), 3, vocab)
    else:
        v.logits.scatter_add_(1, v.drafted.long()[:, None], torch.full((v.rows, 1), 9.0, device="cuda"))
    check_many(v, f"{len(counts)} x {vocab}")


def test_rows_far_apart():
    """Rows further apart than 2^31 elements, and more rows than 2^16."""
    n = H.Norm(dim=40, rows=3, post=1, gate="rows", act="silu")
    stride = (1 << 31) + 8
    far = torch.zeros(2 * stride + 40, dtype=torch.bfloat16, device="cuda")
    for row in range(3):
        far[row * stride:row * stride + 40] = n.block[row]
    p = n.problem()
    p.block, p.block_stride = far.data_ptr(), stride
    (r, y), (tr, ty) = n.reference()
    with sk.sk_norm_plan_create([p], keepalive=(n, far)) as plan:
        sk.sk_norm_launch(plan, H.stream_handle())
        torch.cuda.synchronize()
    H.check(n.residual_out, r, tr)
    H.check(n.next, y, ty)
    del far
    H.check_norms([H.Norm(dim=8, rows=1 << 20, seed=1), H.Norm(dim=1, rows=70000, kind="layer", seed=2), H.Norm(dim=300, rows=100001, used=99999, seed=3)])


@pytest.mark.parametrize("rows", [4, 13, 50])
def test_infinity_and_the_largest_numbers_between_the_products(rows):
    """One row is infinite between the products, one has numbers there that bf16 could only round to infinity: the first's outputs are infinite (no NaN), the second's as large as
    they should be, and the others' what they are without those two."""
    m, clean = (H.Moe(rows=rows, dim=64, ffn=48, experts=3, top_k=1, act="none", gated=False, seed=5) for _ in range(2))  # (one choice: with two, the second's weight is 0)
    for x in (m, clean):
        x.up_b.abs_(), x.down_b.abs_()
    m.x[1], m.x[2] = 2.0 ** 127, 0.0
    clean.x[2] = 0.0
    m.x[2, 0] = 2.0 ** 127
    m.up_b[:, :, 0] = 2.0 - 2.0 ** -7  # (the largest of bf16)
    m.up_b[:, :, 1] = 2.0 ** -7 - 2.0 ** -13
    m.x[2, 1] = 2.0 ** 127  # their sum: 2^128 less 2^114, between the largest of bf16 and that of 32 bits
    m.down_b.mul_(2.0 ** -10)
    clean.up_b.copy_(m.up_b), clean.down_b.copy_(m.down_b)
    for x in (m, clean):
        with sk.sk_moe_plan_create([x.problem()], keepalive=x) as plan:
            sk.sk_moe_launch(plan, H.stream_handle())
            torch.cuda.synchronize()
    out, tol, _, _ = m.reference()
    assert torch.isposinf(m.out[1]).all()
    H.check(m.out[2], out[2], tol[2])
    others = [r for r in range(rows) if r not in (1, 2)]
    assert torch.equal(m.out[others], clean.out[others])
