"""Norms, mixture-of-experts layers and verification where their arithmetic and their rules of choice end: arguments far from 0, numbers of rows and vocabularies at
both ends, the types' lowest values."""
import copy

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
