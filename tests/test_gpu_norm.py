"""Norms around a block against 64 bits: lengths of rows from 1 to 32768, types, strides, gates, what is missing, rows counted on the device."""
import pytest
import torch

import paper_1901_10008_amd as sk
import layer_harness as H

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim", [1, 2, 7, 8, 9, 15, 96, 511, 513, 768, 1283, 2047, 2048, 2049, 2056, 4096, 5120, 8191, 8192, 8193, 8200, 20001, 32768])
def test_lengths(dim):
    H.check_norms([H.Norm(dim=dim, rows=3, post=1, gate="rows", act="sigmoid", stream="f32", seed=dim),
                   H.Norm(dim=dim, rows=2, dtype="f16", kind="layer", post=1, biases=True, gate="one", seed=dim + 1),
                   H.Norm(dim=dim, rows=2, dtype="f32", kind="layer", gate="rows", act="tanh", seed=dim + 2)], f"dim {dim}")


@pytest.mark.parametrize("dim", [1, 8, 100, 255, 256, 257, 768, 1024, 1025, 1283, 2048])
def test_many_rows(dim):
    H.check_norms([H.Norm(dim=dim, rows=2051, post=1, stream="f32", seed=dim), H.Norm(dim=dim, rows=2050, dtype="f16", kind="layer", post=1, biases=True, gate="rows", act="silu", used=2049, seed=dim)])


@pytest.mark.parametrize("dtype,stream", [("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("gate,act", [(None, "none"), ("rows", "none"), ("one", "sigmoid"), ("rows", "silu"), ("one", "tanh"), ("rows", "gelu"), ("rows", "relu")])
def test_types_and_gates(dtype, stream, kind, gate, act):
    H.check_norms([H.Norm(dtype=dtype, stream=stream, kind=kind, gate=gate, act=act, post=post, biases=post == 0, dim=200 + 3 * post, rows=5, pad=7 * post) for post in (0, 1)])


def test_small_values_of_tanh():
    """Near 0 tanh is its argument: relative errors stay small where 2 / (1 + e^-2z) - 1 would lose all digits."""
    n = H.Norm(dtype="f32", dim=64, rows=4, gate="rows", act="tanh", residual=False, bs=1.0)
    n.gate.copy_(torch.tensor([1e-30, 1e-8, 1e-3, 0.2, 0.2499999, 0.25, 0.2500001, -0.1], device="cuda").repeat(4, 8))
    want = n.block.double() * torch.tanh(n.gate.double())
    with sk.sk_norm_plan_create([n.problem()]) as plan:
        sk.sk_norm_launch(plan, H.stream_handle())
        torch.cuda.synchronize()
    H.check(n.residual_out, want, 44 * H.E * want.abs() + H.TINY["f32"])


@pytest.mark.parametrize("what", [dict(block=False), dict(residual=False), dict(residual_out=False), dict(next=False), dict(weights=False), dict(weights=False, biases=True), dict(rs=0.0, bs=0.0),
                                  dict(eps=0.0), dict(in_place=True), dict(in_place=True, stream="f32", pad=5)])
@pytest.mark.parametrize("dim", [72, 1283, 9000])
def test_what_is_missing_or_in_place(what, dim):
    n = H.Norm(dim=dim, rows=4, post=1, gate="rows", act="silu", used=3, **what)
    if what.get("rs") == 0.0:
        n2 = H.Norm(dim=dim, rows=4, post=1, gate="rows", act="silu", used=3, rs=0.0, bs=0.0)
        n2.rs = n2.bs = 1.0  # a scale of 0 means 1
        want, _ = n2.reference()
        with sk.sk_norm_plan_create([n.problem()]) as plan:
            sk.sk_norm_launch(plan, H.stream_handle())
            torch.cuda.synchronize()
        n.rs = n.bs = 1.0
        (r, y), (tr, ty) = n.reference()
        H.check(n.residual_out[:3], r, tr)
        assert torch.equal(r, want[0])
        return
    H.check_norms([n])


@pytest.mark.parametrize("used", [-5, 0, 1, 6, 7, 100])
def test_rows_counted_on_the_device(used):
    H.check_norms([H.Norm(dim=100, rows=7, used=used), H.Norm(dim=9001, rows=7, used=used, stream="f32"), H.Norm(dim=64, rows=2100, used=used)])


def test_many_problems_of_all_forms():
    H.check_norms([H.Norm(dim=(64, 3000, 10000)[i % 3] + i, rows=(3 + i, 2, 1, 2048)[i % 4], dtype=("bf16", "f16", "f32")[i % 3], kind=("rms", "layer")[i % 2], seed=i) for i in range(40)])
    with sk.sk_norm_plan_create([]) as plan:
        sk.sk_norm_launch(plan, H.stream_handle())


def test_a_row_keeps_its_nan_to_itself():
    n, clean = H.Norm(dim=300, rows=6, post=1), H.Norm(dim=300, rows=6, post=1)
    n.block[2, 17], n.block[4, 3] = float("nan"), float("inf")
    for x in (n, clean):
        with sk.sk_norm_plan_create([x.problem()]) as plan:
            sk.sk_norm_launch(plan, H.stream_handle())
            torch.cuda.synchronize()
    for row in (0, 1, 3, 5):
        assert torch.equal(n.next[row], clean.next[row]) and torch.equal(n.residual_out[row], clean.residual_out[row])
    assert torch.isnan(n.next[2]).all() and torch.isnan(n.next[4]).any()


@pytest.mark.parametrize("dim", [24, 200, 700, 1501])
def test_many_rows_in_place_and_their_nan(dim):
    """Several rows of a wave or workgroup: each reads and writes its own alone."""
    H.check_norms([H.Norm(dim=dim, rows=2100, post=1, gate="rows", act="silu", in_place=True, used=2093, pad=3, seed=dim)])
    n, clean = (H.Norm(dim=dim, rows=2100, kind="layer", post=1, seed=1) for _ in range(2))
    n.block[2, dim // 2], n.block[6, 3], n.residual[2099, dim - 1] = float("nan"), float("inf"), float("nan")
    for x in (n, clean):
        with sk.sk_norm_plan_create([x.problem()]) as plan:
            sk.sk_norm_launch(plan, H.stream_handle())
            torch.cuda.synchronize()
    others = torch.ones(2100, dtype=torch.bool, device="cuda")
    others[[2, 6, 2099]] = False
    assert torch.equal(n.next[others], clean.next[others]) and torch.equal(n.residual_out[others], clean.residual_out[others])
    assert torch.isnan(n.next[~others]).any(1).all()


def test_more_than_the_caches_hold():
    """Loads and stores past the caches: 190 MB, against the same rows in launches that fit the caches (the same bits) and 64 bits."""
    big = H.Norm(dim=2056, rows=10000, post=1, stream="f32", gate="rows", act="sigmoid", seed=3)
    with sk.sk_norm_plan_create([big.problem()]) as plan:
        sk.sk_norm_launch(plan, H.stream_handle())
        torch.cuda.synchronize()
    (r, y), (tr, ty) = big.reference()
    H.check(big.residual_out, r, tr)
    H.check(big.next, y, ty)


def test_captured_and_on_another_stream():
    n = H.Norm(dim=500, rows=9, post=1, stream="f32", used=4)
    with sk.sk_norm_plan_create([n.problem()]) as plan:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        sk.sk_norm_launch(plan, side.cuda_stream)
        side.synchronize()
        (r, y), (tr, ty) = n.reference()
        H.check(n.next[:4], y, ty)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            sk.sk_norm_launch(plan, torch.cuda.current_stream().cuda_stream)
        for used in (9, 2, 0, 5):
            n.n_rows.fill_(used)
            n.block.mul_(0.5)
            n.next_b.fill_(float("nan"))
            n.used = used
            graph.replay()
            torch.cuda.synchronize()
            (r, y), (tr, ty) = n.reference()
            H.check(n.residual_out[:used], r, tr)
            H.check(n.next[:used], y, ty)
            assert torch.isnan(n.next_b[used:]).all()
        del graph
