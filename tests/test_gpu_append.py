"""Norm, rotation and append against the formula in 64 bits (cache_harness.Tenant.append), and copies of pages."""
import math

import numpy as np
import pytest
import torch

import paper_1901_10008_amd as sk

import cache_harness as H
from cache_harness import Tenant

pytestmark = pytest.mark.gpu

STEP = ((1, 1), (0, 0), (17, 1), (31, 3), (64, 0), (40, 40), (3, 1), (100, 33), (65, 1))


def check_append(tenants, label=""):
    problems = [t.to_device() for t in tenants]
    for t in tenants:
        t.dq.fill_(math.nan)
    with sk.sk_attn_plan_create(problems) as plan:
        sk.sk_attn_append(plan, H.stream_handle())
        torch.cuda.synchronize()
    for i, t in enumerate(tenants):
        (q, k, v), (tq, tk) = t.append()
        n = t.rows_used
        H.assert_close(t.dq[:n, :, :t.d].cpu(), q[:n], tq[:n], f"{label} tenant {i} queries")
        assert torch.isnan(t.dq[n:]).all() and (not t.q_pad or torch.isnan(t.dq[..., t.d:]).all()), f"{label} tenant {i}: written beyond the rows"
        got_k, got_v = t.cache()
        H.assert_close(got_k, k, tk, f"{label} tenant {i} keys")
        assert torch.equal(got_v.contiguous().view(torch.int16), v.contiguous().view(torch.int16)), f"{label} tenant {i}: values differ"


def tenant(*a, **kw):
    return Tenant(*a, with_qkv=True, with_out=False, **kw)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim,rotary", [(8, 8), (64, 64), (64, 32), (64, 20), (72, 2), (80, 80), (96, 48), (128, 128), (128, 0), (136, 100), (256, 256), (256, 6)])
@pytest.mark.parametrize("neighbours", [False, True])
def test_sizes(dtype, dim, rotary, neighbours):
    check_append([tenant(dtype, (4, 2, dim), STEP, rotary=rotary, neighbours=neighbours, seed=dim + rotary)], f"{dtype} {dim} {rotary}")


@pytest.mark.parametrize("heads", [(1, 1, 64), (12, 12, 64), (32, 8, 128), (7, 1, 80), (3, 3, 256)])
@pytest.mark.parametrize("norm", [False, True])
def test_heads_with_and_without_norm(heads, norm):
    check_append([tenant("bf16", heads, STEP, rotary=heads[2] // 2, norm=norm, seed=1)], f"{heads} {norm}")


@pytest.mark.parametrize("layout", ["page", "token", "heads"])
def test_layouts_and_strides(layout):
    check_append([tenant("f16", (4, 2, 80), STEP, page=32, layout=layout, q_pad=8, spare_rows=7, rotary=40, seed=2)], layout)


def test_prompts_take_several_heads_a_wave():
    check_append([tenant("bf16", (8, 2, 64), ((700, 700), (1, 1), (333, 300)), page=64, rotary=64, seed=3), tenant("f16", (2, 1, 128), STEP, rotary=128, seed=4)], "prompts")


def test_new_tokens_beyond_the_bound_of_attention_are_appended():
    check_append([tenant("bf16", (4, 2, 64), ((50, 9), (60, 3)), rotary=64, max_new=2, seed=10)], "max_new")


def test_many_sequences_and_several_tenants():
    seqs = tuple((1 + i % 50, i % 2) for i in range(5000))
    check_append([tenant("bf16", (1, 1, 8), seqs, rotary=8, seed=5)] + [tenant("f16", (2, 1, 16), STEP, rotary=16, seed=i) for i in range(70)], "many")


def test_rows_before_the_sequence_and_pages_that_are_none():
    """More new rows than tokens: the first of them are not appended.  Page numbers outside the cache: neither."""
    t = tenant("bf16", (4, 2, 64), ((3, 9), (50, 2), (40, 40)), rotary=64, seed=6)
    t.table[1, 3], t.table[2, 1] = -1, 1 << 29
    check_append([t], "absent")


def test_zeros_and_large_values():
    t = tenant("bf16", (4, 2, 64), ((5, 3),), rotary=64, eps=1e-6, seed=7)
    t.qkv[0] = 0
    t.qkv[1] *= 2.0 ** 40
    t.qkv[2] *= 2.0 ** -30
    check_append([t], "zeros and large values")


@pytest.mark.parametrize("neighbours", [False, True])
def test_infinite_elements_touch_their_pair_alone(neighbours):
    t = tenant("bf16", (4, 2, 64), ((5, 2),), rotary=32, neighbours=neighbours, norm=False, seed=9)
    want_t = tenant("bf16", (4, 2, 64), ((5, 2),), rotary=32, neighbours=neighbours, norm=False, seed=9)
    t.qkv[0, :, 40], t.qkv[1, :, 3] = math.inf, -math.inf
    problem = t.to_device()
    with sk.sk_attn_plan_create([problem]) as plan:
        sk.sk_attn_append(plan, H.stream_handle())
        torch.cuda.synchronize()
    (q, k, v), (tq, tk) = want_t.append()
    got = t.dq.cpu().double()
    pair = [3, 2] if neighbours else [3, 19]
    assert (got[0, :, 40] == math.inf).all() and not torch.isfinite(got[1][:, pair]).any()
    for row, odd in ((0, [40]), (1, pair)):
        fine = [e for e in range(64) if e not in odd]
        H.assert_close(got[row][:, fine], q[row][:, fine], tq[row][:, fine], f"row {row}")


def test_append_then_attend_as_a_step():
    """The queries that append has written are attend's, and the keys and values it has appended are seen."""
    t = Tenant("bf16", (4, 2, 64), STEP, with_qkv=True, rotary=64, window=30, sinks=2, seed=8)
    problem = t.to_device()
    t.dq.fill_(math.nan)
    with sk.sk_attn_plan_create([problem]) as plan:
        sk.sk_attn_append(plan, H.stream_handle())
        sk.sk_attn_launch(plan, H.stream_handle())
        torch.cuda.synchronize()
    t.q, (t.k, t.v) = t.dq.cpu(), t.cache()
    want, tol = t.attend()
    H.assert_close(t.out()[:t.rows_used], want[:t.rows_used], tol[:t.rows_used])


# ---- copies of pages -----------------------------------------------------------------------------------------------------------

def arrays_of(tensors):
    return sk.make_page_arrays([(x.data_ptr(), x[0].numel() * x.element_size()) for x in tensors])


@pytest.mark.parametrize("sizes", [(16,), (48, 4096), (32768, 32784, 16), (100000 * 16,)])
def test_copies(sizes):
    n = 23
    tensors = [torch.randint(0, 256, (n, s), dtype=torch.uint8, device="cuda") for s in sizes]
    want = [x.clone() for x in tensors]
    frm, to = [0, 0, 5, 7, 21], [1, 2, 22, 3, 9]
    for w in want:
        w[to] = w[frm]
    sk.sk_pages_copy(arrays_of(tensors), n, frm, to, H.stream_handle())
    torch.cuda.synchronize()
    for x, w in zip(tensors, want):
        assert torch.equal(x, w)


def test_launches_that_go_past_the_caches():
    """More than 160 MiB in a launch: copies, and an append whose rows have room for as much."""
    n = 50
    x = torch.randint(0, 256, (n, 4 << 20), dtype=torch.uint8, device="cuda")
    want = x.clone()
    frm, to = list(range(0, 25)), list(range(25, 50))
    want[to] = want[frm]
    sk.sk_pages_copy(arrays_of([x]), n, frm, to, H.stream_handle())
    torch.cuda.synchronize()
    assert torch.equal(x, want)
    t = tenant("bf16", (32, 8, 128), ((130, 100), (20, 20)), rotary=128, spare_rows=8000, seed=4)
    check_append([t], "past the caches")


def test_more_arrays_and_copies_than_a_launch_holds():
    n, g = 2001, torch.Generator().manual_seed(1)
    tensors = [torch.randint(0, 256, (n, 32), dtype=torch.uint8, device="cuda") for _ in range(150)]
    order = torch.randperm(n, generator=g)
    frm, to = order[:1000].tolist(), order[1000:2000].tolist()
    want = [x.clone() for x in tensors]
    for w in want:
        w[to] = w[frm]
    sk.sk_pages_copy(arrays_of(tensors), n, frm, to, H.stream_handle())
    torch.cuda.synchronize()
    assert all(torch.equal(x, w) for x, w in zip(tensors, want))


def test_copies_of_more_workgroups_than_a_launch_can_have():
    """Large pages in one of many arrays: 2048 chunks x 64 arrays x 130 copies are more than 2^24 workgroups."""
    n, moves = 140, 130
    big = torch.empty((n, 64 << 20), dtype=torch.uint8, device="cuda")
    for i in range(n):
        big[i] = i
        big[i, -16:] = torch.arange(16, dtype=torch.uint8, device="cuda") + i
    small = [torch.randint(0, 256, (n, 48), dtype=torch.uint8, device="cuda") for _ in range(63)]
    frm, to = [i % 10 for i in range(moves)], list(range(10, 10 + moves))
    want = [x.clone() for x in small]
    for w in want:
        w[to] = w[frm]
    sk.sk_pages_copy(arrays_of([big] + small), n, frm, to, H.stream_handle())
    torch.cuda.synchronize()
    for f, t in zip(frm, to):
        assert torch.equal(big[t], big[f]) and int(big[f, 5]) == f and int(big[f, -1]) == f + 15
    assert all(torch.equal(x, w) for x, w in zip(small, want))


def test_more_rows_of_the_table_than_a_launch_can_have_workgroups():
    seqs = (1 << 24) + 5
    table = torch.full((seqs, 1), -7, dtype=torch.int32, device="cuda")
    with sk.sk_pages_create(3, 16, seqs, 1) as account:
        sk.sk_pages_resize(account, [0, 77, seqs - 1], [1, 2, 3])
        sk.sk_pages_apply(account, arrays_of([torch.zeros((3, 16), dtype=torch.uint8, device="cuda")]), table.data_ptr(), H.stream_handle())
        torch.cuda.synchronize()
        assert [int(table[s, 0]) for s in (0, 77, seqs - 1)] == [0, 1, 2] and int((table == -1).sum()) == seqs - 3


def test_copies_in_a_graph():
    x = torch.arange(10 * 64, dtype=torch.int32, device="cuda").view(10, 64)
    arrays = arrays_of([x])
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        sk.sk_pages_copy(arrays, 10, [0, 1], [8, 9], torch.cuda.current_stream().cuda_stream)
    for i in range(3):
        x.random_()
        want = x.clone()
        want[[8, 9]] = want[[0, 1]]
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(x, want)


def test_account_and_device_agree_under_random_calls():
    """Every sequence's tokens, written as numbers into its pages, stay readable through the device's table whatever is forked, grown, freed
    and compacted, with apply now and then."""
    rng = np.random.default_rng(3)
    pages, page, seqs, columns = 60, 4, 9, 12
    pool = torch.zeros((pages, page * 4), dtype=torch.int32, device="cuda")  # 4 numbers a token: 64 bytes a page
    other = torch.zeros((pages, page * 8), dtype=torch.int32, device="cuda")
    table = torch.full((seqs, columns), -5, dtype=torch.int32, device="cuda")
    arrays = arrays_of([pool, other])
    want = {s: [] for s in range(seqs)}
    account = sk.sk_pages_create(pages, page, seqs, columns)
    count, deepest = 0, 0
    for step in range(300):
        for _ in range(int(rng.integers(1, 4))):
            what, s = rng.random(), int(rng.integers(seqs))
            try:
                if what < 0.25:
                    empty = [t for t in range(seqs) if not want[t] and t != s][:2]
                    sk.sk_pages_fork(account, s, empty)
                    for t in empty:
                        want[t] = list(want[s])
                elif what < 0.45:
                    n = int(rng.integers(0, len(want[s]) + 1))
                    sk.sk_pages_resize(account, [s], [n])
                    want[s] = want[s][:n]
                elif what < 0.55:
                    sk.sk_pages_compact(account)
                else:
                    both = sorted({s, int(rng.integers(seqs))})
                    more = [min(len(want[t]) + int(rng.integers(1, 9)), page * columns) for t in both]
                    sk.sk_pages_resize(account, both, more)
                    for t, n in zip(both, more):
                        want[t] += [None] * (n - len(want[t]))
            except sk.SkError as e:
                assert e.status == sk.SK_ERR_ALLOC
        deepest = max(deepest, sk.sk_pages_state(account)[1])
        sk.sk_pages_apply(account, arrays, table.data_ptr(), H.stream_handle())
        # new tokens are written to their places
        for s in range(seqs):
            tokens, row = sk.sk_pages_state(account, s)
            assert tokens == len(want[s])
            for i, w in enumerate(want[s]):
                if w is None:
                    count += 1
                    want[s][i] = count
                    pool[row[i // page], 4 * (i % page):4 * (i % page) + 4] = count
                    other[row[i // page], 8 * (i % page):8 * (i % page) + 8] = -count
        if step % 10 == 0:
            t, p, o = table.cpu(), pool.cpu(), other.cpu()
            for s in range(seqs):
                tokens, row = sk.sk_pages_state(account, s)
                assert t[s].tolist() == row
                for i, w in enumerate(want[s]):
                    assert (p[row[i // page], 4 * (i % page):4 * (i % page) + 4] == w).all() and (o[row[i // page], 8 * (i % page):8 * (i % page) + 8] == -w).all()
    assert deepest > 2
    torch.cuda.synchronize()
    account.close()


@pytest.mark.parametrize("columns", [6, 600])
def test_rows_wait_for_a_table(columns):
    """Calls without a page table make the copies alone: rows changed by then come with the next call that has one."""
    pool = torch.arange(50 * 4, dtype=torch.int32, device="cuda").view(50, 4)
    table = torch.full((5, columns), -7, dtype=torch.int32, device="cuda")
    arrays = arrays_of([pool])
    with sk.sk_pages_create(50, 16, 5, columns) as account:
        sk.sk_pages_resize(account, [0], [40])
        sk.sk_pages_apply(account, arrays, 0, H.stream_handle())
        sk.sk_pages_fork(account, 0, [1, 3])
        sk.sk_pages_resize(account, [1, 3], [41, 41])
        assert sk.sk_pages_state(account)[1] == 2
        sk.sk_pages_apply(account, arrays, 0, H.stream_handle())
        assert sk.sk_pages_state(account)[1] == 0
        torch.cuda.synchronize()
        assert (table == -7).all() and torch.equal(pool[3:5], pool[2].expand(2, 4))
        sk.sk_pages_apply(account, arrays, table.data_ptr(), H.stream_handle())
        torch.cuda.synchronize()
        assert table.cpu().tolist() == [sk.sk_pages_state(account, s)[1] for s in range(5)]
        table.fill_(-9)
        sk.sk_pages_resize(account, [3], [60])
        sk.sk_pages_apply(account, arrays, table.data_ptr(), H.stream_handle())  # what has not changed since is not brought again
        torch.cuda.synchronize()
        assert table[3].tolist() == sk.sk_pages_state(account, 3)[1] and (table[:3] == -9).all() and (table[4] == -9).all()


@pytest.mark.parametrize("columns,seqs", [(12, 9), (120, 9), (300, 40)])
def test_rows_of_the_table_of_any_length(columns, seqs):
    """Rows that fit a launch's arguments, alone or beside the copies, and rows that go through host memory."""
    page, pages = 16, 2000
    pool = torch.randint(0, 1 << 30, (pages, 64), dtype=torch.int32, device="cuda")
    table = torch.full((seqs, columns), -7, dtype=torch.int32, device="cuda")
    arrays = arrays_of([pool] * 1)
    with sk.sk_pages_create(pages, page, seqs, columns) as account:
        for step in range(9):
            sk.sk_pages_resize(account, list(range(1, seqs)), [0] * (seqs - 1))
            sk.sk_pages_resize(account, [0], [min(columns * page - 20, 100 + 37 * step)])
            sk.sk_pages_fork(account, 0, list(range(1, seqs)))
            tokens = sk.sk_pages_state(account, 0)[0]
            sk.sk_pages_resize(account, list(range(1, seqs)), [tokens + 17] * (seqs - 1))
            before = pool.clone()
            copies = sk.sk_pages_state(account)[1]
            sk.sk_pages_apply(account, arrays, table.data_ptr(), H.stream_handle())
            torch.cuda.synchronize()
            rows = [sk.sk_pages_state(account, s)[1] for s in range(seqs)]
            assert table.cpu().tolist() == rows
            last = tokens // page
            assert copies == (seqs - 1 if tokens % page else 0)
            if tokens % page:
                for s in range(1, seqs):
                    assert torch.equal(pool[rows[s][last]], before[rows[0][last]])
