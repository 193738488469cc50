"""Attention over paged caches against the formula in 64 bits (cache_harness.Tenant.attend, which also says how far a result may be)."""
import math

import pytest
import torch

import paper_1901_10008_amd as sk

import cache_harness as H
from cache_harness import Tenant

pytestmark = pytest.mark.gpu

# few rows and many, lengths around the steps of 16, 32, 64 and 128, an empty sequence, one without new rows, more rows than tokens
MIXED = ((1, 1), (0, 0), (17, 1), (31, 3), (64, 0), (129, 1), (65, 65), (200, 9), (3, 7), (128, 40), (0, 2), (16, 16))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [8, 64, 72, 80, 96, 104, 128, 136, 256])
def test_head_sizes(dtype, dim):
    H.check_attend([Tenant(dtype, (4, 2, dim), MIXED, seed=dim)], f"{dtype} {dim}")


@pytest.mark.parametrize("heads", [(1, 1, 64), (8, 8, 64), (8, 1, 128), (6, 2, 128), (12, 4, 80), (20, 1, 64), (64, 2, 64)])
@pytest.mark.parametrize("page", [16, 64])
def test_groups_and_pages(heads, page):
    H.check_attend([Tenant("bf16", heads, MIXED[:9], page=page, seed=3)], f"{heads} {page}")


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 0), (16, 4), (33, 40), (64, 1), (100, 500), (1000, 3), (0, 9), (2 ** 31 - 1, 2 ** 31 - 1)])
@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("f16", 64)])
def test_windows_and_sinks(window, sinks, dtype, dim):
    H.check_attend([Tenant(dtype, (4, 2, dim), MIXED + ((333, 1), (300, 150)), window=window, sinks=sinks, seed=window % 97)], f"{window} {sinks}")


@pytest.mark.parametrize("layout", ["page", "token", "heads"])
@pytest.mark.parametrize("dim", [64, 80])
def test_layouts_and_strides(layout, dim):
    H.check_attend([Tenant("f16", (4, 2, dim), MIXED, layout=layout, q_pad=8, out_pad=16, spare_rows=5, seed=7)], layout)


@pytest.mark.parametrize("workgroups", [1, 40, 600, 5000])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_slices_of_the_keys(workgroups, dim):
    seqs = ((1500, 1), (700, 2), (40, 1), (900, 50), (1, 1), (1200, 9))
    H.check_attend([Tenant("bf16", (4, 2, dim), seqs, seed=workgroups)], f"{workgroups}", workgroups=workgroups)
    H.check_attend([Tenant("f16", (4, 2, dim), seqs, window=300, sinks=5, seed=workgroups)], f"{workgroups} window", workgroups=workgroups)


@pytest.mark.parametrize("dtype,dim", [("bf16", 64), ("f16", 256)])
@pytest.mark.parametrize("count", [65, 90, 300])
def test_slices_of_many_sequences(count, dtype, dim):
    """More sequences than lanes, more than threads; every tenth is long, some with many rows: these are cut, at the least number of blocks a slice."""
    def seq(i):
        return ((1500, 1), (700, 40), (900, 2))[i // 10 % 3] if i % 10 == 3 else (1 + 7 * i % 60, i % 3)

    H.check_attend([Tenant(dtype, (2, 1, dim), [seq(i) for i in range(count)], seed=count)], f"{count}", workgroups=5000)


@pytest.mark.parametrize("dtype,tokens,new", [("bf16", 33000, 1), ("f16", 33000, 3), ("bf16", 66000, 40), ("bf16", 5000, 1), ("f16", 9000, 40)])
def test_as_many_slices_as_there_can_be(dtype, tokens, new):
    """256 slices of a unit of few rows (33000 tokens) and of many (66000), and 35 to 40 of them."""
    H.check_attend([Tenant(dtype, (2, 1, 64), ((tokens, new), (5, 1)), seed=tokens)], f"{tokens}", workgroups=5000)


def test_more_sequences_than_threads():
    seqs = tuple((1 + 37 * i % 90, 1 + (i % 7 == 0) * (i % 30) if (1 + 37 * i % 90) > 30 else 1) for i in range(600))
    H.check_attend([Tenant("bf16", (2, 1, 64), seqs, seed=1), Tenant("bf16", (2, 2, 40), seqs[:100], seed=2, window=20, sinks=2)], "many sequences")


def test_tenants_of_several_kinds_in_one_plan():
    ts = [Tenant("bf16", (4, 2, 64), MIXED, seed=1), Tenant("f16", (4, 4, 128), MIXED[:5], seed=2, window=20, sinks=3), Tenant("bf16", (2, 1, 256), MIXED[4:], seed=3),
          Tenant("bf16", (8, 2, 64), ((77, 1),) * 5, page=32, seed=4), Tenant("f16", (3, 3, 96), MIXED, page=128, seed=5, max_new=70)]
    H.check_attend(ts, "tenants")
    problems = [t.to_device() for t in ts]
    with sk.sk_attn_plan_create(problems) as plan:
        launches, workspace = sk.sk_attn_plan_info(plan)
        assert launches == 2 and workspace > 0


@pytest.mark.parametrize("scale", [0.02, 3.0, -1.0])
def test_scales(scale):
    # 3.0 on values of 2: softmaxes of a single token, scores of several hundred
    H.check_attend([Tenant("bf16", (4, 2, 64), MIXED, scale=scale, q_scale=2.0, seed=11)], f"{scale}")


@pytest.mark.parametrize("dtype,size", [("bf16", 2.0 ** 10), ("bf16", 2.0 ** 20), ("bf16", 2.0 ** 50), ("f16", 2.0 ** 9), ("f16", 2.0 ** 13)])
@pytest.mark.parametrize("dim", [64, 256])
@pytest.mark.parametrize("sign", [1, -1])
def test_large_scores(dtype, size, dim, sign):
    """Scores of up to 2^108 that lie far apart: a row's result is the value of its largest score, exactly up to the last rounding.  With sign -1 all
    scores are far below zero, the largest is the least of them."""
    seqs = ((1, 1), (700, 3), (90, 1), (400, 60), (130, 130), (33, 2))
    t = Tenant(dtype, (4, 2, dim), seqs, seed=dim)
    g = torch.Generator().manual_seed(dim)
    shape = torch.where(torch.rand((dim,), generator=g) < 0.5, -1.0, 1.0)
    t.q = (shape * size * (1 + torch.rand((t.rows, t.hq, dim), generator=g) / 2)).to(t.q.dtype)
    best = {}
    for s, (n, new) in enumerate(seqs):
        for j in range(n):
            # 1, 2, 4, 8 times the size in turn over runs of tokens, larger for few of them
            factor = 2.0 ** (j // 40 % 3) * (1 if j % 40 == 17 else 0.25)
            p, slot = int(t.table[s, j // t.page]), j % t.page
            t.k[p, :, slot] = (sign * shape * size * factor).to(t.k.dtype)
            best[s, j] = sign * factor
    with sk.sk_attn_plan_create([t.to_device()], sk.sk_attn_params_default(workgroups=200)) as plan:
        sk.sk_attn_launch(plan, H.stream_handle())
        torch.cuda.synchronize()
    got = t.out().double()
    for s, (n, new) in enumerate(seqs):
        for i in range(new):
            pos, row = n - new + i, int(t.firsts[s]) + i
            top = max(best[s, j] for j in range(pos + 1))
            winners = [j for j in range(pos + 1) if best[s, j] == top]
            for h in range(t.hq):
                v = torch.stack([t.v[int(t.table[s, j // t.page]), h // 2, j % t.page] for j in winners]).double()
                want = v.mean(0)
                tol = v.abs().mean(0) * (2 * H.U[dtype] + (len(winners) + 64) * 2.0 ** -23) + H.TINY[dtype]
                H.assert_close(got[row, h], want, tol, f"sequence {s} position {pos} head {h}")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("new", [1, 40])
def test_many_small_weights(dtype, new):
    """60000 tokens of weight 2^-25.6 beside four of weight 1, one for each wave: in f16 such weights are kept relative to a base that leaves them
    2^-32 of it as rounding, so that what they add up to is not lost."""
    t = Tenant(dtype, (2, 1, 64), ((60000, new),), page=64, seed=1)
    t.q[:], t.k[:], t.v[:] = 0, 0, 1
    t.q[:, :, 0] = 8
    for j in (0, 32, 64, 96):
        p, slot = int(t.table[0, j // 64]), j % 64
        t.k[p, 0, slot, 0], t.v[p, 0, slot] = 17.75, 0
    with sk.sk_attn_plan_create([t.to_device()], sk.sk_attn_params_default(workgroups=1)) as plan:
        sk.sk_attn_launch(plan, H.stream_handle())
        torch.cuda.synchronize()
    n = torch.arange(60000 - new + 1, 60001, dtype=torch.float64)[:, None, None] - 4
    small = n * math.exp(-17.75)
    want = (small / (4 + small)).expand(new, 2, 64)
    tol = want * (2 * H.U[dtype] + 2.0 ** -18) + H.TINY[dtype] + (n / 4 * 2.0 ** -32 if dtype == "f16" else 0)
    H.assert_close(t.out(), want, tol.expand(new, 2, 64), f"{new}")


@pytest.mark.parametrize("dtype,dim", [("bf16", 64), ("f16", 256)])
@pytest.mark.parametrize("window", [0, 30])
def test_scores_of_minus_infinity_are_hidden(dtype, dim, window):
    """Keys with which every query's product is -inf are as keys that are not there, down to rows that see no others."""
    seqs = ((60, 1), (60, 60), (300, 3), (200, 90))
    t = Tenant(dtype, (4, 2, dim), seqs, window=window, seed=dim)
    t.q[..., 3] = t.q[..., 3].abs() + 0.5
    gone = Tenant(dtype, (4, 2, dim), seqs, window=window, seed=dim)
    gone.q = t.q.clone()
    for s, pages in {0: (0, 1, 2, 3), 1: (0, 1, 3), 2: (2, 5, 17, 18), 3: (0, 7, 8, 9, 10, 11, 12)}.items():
        for c in pages:
            t.k[int(t.table[s, c]), :, :, 3] = -math.inf
            gone.table[s, c] = -1
    want, tol = gone.attend()
    with sk.sk_attn_plan_create([t.to_device()]) as plan:
        sk.sk_attn_launch(plan, H.stream_handle())
        torch.cuda.synchronize()
    assert (want[0] == 0).all() and (want[1:17] == 0).all()
    H.assert_close(t.out(), want, tol)


def test_rows_beyond_the_bound_are_left_alone():
    t = Tenant("bf16", (4, 2, 64), ((50, 9), (60, 3)), max_new=4, seed=1)
    problem = t.to_device()
    with sk.sk_attn_plan_create([problem]) as plan:
        sk.sk_attn_launch(plan, H.stream_handle())
        torch.cuda.synchronize()
    want, tol = t.attend()
    got = t.out()
    H.assert_close(got[:4], want[:4], tol[:4])
    H.assert_close(got[9:12], want[9:12], tol[9:12])
    assert torch.isnan(got[4:9]).all()


def test_what_lies_where_no_token_is_does_not_matter():
    for fill in (math.nan, math.inf, -math.inf):
        H.check_attend([Tenant("bf16", (4, 2, 64), MIXED, fill=fill, seed=5), Tenant("f16", (4, 2, 128), MIXED, window=24, sinks=3, fill=fill, seed=6)], f"{fill}")


def test_pages_that_are_none_of_the_cache():
    t = Tenant("bf16", (4, 2, 64), ((100, 1), (100, 60), (40, 1)), seed=9)
    t.table[0, 2], t.table[1, 0], t.table[2, :3] = -7, 2 ** 30, -1
    H.check_attend([t], "absent pages")


def test_lengths_beyond_the_table_are_cut():
    t = Tenant("bf16", (4, 2, 64), ((100, 1), (40, 2)), seed=9)
    want, tol = t.attend()
    problem = t.to_device()
    t.keep[1][1] = 2 ** 31 - 1  # the second sequence's: to the tokens of its row, none of which beyond the third page exist
    t.keep[2][0] = -5
    with sk.sk_attn_plan_create([problem]) as plan:
        sk.sk_attn_launch(plan, H.stream_handle())
        torch.cuda.synchronize()
        H.assert_close(t.out()[:1], want[:1], tol[:1])
        t.keep[1].copy_(t.lengths)
        t.keep[2].copy_(t.firsts)
        sk.sk_attn_launch(plan, H.stream_handle())
        torch.cuda.synchronize()
    H.assert_close(t.out()[:3], want[:3], tol[:3])


@pytest.mark.parametrize("count", [5, 90])
def test_rows_out_of_order_stay_inside(count):
    """first_row that decreases, or points outside: nothing is promised for such a step, but the next one is right."""
    seqs = ((300, 3), (500, 40), (64, 1), (700, 9), (90, 90)) * (count // 5)
    t = Tenant("bf16", (4, 2, 64), seqs, seed=12)
    want, tol = t.attend()
    problem = t.to_device()
    g = torch.Generator().manual_seed(count)
    with sk.sk_attn_plan_create([problem], sk.sk_attn_params_default(workgroups=60)) as plan:
        for low, high in ((0, t.rows + 1), (-2 ** 31, 2 ** 31 - 1)):
            t.keep[2].copy_(torch.randint(low, high, (count + 1,), generator=g, dtype=torch.int64).to(torch.int32))
            sk.sk_attn_launch(plan, H.stream_handle())
        t.keep[2].copy_(torch.tensor([0, t.rows] * count, dtype=torch.int32)[:count + 1])
        sk.sk_attn_launch(plan, H.stream_handle())
        t.keep[2].copy_(t.firsts)
        sk.sk_attn_launch(plan, H.stream_handle())
        torch.cuda.synchronize()
    H.assert_close(t.out(), want, tol)


def test_rows_out_of_order_leave_no_slices_behind():
    """Every second sequence with all rows: 175 units and slices for a launch of 166 workgroups, cut where one of two slices of a unit has none.  The next
    step uses that unit's count of arrivals."""
    t = Tenant("bf16", (4, 1, 64), ((1949, 1106),) + ((1949, 0),) * 6, seed=13)
    problem = t.to_device()
    with sk.sk_attn_plan_create([problem], sk.sk_attn_params_default(workgroups=111)) as plan:
        t.keep[1].copy_(torch.tensor([1245, 1949, 1909, 1289, 1257, 1350, 1949], dtype=torch.int32))
        t.keep[2].copy_(torch.tensor([0, 1106] * 4, dtype=torch.int32))
        sk.sk_attn_launch(plan, H.stream_handle())
        t.keep[1].copy_(t.lengths)
        t.keep[2].copy_(t.firsts)
        t.dout.fill_(math.nan)
        sk.sk_attn_launch(plan, H.stream_handle())
        torch.cuda.synchronize()
    want, tol = t.attend()
    H.assert_close(t.out(), want, tol)


def test_offsets_beyond_32_bits():
    """A cache of 2^32 elements and more for each of keys and values, tokens in its last pages."""
    dim, heads, page = 128, 8, 64
    count = 2 ** 32 // (page * heads * dim) + 3
    t = Tenant("bf16", (8, heads, dim), ((150, 1), (150, 20)), page=page, seed=4)
    problem = t.to_device()
    big = [torch.empty((count, heads, page, dim), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    shift = count - t.count
    for to, frm in zip(big, (t.dk, t.dv)):
        to[shift:] = frm
    t.keep[0][t.keep[0] >= 0] += shift
    problem.k, problem.v, problem.num_pages = big[0].data_ptr(), big[1].data_ptr(), count
    with sk.sk_attn_plan_create([problem]) as plan:
        sk.sk_attn_launch(plan, H.stream_handle())
        torch.cuda.synchronize()
    want, tol = t.attend()
    H.assert_close(t.out(), want, tol)


@pytest.mark.parametrize("dtype,dim", [("bf16", 64), ("f16", 256)])
def test_the_longest_sequences(dtype, dim):
    """All but 16 of 2^31 tokens, of which the rows see the first few and a window: tiles reach beyond 2^31, and no page number is read outside the
    table.  To the formula only distances count, so the first 16 tokens and the last 256 stand for the sequence."""
    columns, page, tail = 2 ** 27 - 1, 16, 16
    table = torch.full((columns,), -1, dtype=torch.int32, device="cuda")
    for new, window in ((1, 90), (3, 17), (40, 33), (40, 100), (90, 64)):
        t = Tenant(dtype, (4, 2, dim), (((1 + tail) * page, new),), page=page, window=window, sinks=3, seed=new + window)
        want, tol = t.attend()
        problem = t.to_device()
        table[0], table[columns - tail:] = int(t.table[0, 0]), t.table[0, 1:1 + tail].cuda()
        t.keep[1].fill_(columns * page)
        problem.page_table, problem.pages_per_sequence = table.data_ptr(), columns
        with sk.sk_attn_plan_create([problem]) as plan:
            sk.sk_attn_launch(plan, H.stream_handle())
            torch.cuda.synchronize()
        H.assert_close(t.out(), want, tol, f"{new} new, window {window}")


def test_a_plan_serves_steps_in_a_graph_and_on_another_stream():
    """One plan, lengths and rows that change: captured once, replayed with each step's numbers, eager work between."""
    steps = [((20, 1), (200, 1), (5, 1)), ((21, 1), (201, 1), (6, 1)), ((400, 3), (1, 0), (77, 40)), ((22, 1), (202, 1), (7, 1))]
    ts = [Tenant("bf16", (4, 2, 64), s, seed=i, spare_rows=60 - sum(n for _, n in s), spare_pages=60) for i, s in enumerate(steps)]
    base = ts[2]
    problem = base.to_device()
    side = torch.cuda.Stream()
    plan = sk.sk_attn_plan_create([problem])
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        sk.sk_attn_launch(plan, side.cuda_stream)
    side.synchronize()
    with torch.cuda.graph(graph, stream=side):
        sk.sk_attn_launch(plan, torch.cuda.current_stream().cuda_stream)
    for t in ts + ts[:2]:
        # the step's numbers, pages, queries into the plan's places
        table = torch.full_like(base.keep[0], -1)
        cols = min(t.columns, base.columns)
        table[:, :cols] = t.table[:, :cols].cuda()
        base.keep[0].copy_(table)
        base.keep[1].copy_(t.lengths)
        base.keep[2].copy_(t.firsts)
        n = min(t.count, base.count)
        base.dk[:n], base.dv[:n], base.dq[:] = t.k[:n].cuda(), t.v[:n].cuda(), t.q.cuda()
        base.dout.fill_(math.nan)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want, tol = t.attend()
        H.assert_close(base.out()[:t.rows_used], want[:t.rows_used], tol[:t.rows_used], f"{t.seqs}")
        replayed = base.out()
        base.dout.fill_(math.nan)
        torch.cuda.synchronize()
        sk.sk_attn_launch(plan, side.cuda_stream)
        side.synchronize()
        assert torch.equal(replayed[:t.rows_used].view(torch.int16), base.out()[:t.rows_used].view(torch.int16))
    del graph
    plan.close()


def test_empty_plan_and_plan_without_outputs():
    with sk.sk_attn_plan_create([]) as plan:
        sk.sk_attn_launch(plan, H.stream_handle())
        sk.sk_attn_append(plan, H.stream_handle())
    t = Tenant("bf16", (4, 2, 64), ((5, 1),), with_qkv=True, with_out=False)
    with sk.sk_attn_plan_create([t.to_device()]) as plan:
        with pytest.raises(sk.SkError) as e:
            sk.sk_attn_launch(plan, H.stream_handle())
        assert e.value.status == sk.SK_ERR_STATE
    t = Tenant("bf16", (4, 2, 64), ((5, 1),))
    with sk.sk_attn_plan_create([t.to_device()]) as plan:
        with pytest.raises(sk.SkError) as e:
            sk.sk_attn_append(plan, H.stream_handle())
        assert e.value.status == sk.SK_ERR_STATE
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype,dim", [("bf16", 64), ("bf16", 128), ("f16", 80), ("f16", 256)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 3)])
def test_what_a_row_does_not_see_does_not_reach_it(dtype, dim, window, sinks):
    """Infinities and NaN in keys and values of single tokens: rows that do not see them are as if they were not there; those that see one
    in the values are not finite in that element, those that see one in the keys nowhere."""
    seqs = ((200, 200), (90, 5), (150, 70), (300, 300))
    marks = {0: (("v", 100, math.inf), ("v", 101, math.nan), ("v", 1, -math.inf)), 1: (("v", 87, math.nan),), 2: (("k", 120, math.nan), ("v", 30, math.inf)),
             3: (("k", 299, math.inf), ("k", 64, math.nan))}
    t = Tenant(dtype, (4, 2, dim), seqs, window=window, sinks=sinks, seed=dim)
    clean = Tenant(dtype, (4, 2, dim), seqs, window=window, sinks=sinks, seed=dim)
    element = 5
    for s, ms in marks.items():
        for which, j, value in ms:
            p, slot = int(t.table[s, j // t.page]), j % t.page
            (t.v if which == "v" else t.k)[p, :, slot, element] = value
    want, tol = clean.attend()
    with sk.sk_attn_plan_create([t.to_device()]) as plan:
        sk.sk_attn_launch(plan, H.stream_handle())
        torch.cuda.synchronize()
    got = t.out().double()
    for s, (n, new) in enumerate(seqs):
        for i in range(new):
            pos, row = n - new + i, int(t.firsts[s]) + i
            seen = [m for m in marks[s] if m[1] <= pos and (not window or pos - m[1] < window or m[1] < sinks)]
            label = f"sequence {s} position {pos}"
            if any(m[0] == "k" for m in seen):
                assert not torch.isfinite(got[row]).any() or any(m[2] == math.inf for m in seen), label
                continue
            keep = torch.ones(dim, dtype=torch.bool)
            if seen:
                assert not torch.isfinite(got[row, :, element]).any(), label
                keep[element] = False
            H.assert_close(got[row][:, keep], want[row][:, keep], tol[row][:, keep], label)
