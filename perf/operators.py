"""The cases that the operators over paged key/value caches are measured on: what a decoder layer of several tenants' models
needs between its products.  Three operators:

  append  heads of queries and keys normalised, rotated to their positions, keys and values written into their pages
  attend  causal attention over the pages, with an optional sliding window and a few first tokens that stay visible
  pages   copies of pages: sequences that fork from a common prompt, pages moved to other places

A case says which ("op"), the tenants' models ("heads": query heads / key-value heads x size of a head, several joined by "+"
are dealt to the tenants in turn), how many sequences each tenant has in the batch, how many tokens are in a sequence's cache
before the call and how many are new (the bounds of a range, over its logarithm), and a number that fixes these lengths
("shapes"); the values come from the seed.  `run` returns all outputs: queries and whole pages, attention's outputs, pages and
page tables.
"""
from __future__ import annotations

import math
import random
from types import SimpleNamespace

import torch

own = False

TORCH = {"bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-6


# ---- cases -----------------------------------------------------------------------------------------------------------------

def listed():
    return [
        # one short step of one small model: what a call costs (12 heads of 64: the width of this repository's linear layers)
        dict(name="append_step_small", op="append", dtype="bf16", heads="12/12x64", tenants=1, seqs=3, old_min=20, old_max=700, new_min=1, new_max=1, page=16, rotary=64, pairs="halves", shapes=1),
        # one token for every sequence of four tenants
        dict(name="append_step_tenants", op="append", dtype="bf16", heads="32/8x128+12/12x64", tenants=4, seqs=64, old_min=1, old_max=4000, new_min=1, new_max=1, page=16, rotary=64, pairs="halves", shapes=2),
        # prompts of odd lengths; half of each head is rotated, neighbours as pairs
        dict(name="append_prompts", op="append", dtype="f16", heads="32/8x128", tenants=2, seqs=5, old_min=1, old_max=3, new_min=900, new_max=3500, page=64, rotary=64, pairs="neighbours", shapes=3),
        # one token for one sequence: latency
        dict(name="attend_step_one", op="attend", dtype="bf16", heads="12/12x64", tenants=1, seqs=1, old_min=700, old_max=900, new_min=1, new_max=1, page=16, window=0, sinks=0, shapes=4),
        # a serving batch of two tenants, caches from a single token to 8000
        dict(name="attend_step_ragged", op="attend", dtype="bf16", heads="32/8x128+12/12x64", tenants=2, seqs=48, old_min=1, old_max=8000, new_min=1, new_max=1, page=16, window=0, sinks=0, shapes=5),
        # long caches of which a step sees a window and the first four tokens
        dict(name="attend_step_window", op="attend", dtype="f16", heads="32/8x128", tenants=4, seqs=24, old_min=900, old_max=24000, new_min=1, new_max=1, page=32, window=1024, sinks=4, shapes=6),
        # few very long caches: the work of a sequence is split over the card
        dict(name="attend_step_long", op="attend", dtype="bf16", heads="32/8x128", tenants=1, seqs=6, old_min=50000, old_max=120000, new_min=1, new_max=1, page=64, window=0, sinks=0, shapes=7),
        # prompts with a window, head size 80 (no power of two)
        dict(name="attend_prompts_window", op="attend", dtype="f16", heads="16/4x80", tenants=2, seqs=3, old_min=1, old_max=2, new_min=1500, new_max=5000, page=32, window=700, sinks=5, shapes=8),
        # long prompts, every token sees all before it: bound by the matrix units
        dict(name="attend_prompts", op="attend", dtype="bf16", heads="32/8x128", tenants=1, seqs=2, old_min=1, old_max=2, new_min=7000, new_max=8100, page=64, window=0, sinks=0, shapes=9),
        # chunks of prompts (some of a single token) on top of caches of several thousand
        dict(name="attend_chunks", op="attend", dtype="bf16", heads="32/8x128", tenants=1, seqs=12, old_min=50, old_max=15000, new_min=1, new_max=300, page=16, window=0, sinks=0, shapes=10),
        # sixteen continuations of one prompt: they share its pages but for the last, which each gets a copy of
        dict(name="pages_fork", op="pages", way="fork", dtype="bf16", heads="32/8x128", layers=8, page=16, children=16, tokens=777, spare=40, shapes=11),
        # pages moved to other places of their arrays, as when a cache is compacted
        dict(name="pages_move", op="pages", way="move", dtype="bf16", heads="32/8x128", layers=16, page=16, moves=500, spare=60, shapes=12),
    ]


def _log(rng, lo, hi):
    """A whole number, spread over the logarithm of [lo, hi]."""
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


HEADS = ("12/12x64", "32/8x128", "16/4x80", "24/4x96", "16/16x64", "28/4x128", "8/1x256")


def draw(rng: random.Random):
    dtype, page, shapes = rng.choice(["bf16", "f16"]), rng.choice([16, 16, 32, 64, 128]), rng.randrange(100, 1 << 30)
    way = rng.choice(["append_step", "append_prompt", "attend_step", "attend_step", "attend_long", "attend_prompt", "attend_chunks", "fork", "move"])
    heads = rng.choice(HEADS)
    if way in ("fork", "move"):
        case = dict(op="pages", way=way, dtype=dtype, heads=rng.choice(["32/8x128", "12/12x64", "16/4x80"]), page=rng.choice([16, 32]))
        if way == "fork":
            return dict(case, layers=_log(rng, 1, 16), children=_log(rng, 1, 24), tokens=_log(rng, 1, 3000), spare=rng.randrange(0, 50), shapes=shapes)
        return dict(case, layers=_log(rng, 1, 12), moves=_log(rng, 1, 300), spare=rng.randrange(0, 50), shapes=shapes)
    case = dict(op=way.split("_")[0], dtype=dtype, heads=heads if rng.random() < 0.6 else heads + "+" + rng.choice(HEADS), page=page, shapes=shapes)
    if way.startswith("append"):
        dims = [int(h.split("x")[1]) for h in case["heads"].split("+")]
        case |= dict(rotary=rng.choice([min(dims), min(dims) // 2, 32]), pairs=rng.choice(["halves", "neighbours"]))
        if way == "append_step":
            return dict(case, tenants=rng.choice([1, 2, 4]), seqs=_log(rng, 1, 64), old_min=1, old_max=_log(rng, 2, 3000), new_min=1, new_max=rng.choice([1, 1, 4]))
        return dict(case, tenants=rng.choice([1, 2]), seqs=rng.randrange(1, 6), old_min=1, old_max=_log(rng, 2, 500), new_min=1, new_max=_log(rng, 10, 2500))
    window = rng.choice([0, 0, _log(rng, 16, 3000)])
    case |= dict(window=window, sinks=rng.choice([0, 1, 4, 37]) if window else 0)
    if way == "attend_step":
        return dict(case, tenants=rng.choice([1, 2, 3]), seqs=_log(rng, 1, 40), old_min=1, old_max=_log(rng, 2, 8000), new_min=1, new_max=rng.choice([1, 1, 1, 3]))
    if way == "attend_long":
        return dict(case, heads=heads, tenants=1, seqs=rng.randrange(1, 5), old_min=_log(rng, 1000, 30000), old_max=_log(rng, 30001, 90000), new_min=1, new_max=1)
    if way == "attend_prompt":
        return dict(case, heads=heads, tenants=1, seqs=rng.randrange(1, 4), old_min=1, old_max=2, new_min=_log(rng, 20, 1500), new_max=_log(rng, 1501, 5000))
    return dict(case, heads=heads, tenants=1, seqs=rng.randrange(2, 10), old_min=1, old_max=_log(rng, 100, 12000), new_min=1, new_max=_log(rng, 2, 300))


def models(case):
    """(query heads, key-value heads, size of a head) of each tenant."""
    kinds = [(int(h.split("/")[0]), int(h.split("/")[1].split("x")[0]), int(h.split("x")[1])) for h in case["heads"].split("+")]
    return [kinds[t % len(kinds)] for t in range(case.get("tenants", 1))]


def lengths(case):
    """[(tokens before the call, new tokens) of each sequence] of each tenant."""
    rng = random.Random(case["shapes"])
    return [[(_log(rng, case["old_min"], case["old_max"]), _log(rng, case["new_min"], case["new_max"])) for _ in range(case["seqs"])]
            for _ in range(case["tenants"])]


# ---- what has to be read, written and computed -----------------------------------------------------------------------------

def seen_by(case, old, new):
    """(pairs of a new token and a token that it sees, tokens that any of them sees) of one sequence."""
    window, sinks = case["window"], case["sinks"]
    if not window:
        return sum(old + t + 1 for t in range(new)), old + new
    pairs = sum(min(p + 1, window) + max(0, min(sinks, p + 1 - window)) for p in range(old, old + new))
    low = max(0, old - window + 1)
    return pairs, old + new - low + min(sinks, low)


def work(case):
    if case["op"] == "pages":
        (hq, hkv, d), = models(case)
        copies = case["moves"] if case["way"] == "move" else case["children"] * (case["tokens"] % case["page"] != 0)
        rows = 0 if case["way"] == "move" else case["children"] * 4 * (case["tokens"] // case["page"] + 1)
        return {"bytes": 2 * copies * case["layers"] * 2 * hkv * case["page"] * d * 2 + rows, "flops": 0}
    total = {"bytes": 0, "flops": 0}
    for (hq, hkv, d), seqs in zip(models(case), lengths(case)):
        for old, new in seqs:
            pages = -(-(old + new) // case["page"])
            if case["op"] == "append":
                total["bytes"] += new * (2 * (hq + 2 * hkv) * d * 2 + case["rotary"] * 4) + 4 * (-(-new // case["page"])) + 8
                total["flops"] += new * (hq + hkv) * (4 * d + 3 * case["rotary"])
            else:
                pairs, keys = seen_by(case, old, new)
                total["bytes"] += 2 * new * hq * d * 2 + 2 * keys * hkv * d * 2 + 4 * min(pages, keys // case["page"] + 2) + 8
                total["flops"] += 4 * pairs * hq * d
    return total


# ---- inputs ----------------------------------------------------------------------------------------------------------------

def _randn(gen, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32) * scale).to(dtype)


def _tenant(case, model, seqs, gen):
    """One tenant's cache, with its pages in no order, and the inputs of the call."""
    hq, hkv, d = model
    dt, page = TORCH[case["dtype"]], case["page"]
    need = [-(-(o + n) // page) for o, n in seqs]
    columns, count = max(need) + 1, sum(need) + 3
    order = torch.randperm(count, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((len(seqs), columns), -1, dtype=torch.int32, device="cuda")
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n]
        at += n
    rows = sum(n for _, n in seqs)
    firsts = [sum(n for _, n in seqs[:i]) for i in range(len(seqs) + 1)]
    t = SimpleNamespace(case=case, hq=hq, hkv=hkv, d=d, page=page, rows=rows, count=count, columns=columns, seqs=seqs, table=table,
                        longest=max(o + n for o, n in seqs), most_new=max(n for _, n in seqs), lengths=torch.tensor([o + n for o, n in seqs], dtype=torch.int32, device="cuda"),
                        firsts=torch.tensor(firsts, dtype=torch.int32, device="cuda"))
    if case["op"] == "append":
        t.k, t.v = (torch.zeros((count, hkv, page, d), dtype=dt, device="cuda") for _ in range(2))
        t.qkv = _randn(gen, (rows, (hq + 2 * hkv) * d), dt)  # what the layer's product of hidden states and weights gives
        t.q = torch.zeros((rows, hq, d), dtype=dt, device="cuda")
        t.q_weight, t.k_weight = (1.0 + _randn(gen, (d,), torch.float32, 0.1)).to(dt), (1.2 + _randn(gen, (d,), torch.float32, 0.2)).to(dt)
        half = case["rotary"] // 2
        positions = columns * page
        angle = torch.arange(positions, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
        t.cos, t.sin = angle.cos().float().contiguous(), angle.sin().float().contiguous()
    else:
        t.k, t.v = _randn(gen, (count, hkv, page, d), dt), _randn(gen, (count, hkv, page, d), dt)
        t.q = _randn(gen, (rows, hq, d), dt, 1.5)
        t.out = torch.zeros((rows, hq, d), dtype=dt, device="cuda")
    return t


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    if case["op"] == "pages":
        return _prepare_pages(case, gen)
    s = SimpleNamespace(case=case, tenants=[_tenant(case, m, q, gen) for m, q in zip(models(case), lengths(case))])
    if own:
        import paper_1901_10008_amd as sk

        s.sk, s.stream = sk, torch.cuda.current_stream().cuda_stream
        s.plan = sk.sk_attn_plan_create([_problem(sk, case, t) for t in s.tenants], keepalive=s.tenants)
    return s


def _problem(sk, case, t):
    p = dict(dtype=case["dtype"], q_heads=t.hq, kv_heads=t.hkv, head_dim=t.d, page_tokens=t.page, num_pages=t.count, sequences=len(t.seqs),
             pages_per_sequence=t.columns, rows=t.rows, max_new=t.most_new, k=t.k.data_ptr(), v=t.v.data_ptr(), page_table=t.table.data_ptr(),
             lengths=t.lengths.data_ptr(), first_row=t.firsts.data_ptr(), q=t.q.data_ptr())
    if case["op"] == "append":
        p |= dict(qkv=t.qkv.data_ptr(), q_weight=t.q_weight.data_ptr(), k_weight=t.k_weight.data_ptr(), eps=EPS, cos=t.cos.data_ptr(), sin=t.sin.data_ptr(),
                  positions=t.cos.shape[0], rotary_dim=case["rotary"], neighbours=case["pairs"] == "neighbours")
    else:
        p |= dict(out=t.out.data_ptr(), window=case["window"], sinks=case["sinks"])
    return sk.make_attn_problem(**p)


def _prepare_pages(case, gen):
    (hq, hkv, d), = models(case)
    page, layers = case["page"], case["layers"]
    s = SimpleNamespace(case=case)
    if case["way"] == "fork":
        held = -(-case["tokens"] // page)
        s.columns = held + 1
        s.count = held + 2 * case["children"] + case["spare"]
        s.table = torch.full((1 + case["children"], s.columns), -1, dtype=torch.int32, device="cuda")
        s.table[0, :held] = torch.arange(held, dtype=torch.int32, device="cuda")
    else:
        s.count = 2 * case["moves"] + case["spare"]
        order = torch.randperm(s.count, generator=gen, device="cuda")[:2 * case["moves"]].to(torch.int32)
        moves = order.cpu()  # the program decides on the host which page goes where
        s.src, s.dst = moves[:case["moves"]].contiguous(), moves[case["moves"]:].contiguous()
    s.pools = torch.empty((layers, 2, s.count, hkv, page, d), dtype=TORCH[case["dtype"]], device="cuda")
    for layer in range(layers):
        s.pools[layer] = _randn(gen, s.pools.shape[1:], s.pools.dtype)
    if own:
        import paper_1901_10008_amd as sk

        s.sk, s.stream = sk, torch.cuda.current_stream().cuda_stream
        size = s.pools[0, 0].numel() * 2
        s.arrays = sk.make_page_arrays([(s.pools.data_ptr() + i * size, size // s.count) for i in range(2 * layers)])
        if case["way"] == "fork":
            s.pages = sk.sk_pages_create(s.count, page, 1 + case["children"], s.columns)
            sk.sk_pages_resize(s.pages, sk.make_ids([0]), sk.make_ids([case["tokens"]]))
            s.children = sk.make_ids(range(1, 1 + case["children"]))
            s.none, s.more = sk.make_ids([0] * case["children"]), sk.make_ids([case["tokens"] + 1] * case["children"])
        else:
            s.from_, s.to = sk.make_ids(s.src.tolist()), sk.make_ids(s.dst.tolist())
    return s


# ---- one pass --------------------------------------------------------------------------------------------------------------

def run(state):
    case = state.case
    if case["op"] == "append":
        if own:
            state.sk.sk_attn_append(state.plan, state.stream)
        else:
            [append(case, t) for t in state.tenants]
        return [(t.q, t.k, t.v) for t in state.tenants]
    if case["op"] == "attend":
        if own:
            state.sk.sk_attn_launch(state.plan, state.stream)
            return [t.out for t in state.tenants]
        return [attend(case, t) for t in state.tenants]
    if case["way"] == "fork":
        own_fork(state) if own else fork(case, state)
        return state.pools, state.table
    if own:
        state.sk.sk_pages_copy(state.arrays, state.count, state.from_, state.to, state.stream)
    else:
        state.pools[:, :, state.dst.cuda().long()] = state.pools[:, :, state.src.cuda().long()]
    return state.pools


def own_fork(state):
    """Children of sequence 0 take the place of those of the call before, each with room for one more token."""
    sk, pages = state.sk, state.pages
    sk.sk_pages_resize(pages, state.children, state.none)
    sk.sk_pages_fork(pages, 0, state.children)
    sk.sk_pages_resize(pages, state.children, state.more)
    sk.sk_pages_apply(pages, state.arrays, state.table.data_ptr(), state.stream)


# ---- the plain forms -------------------------------------------------------------------------------------------------------

def rows_of(t):
    """Of each row: its sequence, which of the sequence's new tokens it is, and its position."""
    row = torch.arange(t.rows, device="cuda")
    seq = torch.searchsorted(t.firsts[1:].long(), row, right=True)
    new = t.firsts.long()[1:] - t.firsts.long()[:-1]
    nth = row - t.firsts.long()[seq]
    return seq, nth, t.lengths.long()[seq] - new[seq] + nth


def rotated(case, x, cos, sin):
    r = case["rotary"]
    if case["pairs"] == "halves":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., r:]], -1)
    a, b = x[..., 0:r:2], x[..., 1:r:2]
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), x[..., r:]], -1)


def append(case, t):
    seq, _, pos = rows_of(t)
    x = t.qkv.float().view(t.rows, t.hq + 2 * t.hkv, t.d)
    q, k, v = x[:, :t.hq], x[:, t.hq:t.hq + t.hkv], x[:, t.hq + t.hkv:]
    cos, sin = t.cos[pos][:, None], t.sin[pos][:, None]
    q = q * torch.rsqrt((q * q).mean(-1, keepdim=True) + EPS) * t.q_weight.float()
    k = k * torch.rsqrt((k * k).mean(-1, keepdim=True) + EPS) * t.k_weight.float()
    t.q.copy_(rotated(case, q, cos, sin))
    page = t.table[seq, pos // t.page].long()
    t.k[page, :, pos % t.page] = rotated(case, k, cos, sin).to(t.k.dtype)
    t.v[page, :, pos % t.page] = v.to(t.v.dtype)


def attend(case, t):
    seq, nth, _ = rows_of(t)
    n, m, groups = len(t.seqs), t.most_new, t.hq // t.hkv
    used = -(-t.longest // t.page)
    at = t.table[:, :used].long().clamp(min=0)
    k, v = (x[at].permute(0, 2, 1, 3, 4).reshape(n, t.hkv, used * t.page, t.d).float() for x in (t.k, t.v))
    first, new = t.firsts.long()[:-1, None], (t.firsts[1:] - t.firsts[:-1]).long()[:, None]
    nths = torch.arange(m, device="cuda")[None]
    q = t.q[(first + nths).clamp(max=t.rows - 1)].float().view(n, m, t.hkv, groups, t.d)
    q = q.permute(0, 2, 3, 1, 4).reshape(n, t.hkv, groups * m, t.d)
    pos = (t.lengths.long()[:, None] - new + nths)[:, :, None]
    key = torch.arange(used * t.page, device="cuda")[None, None]
    sees = (key <= pos) & (nths < new)[:, :, None]
    if case["window"]:
        sees &= (key > pos - case["window"]) | (key < case["sinks"])
    scores = torch.matmul(q, k.transpose(-1, -2)).mul_(t.d ** -0.5).view(n, t.hkv, groups, m, used * t.page)
    scores.masked_fill_(~sees[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True).clamp(min=-3e38)
    p = scores.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(n, t.hkv, groups * m, -1), v).view(n, t.hkv, groups, m, t.d)
    out = torch.where(total > 0, out / total, torch.zeros_like(out))
    return out[seq, :, :, nth].reshape(t.rows, t.hq, t.d).to(t.q.dtype)


def fork(case, s):
    """Children of sequence 0, in the lowest free pages; the first column behind whole pages gets a page of its own."""
    held, whole, n = -(-case["tokens"] // case["page"]), case["tokens"] // case["page"], case["children"]
    parent = s.table[0].clone()
    free = torch.ones(s.count, dtype=torch.bool, device="cuda")
    free[parent[:held].long()] = False
    fresh = torch.nonzero(free)[:n, 0]
    s.table[1:] = parent
    s.table[1:, whole] = fresh.to(torch.int32)
    if held > whole:
        s.pools[:, :, fresh] = s.pools[:, :, parent[whole:whole + 1].long()]


# ---- the definition in 64 bits ---------------------------------------------------------------------------------------------

def exact(case, seed):
    if case["op"] == "pages":
        return None  # copies of bits
    if case["op"] == "attend" and work(case)["flops"] > 8e12:
        return None
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    tenants = [_tenant(case, m, q, gen) for m, q in zip(models(case), lengths(case))]
    return [exact_append(case, t) if case["op"] == "append" else exact_attend(case, t) for t in tenants]


def exact_append(case, t):
    """Token by token of the sequences, heads as vectors; a pair (a, b) becomes the complex number a + bi times e^(i angle)."""
    q_all = torch.zeros(t.q.shape, dtype=torch.float64, device="cuda")
    k_all, v_all = t.k.double(), t.v.double()
    r, row = case["rotary"], 0
    ia = torch.arange(r // 2, device="cuda") if case["pairs"] == "halves" else torch.arange(0, r, 2, device="cuda")
    ib = ia + r // 2 if case["pairs"] == "halves" else ia + 1
    for s, (old, new) in enumerate(t.seqs):
        x = t.qkv[row:row + new].double().reshape(new, -1, t.d)
        turn = torch.complex(t.cos[old:old + new].double(), t.sin[old:old + new].double())[:, None]
        made = []
        for part, weight in ((x[:, :t.hq], t.q_weight), (x[:, t.hq:t.hq + t.hkv], t.k_weight)):
            y = part / torch.sqrt(part.square().sum(-1, keepdim=True) / t.d + EPS) * weight.double()
            z = torch.complex(y[..., ia].contiguous(), y[..., ib].contiguous()) * turn
            y[..., ia], y[..., ib] = z.real, z.imag
            made.append(y)
        q_all[row:row + new] = made[0]
        where = torch.arange(old, old + new, device="cuda")
        pages = t.table[s].long()[torch.div(where, t.page, rounding_mode="floor")]
        for page in pages.unique().tolist():
            here = pages == page
            slots = where[here] % t.page
            k_all[page][:, slots] = made[1][here].transpose(0, 1)
            v_all[page][:, slots] = x[here][:, t.hq + t.hkv:].transpose(0, 1)
        row += new
    return q_all, k_all, v_all


def exact_attend(case, t):
    """Sequence by sequence and head by head, some rows at a time: the softmax over the list of tokens that a row sees."""
    out, row, group = torch.zeros(t.q.shape, dtype=torch.float64, device="cuda"), 0, t.hq // t.hkv
    for s, (old, new) in enumerate(t.seqs):
        pages = t.table[s].long()[:-(-(old + new) // t.page)]
        for h in range(t.hkv):
            k, v = (x[pages, h].reshape(-1, t.d)[:old + new].double() for x in (t.k, t.v))
            for a in range(0, new, 1024):
                b = min(new, a + 1024)
                low = max(0, old + a - case["window"] + 1) if case["window"] else 0
                keys = torch.arange(low, old + b, device="cuda")
                if low:
                    keys = torch.cat([torch.arange(min(low, case["sinks"]), device="cuda"), keys])
                behind = torch.arange(old + a, old + b, device="cuda")[:, None] - keys[None]
                hidden = behind < 0
                if case["window"]:
                    hidden |= (behind >= case["window"]) & (keys >= case["sinks"])[None]
                for g in range(group):
                    w = t.q[row + a:row + b, h * group + g].double() @ k[keys].T / math.sqrt(t.d)
                    out[row + a:row + b, h * group + g] = torch.softmax(w.masked_fill(hidden, -math.inf), -1) @ v[keys]
        row += new
    return out
