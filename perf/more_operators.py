"""The cases that the rest of a decoder step is measured on: what the models of several tenants need beside their products and
their attention.  Three operators:

  norm    a block's output, normalised, gated and scaled, added to the residual stream, which is normalised for the next block
  moe     a whole mixture-of-experts layer: the router, the choice of experts, their products and the weighted sum
  verify  drafted tokens accepted or rejected against the target's probabilities, and one more token sampled

A case says which ("op") and the sizes of the tenants' models (several joined by "+", one tenant each); what differs from
sequence to sequence comes from a number of the case ("shapes"), the values come from the seed.  Random numbers that a program
draws (of verify) are inputs.  `run` returns all outputs: residual stream and next block's input; sums, chosen experts and their weights; tokens
and numbers of accepted ones.
"""
from __future__ import annotations

import math
import random
from types import SimpleNamespace

import torch

own = False

TORCH = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
EPS = 1e-5


# ---- cases -----------------------------------------------------------------------------------------------------------------

def listed():
    return [
        # a step of three sequences of one small model (768: the width of this repository's linear layers): what a call costs
        dict(name="norm_step_small", op="norm", dtype="bf16", stream="bf16", dims="768", rows=3, spare=1, kind="rms", post=0, gate="none", act="none", biases=0),
        # a step of four tenants' models of different widths, norms on both sides of the block, a gate for every element
        dict(name="norm_step_tenants", op="norm", dtype="bf16", stream="f32", dims="4096+768+2048+5120", rows=64, spare=5, kind="rms", post=1, gate="rows", act="sigmoid", biases=0),
        # prompts: bound by memory
        dict(name="norm_prompts", op="norm", dtype="bf16", stream="f32", dims="4096", rows=16000, spare=0, kind="rms", post=1, gate="none", act="none", biases=0),
        # rows of odd length, mean and variance, biases, a gate that all rows share
        dict(name="norm_layer_odd", op="norm", dtype="f16", stream="f16", dims="1283", rows=5003, spare=10, kind="layer", post=1, gate="one", act="none", biases=1),
        # one token of one small model: latency
        dict(name="moe_step_one", op="moe", dtype="bf16", models="8/2x768x1024", rows=1, spare=0, act="silu", gated=1, scoring="softmax", normalize=1, bias=0, shared=0),
        # four rows each (a sequence with three drafted tokens, or four sequences) of two tenants, many small experts and a few larger ones
        dict(name="moe_step_tenants", op="moe", dtype="bf16", models="64/8x2048x1024+16/2x1024x2048", rows=4, spare=4, act="silu", gated=1, scoring="softmax", normalize=1, bias=0, shared=0),
        # two tokens, large experts
        dict(name="moe_step_large", op="moe", dtype="bf16", models="8/2x4096x12288", rows=2, spare=0, act="silu", gated=1, scoring="softmax", normalize=1, bias=0, shared=0),
        # a serving batch that reaches all experts and the one that every row passes
        dict(name="moe_batch_shared", op="moe", dtype="f16", models="60/4x2048x1408", rows=61, spare=3, act="silu", gated=1, scoring="sigmoid", normalize=1, bias=1, shared=2816),
        # a chunk of a prompt, sizes that are no multiples of a tile, experts of two products
        dict(name="moe_chunk_odd", op="moe", dtype="bf16", models="33/3x1000x1736", rows=250, spare=0, act="gelu", gated=0, scoring="softmax", normalize=0, bias=0, shared=0),
        # one sequence with four drafted tokens: latency
        dict(name="verify_step_one", op="verify", dtype="bf16", vocabs="32000", seqs=1, drafts_min=4, drafts_max=4, draft="logits", greedy=0, shapes=1),
        # a serving batch of two tenants, up to five drafted tokens, a vocabulary of odd length
        dict(name="verify_step_tenants", op="verify", dtype="bf16", vocabs="128000+50257", seqs=24, drafts_min=0, drafts_max=5, draft="logits", greedy=2, shapes=2),
        # drafts that another way than a model made (looked up in the prompt), logits in 32 bits
        dict(name="verify_looked_up", op="verify", dtype="f32", vocabs="150001", seqs=32, drafts_min=0, drafts_max=8, draft="certain", greedy=3, shapes=3),
    ]


def _log(rng, lo, hi):
    """A whole number, spread over the logarithm of [lo, hi]."""
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng: random.Random):
    way = rng.choice(["norm_step", "norm_prompt", "moe_step", "moe_step", "moe_batch", "verify", "verify", "sample"])
    if way.startswith("norm"):
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        layer = rng.random() < 0.3
        case = dict(op="norm", dtype=dtype, stream=rng.choice([dtype, "f32"]), kind="layer" if layer else "rms", post=rng.choice([0, 1]),
                    gate=rng.choice(["none", "one", "rows"]), act=rng.choice(["none", "sigmoid", "silu", "tanh"]), biases=int(layer and rng.random() < 0.7))
        if case["gate"] == "none":
            case["act"] = "none"
        sizes = lambda n: "+".join(str(_log(rng, 100, 8192) // step * step) for step in [rng.choice([8, 8, 1]) for _ in range(n)])  # noqa: E731
        if way == "norm_step":
            return dict(case, dims=sizes(rng.randrange(1, 5)), rows=_log(rng, 1, 256), spare=rng.randrange(0, 6))
        dim = sizes(1)
        return dict(case, dims=dim, rows=min(_log(rng, 256, 8000), 24_000_000 // int(dim)), spare=rng.randrange(0, 6))
    if way.startswith("moe"):
        gated = int(rng.random() < 0.8)

        def model():
            experts, dim, ffn = _log(rng, 4, 128), 8 * _log(rng, 32, 512), 8 * _log(rng, 16, 512)
            experts = max(2, min(experts, 480_000_000 // (3 * dim * ffn)))
            return f"{experts}/{rng.randrange(1, min(8, experts) + 1)}x{dim}x{ffn}"

        scoring = rng.choice(["softmax", "softmax", "sigmoid"])
        case = dict(op="moe", dtype=rng.choice(["bf16", "f16"]), act=rng.choice(["silu", "silu", "gelu", "relu"]), gated=gated, scoring=scoring,
                    normalize=rng.choice([0, 1]), bias=int(scoring == "sigmoid"), shared=rng.choice([0, 0, 8 * _log(rng, 16, 256)]))
        if way == "moe_step":
            models = model() if rng.random() < 0.6 else "+".join(_half(model()) for _ in range(2))
            return dict(case, models=models, rows=_log(rng, 1, 16), spare=rng.randrange(0, 5))
        return dict(case, models=model(), rows=_log(rng, 17, 250), spare=rng.randrange(0, 5))
    dtype, tenants = rng.choice(["bf16", "f16", "f32"]), rng.choice([1, 1, 2])
    case = dict(op="verify", dtype=dtype, vocabs="+".join(str(_log(rng, 300, 128000)) for _ in range(tenants)), seqs=_log(rng, 1, 32 // tenants), shapes=rng.randrange(100, 1 << 30))
    if way == "sample":
        return dict(case, drafts_min=0, drafts_max=0, draft="certain", greedy=rng.choice([0, 2, 4]))
    return dict(case, drafts_min=rng.choice([0, 1]), drafts_max=_log(rng, 1, 6), draft=rng.choice(["logits", "logits", "certain"]), greedy=rng.choice([0, 0, 3]))


def _half(model):
    """A model of half as many experts."""
    experts, rest = model.split("/")
    top, dims = rest.split("x", 1)
    experts = max(1, int(experts) // 2)
    return f"{experts}/{min(int(top), experts)}x{dims}"


def models(case):
    """(experts, chosen a row, width, width of an expert) of each tenant."""
    out = []
    for m in case["models"].split("+"):
        e, rest = m.split("/")
        k, d, f = rest.split("x")
        out.append((int(e), int(k), int(d), int(f)))
    return out


def drafts(case):
    """Drafted tokens of each sequence, and which are greedy, of each tenant."""
    rng = random.Random(case["shapes"])
    out = []
    for _ in case["vocabs"].split("+"):
        counts = [rng.randrange(case["drafts_min"], case["drafts_max"] + 1) for _ in range(case["seqs"])]
        out.append((counts, [bool(case["greedy"]) and rng.randrange(case["greedy"]) == 0 for _ in counts]))
    return out


# ---- what has to be read, written and computed -----------------------------------------------------------------------------

def work(case):
    total = {"bytes": 0, "flops": 0}
    if case["op"] == "norm":
        one, res = SIZE[case["dtype"]], SIZE[case["stream"]]
        for d in map(int, case["dims"].split("+")):
            vectors = (1 + case["post"]) * (1 + case["biases"]) + (case["gate"] == "one")
            total["bytes"] += case["rows"] * d * ((2 + (case["gate"] == "rows")) * one + 2 * res) + vectors * d * one
            total["flops"] += case["rows"] * d * (7 + 4 * case["post"] + 4 * (case["gate"] != "none"))
    elif case["op"] == "moe":
        products = 2 + case["gated"]
        for e, k, d, f in models(case):
            t = case["rows"]
            reached = e * (1.0 - (1.0 - k / e) ** t)  # experts that some row chooses, on average
            total["bytes"] += int(2 * products * d * (reached * f + case["shared"])) + 2 * e * d + 4 * t * d + 8 * t * k
            total["flops"] += 2 * t * d * (e + products * (k * f + case["shared"]))
    else:
        one = SIZE[case["dtype"]]
        for v, (counts, _) in zip(map(int, case["vocabs"].split("+")), drafts(case)):
            rows = sum(counts) + len(counts) + (sum(counts) if case["draft"] == "logits" else 0)
            total["bytes"] += rows * v * one + 16 * len(counts) + 12 * sum(counts)
            total["flops"] += rows * v * 3
    return total


# ---- inputs ----------------------------------------------------------------------------------------------------------------

def _randn(gen, shape, dtype, scale=1.0, shift=0.0):
    return (torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32) * scale + shift).to(TORCH[dtype])


def _count(n):
    return torch.tensor([n], dtype=torch.int32, device="cuda")


def _norm_tenants(case, gen):
    out = []
    for d in map(int, case["dims"].split("+")):
        dt, n = case["dtype"], case["rows"] + case["spare"]
        t = SimpleNamespace(d=d, rows=n, used=case["rows"], n_rows=_count(case["rows"]), block=_randn(gen, (n, d), dt, 0.7), residual=_randn(gen, (n, d), case["stream"], 3.0),
                            gate=None, post_w=None, post_b=None, pre_w=_randn(gen, (d,), dt, 0.2, 1.0), pre_b=None)
        if case["gate"] != "none":
            t.gate = _randn(gen, (n, d) if case["gate"] == "rows" else (d,), dt)
        if case["post"]:
            t.post_w = _randn(gen, (d,), dt, 0.3, 0.8)
        if case["biases"]:
            t.pre_b = _randn(gen, (d,), dt, 0.1)
            t.post_b = _randn(gen, (d,), dt, 0.1) if case["post"] else None
        t.scale, t.block_scale = 0.98, 1.25
        t.residual_out, t.next = torch.zeros_like(t.residual), torch.zeros_like(t.block)
        out.append(t)
    return out


def _moe_tenants(case, gen):
    out = []
    for e, k, d, f in models(case):
        dt, n, s = case["dtype"], case["rows"] + case["spare"], case["shared"]
        t = SimpleNamespace(e=e, k=k, d=d, f=f, rows=n, used=case["rows"], n_rows=_count(case["rows"]), x=_randn(gen, (n, d), dt), router=_randn(gen, (e, d), dt, d ** -0.5),
                            bias=torch.randn((e,), generator=gen, device="cuda") * 0.05 if case["bias"] else None, scale=1.5 if case["scoring"] == "sigmoid" else 1.0,
                            gate=None, up=_randn(gen, (e, f, d), dt, d ** -0.5), down=_randn(gen, (e, d, f), dt, f ** -0.5), s_gate=None, s_up=None, s_down=None)
        if case["gated"]:
            t.gate = _randn(gen, (e, f, d), dt, 1.5 * d ** -0.5)
        if s:
            t.s_up, t.s_down = _randn(gen, (s, d), dt, d ** -0.5), _randn(gen, (d, s), dt, s ** -0.5)
            t.s_gate = _randn(gen, (s, d), dt, 1.5 * d ** -0.5) if case["gated"] else None
        t.out = torch.zeros((n, d), dtype=TORCH[dt], device="cuda")
        t.ids = torch.zeros((n, k), dtype=torch.int32, device="cuda")
        t.weights = torch.zeros((n, k), dtype=torch.float32, device="cuda")
        out.append(t)
    return out


def _verify_tenants(case, gen):
    out = []
    for v, (counts, greedy) in zip(map(int, case["vocabs"].split("+")), drafts(case)):
        rows = sum(counts) + len(counts)
        firsts = [sum(counts[:i]) + i for i in range(len(counts) + 1)]
        likely = torch.zeros((rows, v), device="cuda")
        some = torch.randint(0, v, (rows, 6), generator=gen, device="cuda")  # a few words that fit, by up to e^10
        likely.scatter_reduce_(1, some, torch.rand((rows, 6), generator=gen, device="cuda") * 10.0, "amax")
        base = torch.randn((rows, v), generator=gen, device="cuda") * 2.0 + likely
        t = SimpleNamespace(v=v, rows=rows, counts=counts, seqs=len(counts), firsts=torch.tensor(firsts, dtype=torch.int32, device="cuda"),
                            logits=base.to(TORCH[case["dtype"]]), draft_logits=None, temperature=torch.rand((len(counts),), generator=gen, device="cuda") * 0.7 + 0.6)
        t.temperature[torch.tensor(greedy, device="cuda")] = 0.0
        guess = base * 0.9 + torch.randn((rows, v), generator=gen, device="cuda") * 0.7
        if case["draft"] == "logits":
            t.draft_logits = guess.to(TORCH[case["dtype"]])
            guess = t.draft_logits.float()
        # the draft model's tokens, drawn from its distribution
        noise = -torch.log(torch.empty((rows, v), device="cuda").exponential_(generator=gen))
        t.drafted = (guess + noise).argmax(-1).to(torch.int32)
        t.accept_random = torch.rand((rows,), generator=gen, device="cuda")
        t.sample_random = torch.rand((len(counts),), generator=gen, device="cuda")
        t.tokens = torch.zeros((rows,), dtype=torch.int32, device="cuda")
        t.accepted = torch.zeros((len(counts),), dtype=torch.int32, device="cuda")
        out.append(t)
    return out


def _tenants(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return {"norm": _norm_tenants, "moe": _moe_tenants, "verify": _verify_tenants}[case["op"]](case, gen)


def prepare(case, seed):
    s = SimpleNamespace(case=case, tenants=_tenants(case, seed))
    if own:
        import paper_1901_10008_amd as sk

        s.sk, s.stream = sk, torch.cuda.current_stream().cuda_stream
        make = {"norm": _norm_problem, "moe": _moe_problem, "verify": _verify_problem}[case["op"]]
        create = {"norm": sk.sk_norm_plan_create, "moe": sk.sk_moe_plan_create, "verify": sk.sk_verify_plan_create}[case["op"]]
        s.plan = create([make(sk, case, t) for t in s.tenants], keepalive=s.tenants)
    return s


def _at(x):
    return 0 if x is None else x.data_ptr()


def _norm_problem(sk, case, t):
    return sk.make_norm_problem(
        dtype=case["dtype"], residual_dtype=case["stream"], kind={"rms": sk.SK_NORM_RMS, "layer": sk.SK_NORM_LAYER}[case["kind"]], rows=t.rows, dim=t.d, post=case["post"],
        gate_act={"none": sk.SK_ACT_NONE, "sigmoid": sk.SK_ACT_SIGMOID, "silu": sk.SK_ACT_SILU, "tanh": sk.SK_ACT_TANH}[case["act"]], gate_rows=int(case["gate"] == "rows"),
        eps=EPS, residual_scale=t.scale, block_scale=t.block_scale, n_rows=_at(t.n_rows), block=_at(t.block), gate=_at(t.gate), residual=_at(t.residual),
        post_weight=_at(t.post_w), post_bias=_at(t.post_b), pre_weight=_at(t.pre_w), pre_bias=_at(t.pre_b), residual_out=_at(t.residual_out), next=_at(t.next))


def _moe_problem(sk, case, t):
    return sk.make_moe_problem(
        dtype=case["dtype"], router_dtype=case["dtype"], rows=t.rows, dim=t.d, experts=t.e, top_k=t.k, ffn=t.f, shared_ffn=case["shared"],
        act={"silu": sk.SK_ACT_SILU, "gelu": sk.SK_ACT_GELU, "relu": sk.SK_ACT_RELU}[case["act"]], scoring={"softmax": sk.SK_MOE_SOFTMAX, "sigmoid": sk.SK_MOE_SIGMOID}[case["scoring"]],
        normalize=case["normalize"], scale=t.scale, n_rows=_at(t.n_rows), x=_at(t.x), router=_at(t.router), router_bias=_at(t.bias), gate=_at(t.gate), up=_at(t.up),
        down=_at(t.down), shared_gate=_at(t.s_gate), shared_up=_at(t.s_up), shared_down=_at(t.s_down), out=_at(t.out), expert_ids=_at(t.ids), expert_weights=_at(t.weights))


def _verify_problem(sk, case, t):
    return sk.make_verify_problem(
        dtype=case["dtype"], sequences=t.seqs, rows=t.rows, vocab=t.v, first_row=_at(t.firsts), logits=_at(t.logits), drafted=_at(t.drafted), draft_logits=_at(t.draft_logits),
        temperatures=_at(t.temperature), accept_random=_at(t.accept_random), sample_random=_at(t.sample_random), tokens=_at(t.tokens), accepted=_at(t.accepted))


# ---- one pass --------------------------------------------------------------------------------------------------------------

def run(state):
    case = state.case
    if case["op"] == "norm":
        if own:
            state.sk.sk_norm_launch(state.plan, state.stream)
        else:
            [norm(case, t) for t in state.tenants]
        return [(t.residual_out, t.next) for t in state.tenants]
    if case["op"] == "moe":
        if own:
            state.sk.sk_moe_launch(state.plan, state.stream)
        else:
            [moe(case, t) for t in state.tenants]
        return [(t.out, t.ids, t.weights) for t in state.tenants]
    if own:
        state.sk.sk_verify_launch(state.plan, state.stream)
    else:
        [verify(t) for t in state.tenants]
    return [(t.tokens, t.accepted) for t in state.tenants]


# ---- the plain forms -------------------------------------------------------------------------------------------------------

def activated(name, x):
    if name == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-x))
    if name == "silu":
        return x / (1.0 + torch.exp(-x))
    if name == "tanh":
        return torch.tanh(x)
    if name == "gelu":
        return 0.5 * x * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (x + 0.044715 * x * x * x)))
    if name == "relu":
        return x.clamp(min=0.0)
    return x


def normalised(case, x, weight, bias):
    if case["kind"] == "layer":
        x = x - x.mean(-1, keepdim=True)
    y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()
    return y if bias is None else y + bias.float()


def norm(case, t):
    n = t.used
    u = t.block[:n].float()
    if case["post"]:
        u = normalised(case, u, t.post_w, t.post_b)
    if t.gate is not None:
        u = u * activated(case["act"], (t.gate[:n] if case["gate"] == "rows" else t.gate).float())
    r = t.scale * t.residual[:n].float() + t.block_scale * u
    t.residual_out[:n] = r.to(t.residual.dtype)
    t.next[:n] = normalised(case, r, t.pre_w, t.pre_b).to(t.next.dtype)


def chosen(case, t):
    """(experts in the order of their scores, weights) of each row: in 64 bits, since scores next to each other decide."""
    logits = t.x[:t.used].double() @ t.router.double().T
    scores = torch.softmax(logits, -1) if case["scoring"] == "softmax" else torch.sigmoid(logits)
    rank = scores if t.bias is None else scores + t.bias.double()
    rank = logits if case["scoring"] == "softmax" and t.bias is None else rank
    ids = torch.sort(rank, dim=-1, descending=True, stable=True).indices[:, :t.k]
    w = scores.gather(1, ids)
    if case["normalize"]:
        w = w / w.sum(-1, keepdim=True)
    return ids, (w * t.scale).float()


def expert(case, x, gate, up, down):
    h = x @ up.float().T
    h = activated(case["act"], x @ gate.float().T) * h if gate is not None else activated(case["act"], h)
    return h @ down.float().T


def moe(case, t):
    n = t.used
    x = t.x[:n].float()
    ids, weights = chosen(case, t)
    out = torch.zeros((n, t.d), device="cuda")
    if t.s_up is not None:
        out += expert(case, x, t.s_gate, t.s_up, t.s_down)
    for e in ids.unique().tolist():
        row, nth = torch.where(ids == e)
        out[row] += weights[row, nth, None] * expert(case, x[row], t.gate[e] if t.gate is not None else None, t.up[e], t.down[e])
    t.out[:n], t.ids[:n], t.weights[:n] = out.to(t.out.dtype), ids.to(torch.int32), weights


def distribution(logits, temperature):
    """Probabilities of each row in 64 bits; at temperature 0 the first of the largest."""
    x = logits.double()
    top = x.amax(-1, keepdim=True)
    w = torch.exp((x - top) / torch.where(temperature > 0, temperature, 1.0)[:, None])
    w /= w.sum(-1, keepdim=True)
    v = torch.arange(x.shape[1], device="cuda")
    first = torch.where(x == top, v, x.shape[1]).amin(-1, keepdim=True)
    return torch.where((temperature > 0)[:, None], w, (v == first).double())


def verify(t):
    row = torch.arange(t.rows, device="cuda")
    seq = torch.searchsorted(t.firsts[1:].long(), row, right=True)
    first, last = t.firsts.long()[:-1], t.firsts.long()[1:] - 1
    temperature = t.temperature.double()[seq]
    p = distribution(t.logits, temperature)
    token = t.drafted.long()
    certain = torch.zeros_like(p).scatter_(1, token[:, None], 1.0)
    q = certain if t.draft_logits is None else torch.where((temperature > 0)[:, None], distribution(t.draft_logits, temperature.clamp(min=1e-3)), certain)
    # the first row of each sequence whose drafted token is rejected, or its last, which has none
    fails = ~(t.accept_random.double() * q.gather(1, token[:, None])[:, 0] < p.gather(1, token[:, None])[:, 0]) | (row == last[seq])
    stop = torch.full((t.seqs,), t.rows, device="cuda").scatter_reduce_(0, seq, torch.where(fails, row, t.rows), "amin")
    drafted = (stop < last)[:, None]
    w = torch.where(drafted, (p[stop] - q[stop]).clamp(min=0.0), p[stop])
    w = torch.where(w.sum(-1, keepdim=True) > 0, w, p[stop])
    below = w.cumsum(-1)
    past = below > t.sample_random.double()[:, None] * below[:, -1:]
    v = torch.arange(t.v, device="cuda")
    sampled = torch.where(past & (w > 0), v, t.v).amin(-1)
    sampled = torch.where(sampled < t.v, sampled, torch.where(w > 0, v, -1).amax(-1))
    out = torch.where(row < stop[seq], token, torch.where(row == stop[seq], sampled[seq], -1))
    t.tokens.copy_(out)
    t.accepted.copy_(stop - first)


# ---- the definition in 64 bits ---------------------------------------------------------------------------------------------

def exact(case, seed):
    tenants = _tenants(case, seed)
    return [{"norm": exact_norm, "moe": exact_moe, "verify": exact_verify}[case["op"]](case, t) for t in tenants]


def exact_norm(case, t):
    def standard(x, weight, bias):
        mean = x.sum(1) / t.d if case["kind"] == "layer" else torch.zeros_like(x[:, 0])
        spread = ((x - mean[:, None]) ** 2).sum(1) / t.d
        y = (x - mean[:, None]) * weight.double() / torch.sqrt(spread + EPS)[:, None]
        return y if bias is None else y + bias.double()

    res, out = t.residual_out.double(), t.next.double()
    for a in range(0, t.used, 2000):
        b = min(t.used, a + 2000)
        u = t.block[a:b].double()
        if case["post"]:
            u = standard(u, t.post_w, t.post_b)
        if t.gate is not None:
            g = (t.gate[a:b] if case["gate"] == "rows" else t.gate.expand(b - a, -1)).double()
            u = u * {"none": lambda z: z, "sigmoid": torch.sigmoid, "silu": lambda z: z * torch.sigmoid(z), "tanh": torch.tanh}[case["act"]](g)
        # scales are numbers of 32 bits
        res[a:b] = float(torch.tensor(t.scale)) * t.residual[a:b].double() + float(torch.tensor(t.block_scale)) * u
        out[a:b] = standard(res[a:b], t.pre_w, t.pre_b)
    return res, out


def exact_moe(case, t):
    """Row by row: scores of all experts one by one in order, the best taken out k times, their products as sums over rows of weights."""
    act = {"silu": lambda z: z * torch.sigmoid(z), "relu": torch.relu, "gelu": lambda z: 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))}[case["act"]]
    out, ids, weights = t.out.double(), t.ids.clone(), t.weights.double()
    router, held = t.router.double(), {}

    def through(x, e):
        if e not in held:
            if len(held) == 8:
                held.clear()
            g, u, w = (t.s_gate, t.s_up, t.s_down) if e < 0 else (None if t.gate is None else t.gate[e], t.up[e], t.down[e])
            held[e] = tuple(None if m is None else m.double() for m in (g, u, w))
        g, u, w = held[e]
        h = torch.mv(u, x)
        return torch.mv(w, act(torch.mv(g, x)) * h if g is not None else act(h))

    picks = []
    for r in range(t.used):
        logit = (router * t.x[r].double()).sum(1)
        score = (logit - logit.logsumexp(0)).exp() if case["scoring"] == "softmax" else 1.0 / (1.0 + (-logit).exp())
        rank = (logit if case["scoring"] == "softmax" and t.bias is None else score + (0.0 if t.bias is None else t.bias.double())).tolist()
        pick = sorted(range(t.e), key=lambda e: (-rank[e], e))[:t.k]
        w = score[pick]
        if case["normalize"]:
            w = w / w.sum()
        weights[r] = w * t.scale
        ids[r] = torch.tensor(pick, dtype=torch.int32)
        picks.append(pick)
        out[r] = through(t.x[r].double(), -1) if t.s_up is not None else 0.0
    for e in range(t.e):  # (expert by expert, so that its weights are made 64 bits wide once)
        for r, pick in enumerate(picks):
            if e in pick:
                out[r] += weights[r, pick.index(e)] * through(t.x[r].double(), e)
    return out, ids, weights


def exact_verify(case, t):
    """Sequence by sequence, token by token."""
    tokens, accepted = torch.full_like(t.tokens, -1), torch.zeros_like(t.accepted)

    def probabilities(x, temperature):
        if temperature == 0.0:
            p = torch.zeros(t.v, dtype=torch.float64, device="cuda")
            p[int((x == x.max()).nonzero()[0])] = 1.0
            return p
        return torch.softmax(x.double() / temperature, 0)

    row = 0
    for s, count in enumerate(t.counts):
        temperature, n = float(t.temperature[s]), 0
        while True:
            w = probabilities(t.logits[row + n], temperature)
            if n == count:
                break
            d = int(t.drafted[row + n])
            if t.draft_logits is None or temperature == 0.0:
                q = torch.zeros_like(w)
                q[d] = 1.0
            else:
                q = probabilities(t.draft_logits[row + n], temperature)
            if not float(t.accept_random[row + n]) * float(q[d]) < float(w[d]):
                rest = torch.relu(w - q)
                w = rest if float(rest.sum()) > 0 else w
                break
            tokens[row + n] = d
            n += 1
        bound = float(t.sample_random[s]) * float(w.sum())
        at = int(torch.searchsorted(w.cumsum(0), torch.tensor([bound], dtype=torch.float64, device="cuda"), right=True))
        tokens[row + n] = at if at < t.v else int(w.nonzero()[-1])
        accepted[s] = n
        row += count + 1
    return tokens, accepted
