"""Inputs on the device, plain results in 64 bits, and how far the kernels may be from them, for the operators of a decoder step beside products
and attention.  References are computed on the device, with elementary operations in 64 bits."""
import math

import torch

import paper_1901_10008_amd as sk

TORCH = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
# Unit roundoff of the types, and half of the spacing of their smallest numbers.
U = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}
TINY = {"bf16": 2.0 ** -134, "f16": 2.0 ** -25, "f32": 2.0 ** -126}  # (fp32 arithmetic may take numbers below 2^-126 as 0)
E = 2.0 ** -24  # a rounding to fp32
ACT = {"none": 0, "sigmoid": 1, "silu": 2, "tanh": 3, "gelu": 4, "relu": 5}


def stream_handle():
    return torch.cuda.current_stream().cuda_stream


def generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(g, *shape, scale=1.0, shift=0.0):
    return torch.randn(shape, generator=g, device="cuda") * scale + shift


def at(x):
    return 0 if x is None else x.data_ptr()


def int32(*values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def activated(name, z):
    """(act(z), how far the kernel's may be from it).  exp in fp32 is off by a few units of the last place and its argument by a rounding for every operation
    on the way (|t| of them count); tanh as 2s - 1 is off by 8 roundings of 1, which from 1/4 on is less than 40 of its own."""
    t = z
    if name == "sigmoid":
        y = torch.sigmoid(z)
    elif name == "silu":
        y = z * torch.sigmoid(z)
    elif name == "tanh":
        y, t = torch.tanh(z), 2 * z
    elif name == "gelu":
        w = math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)
        y, t = z * torch.sigmoid(2 * w), 2 * w
    elif name == "relu":
        return z.clamp(min=0), torch.zeros_like(z)
    else:
        return z, torch.zeros_like(z)
    return y, (4 * E * (10 + t.abs()) * y.abs()).clamp(min=0) + 2.0 ** -126


def check(got, want, tol, label=""):
    got = got.double()
    bad = ~((got - want).abs() <= tol)
    if bad.any():
        i = tuple(int(x) for x in bad.nonzero()[0])
        raise AssertionError(f"{label}: {int(bad.sum())} of {bad.numel()} off, first at {i}: {float(got[i])!r} for {float(want[i])!r}, allowed {float(tol[i]):.3g}")


def padded(rows, dim, pad, dtype, fill=float("nan")):
    """A buffer of rows `dim` wide with `pad` elements behind each, and its view of the rows."""
    buffer = torch.full((rows, dim + pad), fill, dtype=dtype, device="cuda")
    return buffer, buffer[:, :dim]


# ---- norms -----------------------------------------------------------------------------------------------------------------

class Norm:
    def __init__(self, dtype="bf16", stream=None, rows=3, dim=96, kind="rms", post=0, gate=None, act="none", biases=False, weights=True, block=True, residual=True,
                 residual_out=True, next=True, eps=1e-5, rs=0.9, bs=1.3, pad=0, used=None, seed=0, in_place=False):
        g = generator(seed)
        self.dtype, self.stream, self.rows, self.dim, self.kind, self.post, self.act, self.eps = dtype, stream or dtype, rows, dim, kind, post, act, eps
        dt, rt = TORCH[dtype], TORCH[self.stream]
        make = lambda t, shift=0.0: padded(rows, dim, pad, t)  # noqa: E731
        self.rs, self.bs, self.pad = rs, bs, pad
        self.block = self.residual = self.gate = None
        if block:
            self.block_b, self.block = make(dt)
            self.block.copy_(randn(g, rows, dim, shift=0.3))
        if residual:
            self.residual_b, self.residual = make(rt)
            self.residual.copy_(randn(g, rows, dim, scale=2.0, shift=-0.5))
        if gate == "rows":
            self.gate_b, self.gate = make(dt)
            self.gate.copy_(randn(g, rows, dim, scale=1.5))
        elif gate == "one":
            self.gate = randn(g, dim).to(dt)
        self.gate_rows = int(gate == "rows")
        vector = lambda shift, scale: randn(g, dim, scale=scale, shift=shift).to(dt)  # noqa: E731
        self.post_w, self.pre_w = (vector(0.9, 0.3), vector(1.1, 0.2)) if weights else (None, None)
        self.post_b, self.pre_b = (vector(0.0, 0.3), vector(0.1, 0.3)) if biases else (None, None)
        if in_place:
            self.residual_out_b, self.residual_out, self.next_b, self.next = self.residual_b, self.residual, self.block_b, self.block
        else:
            self.residual_out_b, self.residual_out = make(rt) if residual_out else (None, None)
            self.next_b, self.next = make(dt) if next else (None, None)
        self.n_rows = None if used is None else int32(used)
        self.used = rows if used is None else max(0, min(used, rows))

    def problem(self):
        s = self.dim + self.pad if self.pad else 0
        return sk.make_norm_problem(
            dtype=self.dtype, residual_dtype=self.stream, kind={"rms": 0, "layer": 1}[self.kind], rows=self.rows, dim=self.dim, post=self.post, gate_act=ACT[self.act],
            gate_rows=self.gate_rows, eps=self.eps, residual_scale=self.rs, block_scale=self.bs, block_stride=s, gate_stride=s if self.gate_rows else 0, residual_stride=s,
            residual_out_stride=s, next_stride=s, n_rows=at(self.n_rows), block=at(self.block), gate=at(self.gate), residual=at(self.residual), post_weight=at(self.post_w),
            post_bias=at(self.post_b), pre_weight=at(self.pre_w), pre_bias=at(self.pre_b), residual_out=at(self.residual_out), next=at(self.next))

    def standard(self, x, e, weight, bias):
        """N(x) * weight + bias of numbers that are off by e, and how far off that is: sums in fp32 in any order are off by a rounding per term."""
        n = self.dim
        if self.kind == "layer":
            mean = x.mean(-1, keepdim=True)
            e = e + e.mean(-1, keepdim=True) + (n + 3) * E * x.abs().mean(-1, keepdim=True)
            x = x - mean
            e = e + E * x.abs()
        square = x.square().mean(-1, keepdim=True)
        off = 2 * (x.abs() * e).mean(-1, keepdim=True) + e.square().mean(-1, keepdim=True) + (n + 4) * E * square + 2.0 ** -126
        scale = 1.0 / torch.sqrt(square + self.eps)
        relative = off * scale * scale / 2 + (off * scale * scale) ** 2 + 6 * E
        w = torch.ones(n, dtype=torch.float64, device="cuda") if weight is None else weight.double()
        y = x * scale * w
        tol = w.abs() * scale * (e + x.abs() * (relative + e * 0)) * (1 + relative) + 2 * E * y.abs()
        if bias is not None:
            y = y + bias.double()
            tol = tol + E * y.abs()
        return y, tol

    def reference(self):
        """((residual_out, next), (how far from them they may be))."""
        n = self.used
        f32 = lambda v: float(torch.tensor(v, dtype=torch.float32))  # noqa: E731
        r, tr = torch.zeros((n, self.dim), dtype=torch.float64, device="cuda"), torch.zeros((n, self.dim), dtype=torch.float64, device="cuda")
        if self.block is not None:
            u, tu = self.block[:n].double(), torch.zeros((n, self.dim), dtype=torch.float64, device="cuda")
            if self.post:
                u, tu = self.standard(u, tu, self.post_w, self.post_b)
            if self.gate is not None:
                a, ta = activated(self.act, (self.gate[:n] if self.gate_rows else self.gate).double())
                u, tu = u * a, tu * a.abs() + u.abs() * ta + tu * ta + E * (u * a).abs()
            r, tr = f32(self.bs) * u, abs(f32(self.bs)) * tu + E * (f32(self.bs) * u).abs()
        if self.residual is not None:
            add = f32(self.rs) * self.residual[:n].double()
            r = r + add
            tr = tr + E * add.abs() + E * r.abs()
        y, ty = self.standard(r, tr, self.pre_w, self.pre_b)
        return (r, y), (tr + U[self.stream] * r.abs() + TINY[self.stream], ty + U[self.dtype] * y.abs() + TINY[self.dtype])


def check_norms(norms, label=""):
    wants = [n.reference() for n in norms]
    untouched = [[None if b is None else b[n.used:].clone() for b in (n.residual_out_b, n.next_b)] for n in norms]
    with sk.sk_norm_plan_create([n.problem() for n in norms], keepalive=norms) as plan:
        sk.sk_norm_launch(plan, stream_handle())
        torch.cuda.synchronize()
    for i, (n, ((r, y), (tr, ty))) in enumerate(zip(norms, wants)):
        if n.residual_out is not None:
            check(n.residual_out[:n.used], r, tr, f"{label} problem {i}: residual")
        if n.next is not None:
            check(n.next[:n.used], y, ty, f"{label} problem {i}: next")
        for b, was in zip((n.residual_out_b, n.next_b), untouched[i]):
            if b is not None:
                assert torch.equal(torch.nan_to_num(b[n.used:].float(), nan=1e30), torch.nan_to_num(was.float(), nan=1e30)), f"{label} problem {i}: rows behind the last were written"
                assert not n.pad or torch.isnan(b[:, n.dim:]).all(), f"{label} problem {i}: written between rows"


# ---- mixture of experts ----------------------------------------------------------------------------------------------------

class Moe:
    def __init__(self, dtype="bf16", rows=4, dim=64, experts=8, top_k=2, ffn=64, shared=0, act="silu", gated=True, scoring="softmax", normalize=1, bias=False, router="own",
                 scale=0.0, pad=0, used=None, seed=0, bias_value=None, outputs=True):
        g = generator(seed)
        dt = TORCH[dtype]
        self.dtype, self.rows, self.dim, self.experts, self.top_k, self.ffn, self.shared = dtype, rows, dim, experts, top_k, ffn, shared
        self.act, self.scoring, self.normalize, self.scale, self.pad = act, scoring, normalize, scale, pad
        self.x_b, self.x = padded(rows, dim, pad, dt)
        self.x.copy_(randn(g, rows, dim))
        self.router_dtype = "f32" if router == "f32" else dtype
        self.router = randn(g, experts, dim, scale=dim ** -0.5).to(TORCH[self.router_dtype])
        self.bias = randn(g, experts, scale=0.1) if bias else None
        if bias_value is not None:
            self.bias = torch.tensor(bias_value, dtype=torch.float32, device="cuda")

        def weights(*shape):  # with `pad` elements behind each row and, of the experts, a spare row behind each
            b = torch.full((*shape[:-2], shape[-2] + (1 if pad else 0), shape[-1] + pad), float("nan"), dtype=dt, device="cuda")
            b[..., :shape[-2], :shape[-1]] = randn(g, *shape, scale=shape[-1] ** -0.5)
            return b

        self.gate_b = weights(experts, ffn, dim) if gated else None
        self.up_b, self.down_b = weights(experts, ffn, dim), weights(experts, dim, ffn)
        self.s = [None] * 3
        if shared:
            self.s = [randn(g, shared, dim, scale=dim ** -0.5).to(dt) if gated else None, randn(g, shared, dim, scale=dim ** -0.5).to(dt), randn(g, dim, shared, scale=shared ** -0.5).to(dt)]
        self.out_b, self.out = padded(rows, dim, pad, dt)
        self.ids = torch.full((rows, top_k), -7, dtype=torch.int32, device="cuda") if outputs else None
        self.weights = torch.full((rows, top_k), float("nan"), device="cuda") if outputs else None
        self.n_rows = None if used is None else int32(used)
        self.used = rows if used is None else max(0, min(used, rows))

    def problem(self):
        p = self.pad
        return sk.make_moe_problem(
            dtype=self.dtype, router_dtype=self.router_dtype, rows=self.rows, dim=self.dim, experts=self.experts, top_k=self.top_k, ffn=self.ffn, shared_ffn=self.shared,
            act=ACT[self.act], scoring={"softmax": 0, "sigmoid": 1}[self.scoring], normalize=self.normalize, scale=self.scale, x_stride=self.dim + p if p else 0,
            out_stride=self.dim + p if p else 0, up_expert_stride=(self.ffn + 1) * (self.dim + p) if p else 0, down_expert_stride=(self.dim + 1) * (self.ffn + p) if p else 0,
            up_row_stride=self.dim + p if p else 0, down_row_stride=self.ffn + p if p else 0, n_rows=at(self.n_rows), x=at(self.x), router=at(self.router), router_bias=at(self.bias),
            gate=at(self.gate_b), up=at(self.up_b), down=at(self.down_b), shared_gate=at(self.s[0]), shared_up=at(self.s[1]), shared_down=at(self.s[2]), out=at(self.out),
            expert_ids=at(self.ids), expert_weights=at(self.weights))

    def choice(self, n):
        x = self.x[:n].double()
        logits = (x[:, None] * self.router.double()[None]).sum(-1)
        scores = torch.softmax(logits, -1) if self.scoring == "softmax" else torch.sigmoid(logits)
        rank = logits if self.scoring == "softmax" and self.bias is None else scores + (0 if self.bias is None else self.bias.double())
        rank = torch.where(torch.isnan(rank), -math.inf, rank)
        ids = torch.sort(rank, dim=-1, descending=True, stable=True).indices[:, :self.top_k]
        w = scores.gather(1, ids)
        if self.normalize:
            w = w / w.sum(-1, keepdim=True)
        return ids, w * (self.scale or 1.0)

    def through(self, x, gate, up, down):
        """An expert's output for rows x, and how far off it may be: products in fp32 in any order, act, h as the sum of
        two numbers of the type (the second is h less the first, rounded), another product of twice as many terms."""
        k, f = x.shape[-1], up.shape[0]
        z, tz = x @ up.T, (k + 8) * 2 * E * (x.abs() @ up.abs().T)
        if gate is not None:
            v, tv = x @ gate.T, (k + 8) * 2 * E * (x.abs() @ gate.abs().T)
        else:
            v, tv = z, tz
        a, ta = activated(self.act, v)
        ta = ta + 1.2 * tv  # (no act's slope is larger)
        h, th = (a * z, ta * z.abs() + tz * a.abs() + ta * tz + E * (a * z).abs()) if gate is not None else (a, ta)
        rounded = th + U[self.dtype] ** 2 * (h.abs() + th) + TINY[self.dtype]
        return h @ down.T, rounded @ down.abs().T + (2 * f + 8) * 2 * E * (h.abs() @ down.abs().T)

    def reference(self, n=None):
        n = self.used if n is None else n
        ids, w = self.choice(n)
        cut = lambda b, r, c: None if b is None else b[:, :r, :c].double()  # noqa: E731
        gate, up, down = cut(self.gate_b, self.ffn, self.dim), cut(self.up_b, self.ffn, self.dim), cut(self.down_b, self.dim, self.ffn)
        out = torch.zeros((n, self.dim), dtype=torch.float64, device="cuda")
        tol = torch.zeros_like(out)
        x = self.x[:n].double()
        if self.shared:
            y, ty = self.through(x, *(None if m is None else m.double() for m in self.s))
            out, tol = out + y, tol + ty + 4 * E * y.abs()
        for e in ids.unique().tolist():
            row, nth = torch.where(ids == e)
            y, ty = self.through(x[row], None if gate is None else gate[e], up[e], down[e])
            v = w[row, nth, None]
            out.index_add_(0, row, v * y)
            tol.index_add_(0, row, v.abs() * ty + (self.top_k + 4) * E * (v * y).abs())
        return out, tol + U[self.dtype] * (out.abs() + tol) + TINY[self.dtype], ids, w


def check_moe(m, label="", n=None):
    out, tol, ids, w = m.reference(n)
    n = out.shape[0]
    if m.ids is not None:
        assert torch.equal(m.ids[:n].long(), ids), f"{label}: other experts"
        check(m.weights[:n], w, 4 * E * w.abs() + 2.0 ** -126, f"{label}: weights")
        assert (m.ids[n:] == -7).all() and torch.isnan(m.weights[n:]).all(), f"{label}: choices behind the last row were written"
    check(m.out[:n], out, tol, f"{label}: out")
    # the rounding of the outputs is at most one unit of each; what came before it is far smaller, measured over all outputs
    if n and float(out.norm()) > 0:
        assert float((m.out[:n].double() - out).norm()) <= 1.1 * U[m.dtype] * float(out.norm()), f"{label}: {float((m.out[:n].double() - out).norm() / out.norm()):.3g}"
    assert torch.isnan(m.out_b[n:]).all() and (not m.pad or torch.isnan(m.out_b[:, m.dim:]).all()), f"{label}: written outside the rows"


def run_moe(moes, label="", **params):
    with sk.sk_moe_plan_create([m.problem() for m in moes], sk.sk_layer_params_default(**params), keepalive=moes) as plan:
        sk.sk_moe_launch(plan, stream_handle())
        torch.cuda.synchronize()
        first = [m.out.clone() for m in moes]
        for i, m in enumerate(moes):
            check_moe(m, f"{label} problem {i}")
        sk.sk_moe_launch(plan, stream_handle())  # again: the workspace was left as it was found, the same bits
        torch.cuda.synchronize()
    for i, m in enumerate(moes):
        assert torch.equal(first[i][:m.used], m.out[:m.used]), f"{label} problem {i}: two launches differ"


# ---- verification ----------------------------------------------------------------------------------------------------------

class Verify:
    def __init__(self, dtype="bf16", vocab=300, counts=(2,), draft="logits", temperature=1.0, temperatures=None, pad=0, spread=2.0, seed=0, spare=0):
        g = generator(seed)
        self.dtype, self.vocab, self.counts, self.pad, self.draft = dtype, vocab, list(counts), pad, draft
        self.firsts = [sum(counts[:i]) for i in range(len(counts) + 1)]  # counts: rows of each sequence, drafts and one more
        self.rows = max(self.firsts[-1] + spare, 1)
        dt = TORCH[dtype]
        self.logits_b, self.logits = padded(self.rows, vocab, pad, dt)
        self.logits.copy_(randn(g, self.rows, vocab, scale=spread))
        self.draft_logits = None
        guess = self.logits.float() * 0.8 + randn(g, self.rows, vocab, scale=0.5)
        if draft == "logits":
            self.draft_b, self.draft_logits = padded(self.rows, vocab, pad, dt)
            self.draft_logits.copy_(guess)
        noise = -torch.log(torch.empty((self.rows, vocab), device="cuda").exponential_(generator=g))
        self.drafted = (guess + noise).argmax(-1).to(torch.int32) if draft != "none" else None
        self.temperature = temperature
        self.temperatures = None if temperatures is None else torch.tensor(temperatures, dtype=torch.float32, device="cuda")
        self.accept_random = torch.rand((self.rows,), generator=g, device="cuda")
        self.sample_random = torch.rand((len(counts),), generator=g, device="cuda")
        self.first_row = int32(*self.firsts)
        self.tokens = torch.full((self.rows,), -9, dtype=torch.int32, device="cuda")
        self.accepted = torch.full((len(counts),), -9, dtype=torch.int32, device="cuda")

    def problem(self):
        s = self.vocab + self.pad if self.pad else 0
        return sk.make_verify_problem(
            dtype=self.dtype, sequences=len(self.counts), rows=self.rows, vocab=self.vocab, temperature=self.temperature, logits_stride=s, draft_stride=s,
            first_row=at(self.first_row), logits=at(self.logits), drafted=at(self.drafted), draft_logits=at(self.draft_logits), temperatures=at(self.temperatures),
            accept_random=at(self.accept_random), sample_random=at(self.sample_random), tokens=at(self.tokens), accepted=at(self.accepted))

    def probabilities(self, x, t):
        """The distribution of a row, or None."""
        if torch.isnan(x).any() or (x == math.inf).any() or (x == -math.inf).all():
            return None
        if not t > 0:
            p = torch.zeros(self.vocab, dtype=torch.float64, device="cuda")
            p[int((x == x.max()).nonzero()[0])] = 1.0
            return p
        return torch.softmax((x.double() - x.double().max()) / t, 0)

    def reference(self):
        tokens, accepted = [-9] * self.rows, []
        for s, count in enumerate(self.counts):
            if not count:
                accepted.append(0)
                continue
            r0, n = self.firsts[s], 0
            t = self.temperature if self.temperatures is None else float(self.temperatures[s])
            cut = lambda u: min(max(u, 0.0), 1 - 2.0 ** -24) if u == u else 0.0  # noqa: E731
            while True:
                row = r0 + n
                p = self.probabilities(self.logits[row], t)
                w = p
                if p is None or n == count - 1 or self.drafted is None:
                    break
                d = int(self.drafted[row])
                if not 0 <= d < self.vocab:
                    break
                q = None if self.draft_logits is None or not t > 0 else self.probabilities(self.draft_logits[row], t)
                if q is None:
                    q = torch.zeros_like(p)
                    q[d] = 1.0
                if cut(float(self.accept_random[row])) * float(q[d]) < float(p[d]):
                    tokens[row] = d
                    n += 1
                    continue
                w = (p - q).clamp(min=0)
                w = w if float(w.sum()) > 0 else p
                break
            if w is None:
                tokens[r0 + n] = -1
            else:
                upto = w.cumsum(0)
                past = (upto > cut(float(self.sample_random[s])) * upto[-1]) & (w > 0)
                tokens[r0 + n] = int(past.nonzero()[0]) if past.any() else int((w > 0).nonzero()[-1])
            for i in range(n + 1, count):
                tokens[r0 + i] = -1
            accepted.append(n)
        return tokens, accepted


def check_verify(problems, label="", **params):
    wants = [v.reference() for v in problems]
    with sk.sk_verify_plan_create([v.problem() for v in problems], sk.sk_layer_params_default(**params), keepalive=problems) as plan:
        for turn in range(2):  # again: the workspace was left as it was found
            for v in problems:
                v.tokens.fill_(-9)
                v.accepted.fill_(-9)
            sk.sk_verify_launch(plan, stream_handle())
            torch.cuda.synchronize()
            for i, (v, (tokens, accepted)) in enumerate(zip(problems, wants)):
                assert v.accepted.tolist() == accepted, f"{label} problem {i} launch {turn}: accepted {v.accepted.tolist()} for {accepted}"
                assert v.tokens.tolist() == tokens, f"{label} problem {i} launch {turn}: tokens {v.tokens.tolist()} for {tokens}"
