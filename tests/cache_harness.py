"""Inputs on the device, plain results in 64 bits on the host, and how far the kernels may be from them, for the operators over paged
caches."""
import math

import torch

import paper_1901_10008_amd as sk

TORCH = {"bf16": torch.bfloat16, "f16": torch.float16}
# Unit roundoff of the types, and half of the spacing of their smallest numbers.
U = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"bf16": 2.0 ** -134, "f16": 2.0 ** -25}


def stream_handle():
    return torch.cuda.current_stream().cuda_stream


class Tenant:
    """A cache with its pages in no order and a step on it.  seqs: (tokens, new rows) of each sequence."""

    def __init__(self, dtype="bf16", heads=(4, 2, 64), seqs=((5, 1),), page=16, window=0, sinks=0, scale=0.0, layout="page", rotary=0, neighbours=False,
                 norm=True, eps=1e-5, seed=0, max_new=0, spare_rows=0, q_pad=0, out_pad=0, fill=0.0, spare_pages=2, with_qkv=False, with_out=True, q_scale=1.0):
        self.dtype, (self.hq, self.hkv, self.d), self.seqs, self.page = dtype, heads, list(seqs), page
        self.window, self.sinks, self.scale, self.eps = window, sinks, scale, eps
        self.rotary, self.neighbours, self.norm = rotary, neighbours, norm
        dt = TORCH[dtype]
        g = torch.Generator().manual_seed(seed)
        held = [-(-t // page) for t, _ in seqs]
        self.columns = max(max(held), 1) + 1
        self.count = sum(held) + spare_pages
        order = torch.randperm(self.count, generator=g).to(torch.int32)
        self.table = torch.full((len(seqs), self.columns), -1, dtype=torch.int32)
        at = 0
        for s, n in enumerate(held):
            self.table[s, :n] = order[at:at + n]
            at += n
        self.rows_used = sum(n for _, n in seqs)
        self.rows = max(self.rows_used + spare_rows, 1)
        self.max_new = max_new
        self.lengths = torch.tensor([t for t, _ in seqs], dtype=torch.int32)
        self.firsts = torch.tensor([sum(n for _, n in seqs[:i]) for i in range(len(seqs) + 1)], dtype=torch.int32)
        # logical values, rounded to the type; `fill` stands wherever no token is
        shape = (self.count, self.hkv, page, self.d)
        k = torch.full(shape, fill, dtype=torch.float32)
        v = torch.full(shape, fill, dtype=torch.float32)
        for s, (t, _) in enumerate(seqs):
            for i in range(t):
                p, slot = int(self.table[s, i // page]), i % page
                k[p, :, slot] = torch.randn((self.hkv, self.d), generator=g)
                v[p, :, slot] = torch.randn((self.hkv, self.d), generator=g)
        self.k, self.v = k.to(dt), v.to(dt)
        self.q = (torch.randn((self.rows, self.hq, self.d), generator=g) * q_scale).to(dt)
        self.qkv = torch.randn((self.rows, self.hq + 2 * self.hkv, self.d), generator=g).to(dt) if with_qkv else None
        self.qw = (1 + 0.2 * torch.randn((self.d,), generator=g)).to(dt)
        self.kw = (1 + 0.2 * torch.randn((self.d,), generator=g)).to(dt)
        positions = self.columns * page
        if rotary:
            angle = torch.arange(positions)[:, None].double() * 100.0 ** (-torch.arange(rotary // 2).double() / (rotary // 2))
            self.cos, self.sin = angle.cos().float(), angle.sin().float()
        self.layout, self.q_pad, self.out_pad, self.with_out = layout, q_pad, out_pad, with_out

    # ---- on the device ----
    def to_device(self):
        dt = TORCH[self.dtype]
        if self.layout == "page":  # [page][head][token][dim]
            self.dk, self.dv = self.k.cuda().contiguous(), self.v.cuda().contiguous()
            self.strides = (0, 0, 0)
            self.kp, self.vp = self.dk.data_ptr(), self.dv.data_ptr()
        elif self.layout == "token":  # [page][k or v][token][head][dim]
            self.pool = torch.stack([self.k.transpose(1, 2), self.v.transpose(1, 2)], 1).contiguous().cuda()
            one = self.page * self.hkv * self.d
            self.strides = (2 * one, self.d, self.hkv * self.d)
            self.kp, self.vp = self.pool.data_ptr(), self.pool.data_ptr() + 2 * one
        else:  # "heads": [head][page][token][dim], with a gap behind each token
            gap = 8
            self.dk, self.dv = (torch.nn.functional.pad(x.transpose(0, 1), (0, gap)).contiguous().cuda() for x in (self.k, self.v))
            t = self.d + gap
            self.strides = (self.page * t, self.count * self.page * t, t)
            self.kp, self.vp = self.dk.data_ptr(), self.dv.data_ptr()
        q = torch.full((self.rows, self.hq, self.d + self.q_pad), float("nan"), dtype=dt)
        q[:, :, :self.d] = self.q
        self.dq = q.cuda()
        self.dout = torch.full((self.rows, self.hq, self.d + self.out_pad), float("nan"), dtype=dt).cuda() if self.with_out else None
        self.keep = [x.cuda().contiguous() for x in (self.table, self.lengths, self.firsts)]
        f = dict(dtype=self.dtype, q_heads=self.hq, kv_heads=self.hkv, head_dim=self.d, page_tokens=self.page, num_pages=self.count, sequences=len(self.seqs),
                 pages_per_sequence=self.columns, rows=self.rows, max_new=self.max_new, window=self.window, sinks=self.sinks, scale=self.scale, eps=self.eps,
                 page_stride=self.strides[0], kv_head_stride=self.strides[1], token_stride=self.strides[2], k=self.kp, v=self.vp,
                 page_table=self.keep[0].data_ptr(), lengths=self.keep[1].data_ptr(), first_row=self.keep[2].data_ptr(), q=self.dq.data_ptr())
        if self.q_pad:
            f |= dict(q_row_stride=self.hq * (self.d + self.q_pad), q_head_stride=self.d + self.q_pad)
        if self.with_out:
            f |= dict(out=self.dout.data_ptr())
            if self.out_pad:
                f |= dict(out_row_stride=self.hq * (self.d + self.out_pad), out_head_stride=self.d + self.out_pad)
        if self.qkv is not None:
            self.dqkv = self.qkv.cuda().contiguous()
            f |= dict(qkv=self.dqkv.data_ptr())
            if self.norm:
                self.keep += [self.qw.cuda(), self.kw.cuda()]
                f |= dict(q_weight=self.keep[-2].data_ptr(), k_weight=self.keep[-1].data_ptr())
            if self.rotary:
                self.keep += [self.cos.cuda(), self.sin.cuda()]
                f |= dict(cos=self.keep[-2].data_ptr(), sin=self.keep[-1].data_ptr(), positions=self.cos.shape[0], rotary_dim=self.rotary, neighbours=int(self.neighbours))
        self.fields = f
        return sk.make_attn_problem(**f)

    def out(self):
        return self.dout[:, :, :self.d].cpu()

    def cache(self):
        """(k, v) from the device as [page][head][token][dim]."""
        if self.layout == "page":
            return self.dk.cpu(), self.dv.cpu()
        if self.layout == "token":
            p = self.pool.cpu()
            return p[:, 0].transpose(1, 2), p[:, 1].transpose(1, 2)
        return tuple(x.cpu().transpose(0, 1)[..., :self.d] for x in (self.dk, self.dv))

    # ---- in 64 bits ----
    def tokens_of(self, s, h, n):
        """Keys and values of the first n tokens of a sequence; NaN where its page is not one of the cache's."""
        k, v = torch.full((n, self.d), math.nan, dtype=torch.float64), torch.full((n, self.d), math.nan, dtype=torch.float64)
        there = torch.zeros(n, dtype=torch.bool)
        for i in range(n):
            p = int(self.table[s, i // self.page])
            if 0 <= p < self.count:
                k[i], v[i], there[i] = self.k[p, h, i % self.page].double(), self.v[p, h, i % self.page].double(), True
        return k, v, there

    def attend(self):
        """(outputs, how far from them each may be)."""
        out = torch.zeros((self.rows, self.hq, self.d), dtype=torch.float64)
        tol = torch.zeros_like(out)
        u, scale = U[self.dtype], self.scale or self.d ** -0.5
        for s, (t, new) in enumerate(self.seqs):
            for h in range(self.hkv):
                k, v, there = self.tokens_of(s, h, t)
                for n in range(new):
                    pos, row = t - new + n, int(self.firsts[s]) + n
                    j = torch.arange(t)
                    see = (j <= pos) & there
                    if self.window:
                        see &= (pos - j < self.window) | (j < self.sinks)
                    if not see.any():
                        continue
                    ks, vs, count = k[see], v[see], int(see.sum())
                    for g in range(self.hq // self.hkv):
                        q = self.q[row, h * (self.hq // self.hkv) + g].double()
                        score = ks @ q * scale
                        w = torch.softmax(score, 0)
                        o = w @ vs
                        # The scores' products are exact and their sums fp32 in some order; scaling, the subtraction of the maximum and
                        # exp2 add a few roundings of numbers as large as the scores.  A weight is off by that twice (its own score and the
                        # sum), is rounded to the type, and products are summed in fp32 with a rescaling per block of keys.
                        delta = 2.0 ** -23 * ((self.d + 4) * float((ks.abs() @ q.abs()).max()) * abs(scale) + 4 * float(score.abs().max()) + 8)
                        spread = w @ vs.abs()
                        tol[row, h * (self.hq // self.hkv) + g] = (spread * (u + 2 * delta + (count + 64) * 2.0 ** -23) + u * o.abs() + TINY[self.dtype]
                                                                  + (2.0 ** -25 * vs.abs().sum(0) if self.dtype == "f16" else 0.0))
                        out[row, h * (self.hq // self.hkv) + g] = o
        return out, tol

    def append(self):
        """(queries, keys, values) as they shall be, and how far from them queries and keys may be; keys and values are the cache's where
        nothing is written."""
        u, r = U[self.dtype], self.rotary
        q, tq = torch.zeros((self.rows, self.hq, self.d), dtype=torch.float64), torch.zeros((self.rows, self.hq, self.d), dtype=torch.float64)
        k, v, tk = self.k.double(), self.v.clone(), torch.zeros(self.k.shape, dtype=torch.float64)
        a = list(range(0, r, 2)) if self.neighbours else list(range(r // 2))
        b = [x + 1 for x in a] if self.neighbours else [x + r // 2 for x in a]
        for s, (t, new) in enumerate(self.seqs):
            for n in range(new):
                pos, row = t - new + n, int(self.firsts[s]) + n
                for h in range(self.hq + self.hkv):
                    x = self.qkv[row, h].double()
                    if self.norm:
                        x = x / torch.sqrt((x * x).mean() + self.eps) * (self.qw if h < self.hq else self.kw).double()
                    y, most = x.clone(), x.abs()
                    if r:
                        c, si = self.cos[max(pos, 0)].double(), self.sin[max(pos, 0)].double()
                        y[a], y[b] = x[a] * c - x[b] * si, x[b] * c + x[a] * si
                        most = most.clone()
                        most[a], most[b] = (x[a] * c).abs() + (x[b] * si).abs(), (x[b] * c).abs() + (x[a] * si).abs()
                    # the sum of squares in any order, its root, two or three products, one rounding at the end
                    tol = u * y.abs() + most * (self.d + 24) * 2.0 ** -24 + TINY[self.dtype] if (self.norm or r) else torch.zeros_like(y)
                    if h < self.hq:
                        q[row, h], tq[row, h] = y, tol
                    elif pos >= 0:
                        p = int(self.table[s, pos // self.page])
                        if 0 <= p < self.count:
                            k[p, h - self.hq, pos % self.page], tk[p, h - self.hq, pos % self.page] = y, tol
                            v[p, h - self.hq, pos % self.page] = self.qkv[row, h + self.hkv]
        return (q, k, v), (tq, tk)


def assert_close(got, want, tol, label=""):
    got = got.double()
    bad = ~((got - want).abs() <= tol)
    if bad.any():
        i = tuple(int(x) for x in bad.nonzero()[0])
        raise AssertionError(f"{label}: {int(bad.sum())} of {bad.numel()} off, first at {i}: {float(got[i])!r} for {float(want[i])!r}, allowed {float(tol[i]):.3g}")


def check_attend(tenants, label="", **params):
    problems = [t.to_device() for t in tenants]
    with sk.sk_attn_plan_create(problems, sk.sk_attn_params_default(**params)) as plan:
        sk.sk_attn_launch(plan, stream_handle())
        torch.cuda.synchronize()
        first = [t.out() for t in tenants]
        sk.sk_attn_launch(plan, stream_handle())  # again: the workspace was left as it was found, the same bits
        torch.cuda.synchronize()
    for i, t in enumerate(tenants):
        want, tol = t.attend()
        n = t.rows_used
        assert_close(first[i][:n], want[:n], tol[:n], f"{label} tenant {i}")
        assert torch.isnan(first[i][n:]).all(), f"{label} tenant {i}: rows of no sequence were written"
        assert torch.equal(first[i][:n].view(torch.int16), t.out()[:n].view(torch.int16)), f"{label} tenant {i}: two launches differ"
        if t.out_pad:
            assert torch.isnan(t.dout[:, :, t.d:]).all(), f"{label} tenant {i}: written between rows"
    return first
