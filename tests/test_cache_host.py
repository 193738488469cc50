"""Host side of the operators over paged caches, no GPU: what plans refuse, the account of pages against a plain one, layouts, sanitizers."""
import ctypes
import os
import random
import re
import shutil
import subprocess

import pytest

import paper_1901_10008_amd as sk

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

BASE = 1 << 40  # addresses that nothing touches: plans here are host-only
GOOD = dict(dtype="bf16", q_heads=8, kv_heads=2, head_dim=64, page_tokens=16, num_pages=100, sequences=4, pages_per_sequence=10, rows=32, k=BASE, v=BASE << 1,
            page_table=BASE + 4, lengths=BASE + 8, first_row=BASE + 12, q=BASE << 2, out=BASE << 3, qkv=BASE << 4, cos=BASE, sin=BASE, positions=160, rotary_dim=64,
            eps=1e-5)


def plan(*problems):
    return sk.sk_attn_plan_create([sk.make_attn_problem(**p) for p in problems], sk.sk_attn_params_default(host_only=1))


def test_good_problems_are_planned():
    with plan(GOOD) as p:
        launches, workspace = sk.sk_attn_plan_info(p)
        assert launches == 1 and workspace > 0
        for call in (sk.sk_attn_append, sk.sk_attn_launch):
            with pytest.raises(sk.SkError) as e:
                call(p)
            assert e.value.status == sk.SK_ERR_STATE and "host-only" in e.value.detail
    with plan(GOOD | dict(qkv=0, cos=0, sin=0), GOOD | dict(out=0, q=BASE << 5), GOOD | dict(dtype="f16", q=BASE << 6, out=BASE << 7, head_dim=256, window=5, sinks=2)) as p:
        assert sk.sk_attn_plan_info(p)[0] == 2
    with plan() as p:
        assert sk.sk_attn_plan_info(p) == (0, 0)


INVALID, UNSUPPORTED, OVERLAP = -1, -2, -3
REFUSALS = [
    (dict(dtype="f32"), UNSUPPORTED), (dict(dtype=7), UNSUPPORTED), (dict(head_dim=60), UNSUPPORTED), (dict(head_dim=264), UNSUPPORTED), (dict(head_dim=0), INVALID),
    (dict(q_heads=0), INVALID), (dict(kv_heads=0), INVALID), (dict(q_heads=7), INVALID), (dict(page_tokens=8), UNSUPPORTED), (dict(page_tokens=48), UNSUPPORTED),
    (dict(page_tokens=1 << 17), UNSUPPORTED), (dict(page_tokens=0), INVALID), (dict(num_pages=0), INVALID), (dict(sequences=-1), INVALID), (dict(sequences=(1 << 20) + 1), UNSUPPORTED),
    (dict(pages_per_sequence=0), INVALID), (dict(pages_per_sequence=1 << 27, rotary_dim=0), UNSUPPORTED), (dict(rows=0), INVALID), (dict(max_new=-1), INVALID),
    (dict(window=-1), INVALID), (dict(sinks=-1), INVALID), (dict(reserved=1), INVALID), (dict(rotary_dim=63), INVALID), (dict(rotary_dim=66), INVALID),
    (dict(rotary_dim=-2), INVALID), (dict(neighbours=2), INVALID), (dict(positions=159), INVALID), (dict(cos=0), INVALID), (dict(sin=0), INVALID),
    (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(scale=float("inf")), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(k=0), INVALID), (dict(v=0), INVALID), (dict(page_table=0), INVALID), (dict(lengths=0), INVALID), (dict(first_row=0), INVALID), (dict(q=0), INVALID),
    (dict(qkv=0, out=0), INVALID), (dict(k=BASE + 8), UNSUPPORTED), (dict(q=(BASE << 2) + 2), UNSUPPORTED), (dict(cos=BASE + 4), UNSUPPORTED),
    (dict(lengths=BASE + 1), UNSUPPORTED), (dict(q_weight=BASE + 8), UNSUPPORTED), (dict(rows=1 << 30), UNSUPPORTED),
    (dict(token_stride=-8), INVALID), (dict(token_stride=1 << 26, kv_head_stride=64, page_stride=1 << 31), UNSUPPORTED), (dict(token_stride=64), INVALID), (dict(token_stride=64, kv_head_stride=1024), INVALID),
    (dict(token_stride=64, kv_head_stride=960, page_stride=2048), INVALID), (dict(token_stride=64, kv_head_stride=1024, page_stride=2040), INVALID),
    (dict(token_stride=68, kv_head_stride=1088, page_stride=2176), UNSUPPORTED), (dict(token_stride=128, kv_head_stride=64, page_stride=2040), INVALID),
    (dict(token_stride=64, kv_head_stride=1024 * 99, page_stride=1024), INVALID), (dict(qkv_row_stride=760), INVALID), (dict(qkv_row_stride=772), UNSUPPORTED),
    (dict(q_row_stride=512, q_head_stride=56), INVALID), (dict(q_head_stride=64), INVALID), (dict(out_row_stride=504, out_head_stride=64), INVALID),
    (dict(out_row_stride=544, out_head_stride=68), UNSUPPORTED), (dict(page_stride=1 << 61, token_stride=64, kv_head_stride=1024), UNSUPPORTED),
    (dict(out=(BASE << 2) + 64), OVERLAP),
]


@pytest.mark.parametrize("change,status", REFUSALS)
def test_refusals(change, status):
    with pytest.raises(sk.SkError) as e:
        plan(GOOD | change)
    assert e.value.status == status, e.value.detail
    assert e.value.detail


@pytest.mark.parametrize("change", [
    dict(sequences=1 << 20, q_heads=8, kv_heads=8, rows=1 << 21),  # two blocks of rows for each of 2^20 sequences' 8 heads: 2^24 workgroups of 256
    dict(rows=1 << 27),  # rows of append: four a workgroup, 2^25
    dict(rows=1 << 24, q_heads=127, kv_heads=127, qkv=0, sequences=1000),  # blocks of 128 rows: 127 x 2^17, and one for the last rows of each sequence
    dict(sequences=1 << 20, q_heads=1 << 28, kv_heads=1 << 28, rows=1, head_dim=8, num_pages=1, rotary_dim=0, qkv=0, q=1 << 44, out=1 << 45),  # 2^48
    dict(q_heads=1 << 30, kv_heads=1 << 29, rows=1, head_dim=8, num_pages=1, rotary_dim=0, q=1 << 44, out=1 << 45)])  # numbers of heads beyond 2^30
def test_more_workgroups_than_a_launch_can_have(change):
    """The runtime refuses launches of 2^32 threads and more: plans of more than 2^24 - 1 workgroups are refused, not their launches."""
    with pytest.raises(sk.SkError) as e:
        plan(GOOD | change)
    assert e.value.status == UNSUPPORTED, e.value.detail
    assert "grid" in e.value.detail or "heads" in e.value.detail


@pytest.mark.parametrize("scale", [3e38, -2.4e38])
def test_scales_beyond_fp32(scale):
    """Scores are kept in powers of two: the scale times log2(e) has to be a number too."""
    with pytest.raises(sk.SkError) as e:
        plan(GOOD | dict(scale=scale))
    assert e.value.status == INVALID and "scale" in e.value.detail
    plan(GOOD | dict(scale=2.3e38)).close()


def test_the_largest_grids_are_planned():
    plan(GOOD | dict(sequences=1 << 20, q_heads=8, kv_heads=8, rows=1 << 20, max_new=1)).close()
    plan(GOOD | dict(rows=(1 << 26) - 64, out=0)).close()


def test_strides_that_are_fine():
    for change in (dict(token_stride=128, kv_head_stride=64, page_stride=2048), dict(token_stride=128, kv_head_stride=64, page_stride=2048 * 2),
                   dict(token_stride=64, kv_head_stride=1024, page_stride=2048 + 8), dict(token_stride=64, kv_head_stride=1024 * 100, page_stride=1024),
                   dict(q_row_stride=64, q_head_stride=64 * 32), dict(out_row_stride=600, out_head_stride=72)):
        plan(GOOD | change).close()


def test_outputs_of_two_problems_may_not_meet():
    end = 32 * 8 * 64 * 2
    with pytest.raises(sk.SkError) as e:
        plan(GOOD, GOOD | dict(q=BASE << 5, out=(BASE << 3) + end - 16))
    assert e.value.status == OVERLAP
    plan(GOOD, GOOD | dict(q=BASE << 5, out=(BASE << 3) + end)).close()


def test_bad_calls():
    L = sk.cache_lib()
    out = ctypes.c_void_p()
    assert L.sk_attn_plan_create(None, 0, None, None) == INVALID
    assert L.sk_attn_plan_create(None, 1, ctypes.byref(sk.sk_attn_params_default(host_only=1)), ctypes.byref(out)) == INVALID and not out.value
    for bad in (dict(host_only=2), dict(host_only=1, workgroups=-1), dict(host_only=1, workgroups=1 << 20)):
        assert L.sk_attn_plan_create(None, 0, ctypes.byref(sk.sk_attn_params_default(**bad)), ctypes.byref(out)) == INVALID
    assert L.sk_attn_append(None, None) == INVALID and L.sk_attn_launch(None, None) == INVALID and L.sk_attn_plan_destroy(None) == 0
    assert L.sk_pages_destroy(None) == 0 and L.sk_pages_resize(None, None, None, 0) == INVALID and L.sk_pages_compact(None) == INVALID
    for args in ((0, 16, 1, 1), (4, 0, 1, 1), (4, 16, 0, 1), (4, 16, 1, 0)):
        with pytest.raises(sk.SkError) as e:
            sk.sk_pages_create(*args)
        assert e.value.status == INVALID
    with pytest.raises(sk.SkError) as e:
        sk.sk_pages_create(4, 1 << 16, 1, 1 << 16)
    assert e.value.status == UNSUPPORTED
    arrays = sk.make_page_arrays([(BASE, 64)])
    for arr, frm, to, status in ((arrays, [0], [9], INVALID), (arrays, [-1], [1], INVALID), (arrays, [0, 1], [2, 2], OVERLAP), (arrays, [0, 2], [2, 3], OVERLAP),
                                 (arrays, [1], [1], OVERLAP), (sk.make_page_arrays([(0, 64)]), [0], [1], INVALID), (sk.make_page_arrays([(BASE, 0)]), [0], [1], INVALID),
                                 (sk.make_page_arrays([(BASE, 24)]), [0], [1], UNSUPPORTED), (sk.make_page_arrays([(BASE + 8, 32)]), [0], [1], UNSUPPORTED)):
        with pytest.raises(sk.SkError) as e:
            sk.sk_pages_copy(arr, 9, frm, to)
        assert e.value.status == status, e.value.detail


def test_header_and_binding_agree():
    with open(os.path.join(ROOT, "include", "sk_cache.h")) as f:
        text = re.sub(r"/\*.*?\*/", "", f.read(), flags=re.S)
    assert set(re.findall(r"\b(sk_[a-z_]+)\s*\(", text)) == set(sk.CACHE_SYMBOLS)
    assert ctypes.sizeof(sk.sk_attn_problem) == 18 * 4 + 8 * 8 + 12 * 8 and ctypes.sizeof(sk.AttnParams) == 16 and ctypes.sizeof(sk.sk_page_array) == 16
    names = re.search(r"typedef struct \{([^}]*)\} sk_attn_problem;", text).group(1)
    declared = [n for line in names.split(";") for n in re.findall(r"\*?\s*(\w+)\s*(?:,|$)", line.strip())]
    assert declared == [n for n, _ in sk.sk_attn_problem._fields_]


# ---- the account of pages ------------------------------------------------------------------------------------------------------

class Plain:
    """Sequences as lists of page numbers, pages' contents as what was written to them."""

    def __init__(self, pages, page, seqs, columns):
        self.pages, self.page, self.columns = pages, page, columns
        self.rows, self.tokens = [[] for _ in range(seqs)], [0] * seqs

    def refs(self, p):
        return sum(r.count(p) for r in self.rows)

    def lowest(self):
        used = {p for r in self.rows for p in r}
        return next(p for p in range(self.pages) if p not in used)

    def resize(self, seqs, tokens):
        held = [-(-t // self.page) for t in tokens]
        rows = [list(r) for r in self.rows]
        try:
            for s, t, h in zip(seqs, tokens, held):
                if t < self.tokens[s]:
                    self.rows[s] = self.rows[s][:h]
            for s, t, h in zip(seqs, tokens, held):
                if t > self.tokens[s]:
                    if self.tokens[s] % self.page and self.refs(self.rows[s][-1]) > 1:
                        self.rows[s][-1] = self.lowest()
                    while len(self.rows[s]) < h:
                        self.rows[s].append(self.lowest())
        except StopIteration:
            self.rows = rows
            return False
        for s, t in zip(seqs, tokens):
            self.tokens[s] = t
        return True

    def compact(self):
        used = sorted({p for r in self.rows for p in r})
        free = [p for p in range(len(used)) if p not in used]
        now = dict(zip([p for p in used if p >= len(used)], free))
        self.rows = [[now.get(p, p) for p in r] for r in self.rows]


@pytest.mark.parametrize("seed", range(8))
def test_account_against_a_plain_one(seed):
    rng = random.Random(seed)
    shape = (rng.choice([5, 17, 60]), rng.choice([1, 4, 16]), rng.choice([1, 3, 8]), rng.choice([1, 4, 9]))
    plain, account = Plain(*shape), sk.sk_pages_create(*shape)
    seqs, refused = range(shape[2]), 0
    for _ in range(600):
        what = rng.random()
        if what < 0.2:
            s = rng.choice(seqs)
            to = [t for t in seqs if t != s and not plain.tokens[t]][:rng.randrange(3)]
            sk.sk_pages_fork(account, s, to)
            for t in to:
                plain.rows[t], plain.tokens[t] = list(plain.rows[s]), plain.tokens[s]
        elif what < 0.3:
            sk.sk_pages_compact(account)
            plain.compact()
        else:
            some = rng.sample(list(seqs), rng.randrange(1, len(seqs) + 1))
            tokens = [rng.choice([0, plain.tokens[s], min(plain.tokens[s] + 1, shape[1] * shape[3]), rng.randrange(shape[1] * shape[3] + 1)]) for s in some]
            if plain.resize(some, tokens):
                sk.sk_pages_resize(account, some, tokens)
            else:
                refused += 1
                with pytest.raises(sk.SkError) as e:
                    sk.sk_pages_resize(account, some, tokens)
                assert e.value.status == sk.SK_ERR_ALLOC
        assert sk.sk_pages_state(account)[0] == shape[0] - len({p for r in plain.rows for p in r})
        for s in seqs:
            assert sk.sk_pages_state(account, s) == (plain.tokens[s], plain.rows[s] + [-1] * (shape[3] - len(plain.rows[s])))
    account.close()


def test_account_refuses():
    a = sk.sk_pages_create(10, 16, 4, 3)
    sk.sk_pages_resize(a, [0], [20])
    for call in (lambda: sk.sk_pages_resize(a, [4], [1]), lambda: sk.sk_pages_resize(a, [-1], [1]), lambda: sk.sk_pages_resize(a, [1, 1], [1, 2]),
                 lambda: sk.sk_pages_resize(a, [1], [-1]), lambda: sk.sk_pages_resize(a, [1], [49]), lambda: sk.sk_pages_fork(a, 0, [0]),
                 lambda: sk.sk_pages_fork(a, 1, [0]), lambda: sk.sk_pages_fork(a, 9, [1]), lambda: sk.sk_pages_fork(a, 0, [1, 1]),
                 lambda: sk.sk_pages_state(a, 7)):
        with pytest.raises(sk.SkError) as e:
            call()
        assert e.value.status == INVALID and e.value.detail
    with pytest.raises(ValueError):
        sk.sk_pages_resize(a, [1], [1, 2])
    assert sk.sk_pages_state(a) == (8, 0) and sk.sk_pages_state(a, 1) == (0, [-1] * 3)
    a.close()


SAN = ["-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-static-libasan", "-g", "-O1"]
ENV = dict(os.environ, ASAN_OPTIONS="verify_asan_link_order=0:detect_leaks=1", UBSAN_OPTIONS="print_stacktrace=1")


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host C++ compiler")
def test_host_code_under_sanitizers(tmp_path):
    exe, csrc = str(tmp_path / "cache_driver"), os.path.join(ROOT, "paper_1901_10008_amd", "csrc")
    res = subprocess.run(["g++", "-std=c++17", *SAN, "-I", os.path.join(ROOT, "include"), "-I", csrc, os.path.join(ROOT, "tests", "sanitize", "cache_driver.cpp"),
                          os.path.join(csrc, "cache_plan.cpp"), "-o", exe], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    res = subprocess.run([exe], capture_output=True, text=True, env=ENV)
    assert res.returncode == 0 and "cache_driver: ok" in res.stdout, res.stdout + res.stderr


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host C++ compiler")
def test_account_without_memory(tmp_path):
    """Calls that run out of host memory, at whichever allocation, leave the account as it was."""
    exe, csrc = str(tmp_path / "cache_memory_driver"), os.path.join(ROOT, "paper_1901_10008_amd", "csrc")
    res = subprocess.run(["g++", "-std=c++17", "-g", "-O1", "-Wall", "-D_GLIBCXX_ASSERTIONS", "-I", os.path.join(ROOT, "include"), "-I", csrc,
                          os.path.join(ROOT, "tests", "sanitize", "cache_memory_driver.cpp"), os.path.join(csrc, "cache_plan.cpp"), "-o", exe], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    res = subprocess.run([exe], capture_output=True, text=True)
    assert res.returncode == 0 and "cache_memory_driver: ok" in res.stdout, res.stdout + res.stderr


def _all(blob, key):
    found = []
    for m in re.finditer(re.escape(key), blob):
        at = m.end()  # a MessagePack unsigned integer
        n = {0xCC: 1, 0xCD: 2, 0xCE: 4}.get(blob[at], 0)
        found.append(int.from_bytes(blob[at + 1:at + 1 + n], "big") if n else blob[at])
    return found


def test_no_kernel_spills_or_has_a_stack():
    with open(sk.cache.cache_lib_path(), "rb") as f:
        blob = f.read()
    n = 8  # four of attention, two each of append and copies
    assert len(_all(blob, b".vgpr_count")) == n
    assert _all(blob, b".vgpr_spill_count") == [0] * n and _all(blob, b".private_segment_fixed_size") == [0] * n


def test_ids_of_any_kind():
    """Lists, iterators and arrays of other types mean the numbers in them; tokens up to the last that an account can hold."""
    with sk.sk_pages_create(60, 16, 4, 20) as pages:
        sk.sk_pages_resize(pages, [0], (ctypes.c_int64 * 1)(33))
        sk.sk_pages_fork(pages, 0, (ctypes.c_int16 * 2)(1, 3))
        assert [sk.sk_pages_state(pages, s)[0] for s in range(4)] == [33, 33, 0, 33]
        assert sk.sk_pages_state(pages) == (57, 0)
        sk.sk_pages_resize(pages, [1, 3], sk.make_ids(n for n in (34, 0)))
        assert [sk.sk_pages_state(pages, s)[0] for s in range(4)] == [33, 34, 0, 0]
        assert sk.sk_pages_state(pages) == (56, 1)
    with sk.sk_pages_create(32767, 65536, 1, 32767) as pages:  # one page more would be 2^31 tokens, which are refused
        sk.sk_pages_resize(pages, [0], [2**31 - 65536])
        assert sk.sk_pages_state(pages) == (0, 0)
        assert sk.sk_pages_state(pages, 0)[1] == list(range(32767))
