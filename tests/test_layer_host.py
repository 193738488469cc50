"""Host side of the operators of a decoder step beside products and attention, no GPU: what plans refuse, layouts, sanitizers, what the compiler made."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest

import paper_1901_10008_amd as sk

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SAN = ["-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-static-libasan", "-g", "-O1"]
ENV = dict(os.environ, ASAN_OPTIONS="verify_asan_link_order=0:detect_leaks=1", UBSAN_OPTIONS="print_stacktrace=1")

BASE = 1 << 40  # addresses that nothing touches: plans here are host-only
INVALID, UNSUPPORTED, OVERLAP, STATE = -1, -2, -3, -7
NAN, INF = float("nan"), float("inf")
HOST = dict(host_only=1)

NORM = dict(dtype="bf16", rows=8, dim=100, block=BASE, residual=BASE << 1, post=1, gate=BASE << 2, gate_rows=1, gate_act=sk.SK_ACT_SILU, eps=1e-5, residual_out=BASE << 3, next=BASE << 4)
MOE = dict(dtype="bf16", rows=8, dim=64, experts=8, top_k=2, ffn=32, shared_ffn=16, act=sk.SK_ACT_SILU, normalize=1, x=BASE, router=BASE, gate=BASE, up=BASE, down=BASE, shared_gate=BASE,
           shared_up=BASE, shared_down=BASE, out=BASE << 1, expert_ids=BASE << 2, expert_weights=BASE << 3)
VERIFY = dict(dtype="bf16", sequences=4, rows=12, vocab=1000, temperature=1.0, first_row=BASE, logits=BASE, drafted=BASE, draft_logits=BASE, accept_random=BASE, sample_random=BASE,
              tokens=BASE << 1, accepted=BASE << 2)


def plan(kind, *problems, **params):
    make, create = getattr(sk, f"make_{kind}_problem"), getattr(sk, f"sk_{kind}_plan_create")
    return create([make(**p) for p in problems], sk.sk_layer_params_default(**(HOST | params)))


@pytest.mark.parametrize("kind,good", [("norm", NORM), ("moe", MOE), ("verify", VERIFY)])
def test_good_problems_are_planned(kind, good):
    with plan(kind, good) as p:
        with pytest.raises(sk.SkError) as e:
            getattr(sk, f"sk_{kind}_launch")(p)
        assert e.value.status == STATE and "host-only" in e.value.detail
        if kind != "norm":
            launches, workspace = getattr(sk, f"sk_{kind}_plan_info")(p)
            assert launches > 0 and workspace > 0
    with plan(kind) as p:
        if kind != "norm":
            assert getattr(sk, f"sk_{kind}_plan_info")(p) == (0, 0)


@pytest.mark.parametrize("kind,good,fields", [
    ("norm", NORM, dict(block=0, gate=0)), ("norm", NORM, dict(residual=0)), ("norm", NORM, dict(next=0)), ("norm", NORM, dict(residual_out=0)), ("norm", NORM, dict(residual_out=BASE << 1)),
    ("norm", NORM, dict(next=BASE)), ("norm", NORM, dict(residual_dtype="f32", dim=32768)), ("norm", NORM, dict(gate_rows=0, dtype="f32", residual_dtype="f32")), ("norm", NORM, dict(dim=1, rows=1 << 24)),
    ("norm", NORM, dict(block=BASE + 2, next_stride=101)), ("norm", NORM, dict(n_rows=BASE + 4)), ("norm", NORM, dict(eps=0.0)),
    ("moe", MOE, dict(gate=0, shared_gate=0)), ("moe", MOE, dict(shared_ffn=0, shared_gate=0, shared_up=0, shared_down=0)), ("moe", MOE, dict(router_dtype="f32")), ("moe", MOE, dict(rows=100000)),
    ("moe", MOE, dict(experts=512, top_k=32)), ("moe", MOE, dict(expert_ids=0, expert_weights=0)), ("moe", MOE, dict(x_stride=72, up_row_stride=72, up_expert_stride=72 * 40, down_row_stride=40)),
    ("moe", MOE, dict(router_bias=BASE + 4)), ("moe", MOE, dict(dtype="f16", router_dtype="f16")),
    ("verify", VERIFY, dict(drafted=0, accept_random=0, draft_logits=0)), ("verify", VERIFY, dict(dtype="f32", vocab=1 << 20)), ("verify", VERIFY, dict(logits=BASE + 2, logits_stride=1001)),
    ("verify", VERIFY, dict(temperature=0.0, draft_logits=0)), ("verify", VERIFY, dict(temperature=NAN)), ("verify", VERIFY, dict(sequences=100, rows=1)),
])
def test_other_good_problems(kind, good, fields):
    plan(kind, good | fields).close()


@pytest.mark.parametrize("kind,good,fields,status", [("norm", NORM, f, s) for f, s in [
    (dict(dtype=3), UNSUPPORTED), (dict(residual_dtype="f16"), UNSUPPORTED), (dict(dtype="f32", residual_dtype="bf16"), UNSUPPORTED), (dict(rows=0), INVALID), (dict(dim=0), INVALID),
    (dict(dim=-5), INVALID), (dict(dim=32769), UNSUPPORTED), (dict(kind=2), INVALID), (dict(kind=-1), INVALID), (dict(post=2), INVALID), (dict(gate_rows=2), INVALID), (dict(reserved=1), INVALID),
    (dict(gate_act=6), INVALID), (dict(gate_act=-1), INVALID), (dict(eps=-1e-9), INVALID), (dict(eps=NAN), INVALID), (dict(eps=INF), INVALID), (dict(residual_scale=INF), INVALID),
    (dict(block_scale=NAN), INVALID), (dict(block=0, residual=0), INVALID), (dict(next=0, residual_out=0), INVALID), (dict(block_stride=99), INVALID), (dict(gate_stride=99), INVALID),
    (dict(residual_stride=-100), INVALID), (dict(next_stride=99), INVALID), (dict(residual_out_stride=1), INVALID), (dict(block=BASE + 1), UNSUPPORTED), (dict(gate=BASE + 1), UNSUPPORTED),
    (dict(pre_weight=BASE + 1), UNSUPPORTED), (dict(residual_dtype="f32", residual=BASE + 2), UNSUPPORTED), (dict(n_rows=BASE + 2), UNSUPPORTED), (dict(rows=1 << 26, dim=4096), UNSUPPORTED),
    (dict(next_stride=1 << 62), UNSUPPORTED), (dict(block_stride=1 << 62), UNSUPPORTED), (dict(next=(BASE << 3) + 200), OVERLAP), (dict(rows=1 << 23, dim=9000), UNSUPPORTED),
]] + [("moe", MOE, f, s) for f, s in [
    (dict(dtype="f32", router_dtype="f32"), UNSUPPORTED), (dict(dtype=9), UNSUPPORTED), (dict(router_dtype="f16"), UNSUPPORTED), (dict(rows=0), INVALID), (dict(dim=0), INVALID), (dict(experts=0), INVALID),
    (dict(top_k=0), INVALID), (dict(ffn=0), INVALID), (dict(shared_ffn=-8), INVALID), (dict(top_k=9), INVALID), (dict(experts=513), UNSUPPORTED), (dict(experts=64, top_k=33), UNSUPPORTED),
    (dict(dim=60), UNSUPPORTED), (dict(ffn=20), UNSUPPORTED), (dict(shared_ffn=12), UNSUPPORTED), (dict(act=6), INVALID), (dict(scoring=2), INVALID), (dict(normalize=2), INVALID), (dict(scale=INF), INVALID),
    (dict(x=0), INVALID), (dict(router=0), INVALID), (dict(up=0), INVALID), (dict(down=0), INVALID), (dict(out=0), INVALID), (dict(shared_up=0), INVALID), (dict(shared_down=0), INVALID),
    (dict(shared_gate=0), INVALID), (dict(gate=0), INVALID), (dict(x_stride=56), INVALID), (dict(out_stride=-64), INVALID), (dict(router_stride=32), INVALID), (dict(up_row_stride=60), INVALID),
    (dict(down_row_stride=24), INVALID), (dict(up_expert_stride=64 * 31), INVALID), (dict(down_expert_stride=32 * 62), INVALID), (dict(x_stride=68), UNSUPPORTED), (dict(out_stride=68), UNSUPPORTED),
    (dict(router_stride=66), UNSUPPORTED), (dict(up_row_stride=66), UNSUPPORTED), (dict(down_expert_stride=64 * 32 + 4), UNSUPPORTED), (dict(x=BASE + 8), UNSUPPORTED), (dict(router=BASE + 2), UNSUPPORTED),
    (dict(gate=BASE + 4), UNSUPPORTED), (dict(shared_down=BASE + 8), UNSUPPORTED), (dict(out=(BASE << 1) + 2), UNSUPPORTED), (dict(expert_ids=BASE + 2), UNSUPPORTED), (dict(n_rows=BASE + 1), UNSUPPORTED),
    (dict(expert_ids=BASE << 1), OVERLAP), (dict(expert_weights=(BASE << 2) + 32), OVERLAP), (dict(x_stride=1 << 41), UNSUPPORTED), (dict(up_expert_stride=1 << 51), UNSUPPORTED),
    (dict(dim=1 << 21), UNSUPPORTED), (dict(ffn=(1 << 24) + 8), UNSUPPORTED), (dict(x_stride=1 << 21), UNSUPPORTED), (dict(up_row_stride=1 << 26), UNSUPPORTED), (dict(down_row_stride=1 << 26), UNSUPPORTED), (dict(rows=2**31 - 1, experts=512, top_k=32), UNSUPPORTED),
]] + [("verify", VERIFY, f, s) for f, s in [
    (dict(dtype=-1), UNSUPPORTED), (dict(sequences=0), INVALID), (dict(rows=0), INVALID), (dict(vocab=0), INVALID), (dict(sequences=(1 << 20) + 1), UNSUPPORTED), (dict(vocab=(1 << 30) + 1), UNSUPPORTED),
    (dict(reserved=1), INVALID), (dict(first_row=0), INVALID), (dict(logits=0), INVALID), (dict(sample_random=0), INVALID), (dict(tokens=0), INVALID), (dict(accepted=0), INVALID),
    (dict(accept_random=0), INVALID), (dict(logits_stride=999), INVALID), (dict(draft_stride=-1), INVALID), (dict(logits=BASE + 1), UNSUPPORTED), (dict(draft_logits=BASE + 1), UNSUPPORTED),
    (dict(tokens=(BASE << 1) + 2), UNSUPPORTED), (dict(temperatures=BASE + 1), UNSUPPORTED), (dict(logits_stride=1 << 62), UNSUPPORTED), (dict(draft_stride=1 << 62), UNSUPPORTED),
    (dict(accepted=(BASE << 1) + 44), OVERLAP), (dict(rows=1 << 30, vocab=1 << 30), UNSUPPORTED),
]])
def test_refusals(kind, good, fields, status):
    for problems in ([good | fields], [good | {k: v << 5 if k in OUT else v for k, v in good.items()}, good | fields]):  # alone, and behind a good one elsewhere
        with pytest.raises(sk.SkError) as e:
            plan(kind, *problems)
        assert e.value.status == status, e.value
        assert status == OVERLAP or e.value.detail.startswith(f"problem {len(problems) - 1}: ")


OUT = ("out", "expert_ids", "expert_weights", "residual_out", "next", "tokens", "accepted")


@pytest.mark.parametrize("kind,good", [("norm", NORM), ("moe", MOE), ("verify", VERIFY)])
def test_outputs_of_two_problems(kind, good):
    with pytest.raises(sk.SkError) as e:
        plan(kind, good, good)
    assert e.value.status == OVERLAP
    plan(kind, good, good | {k: v << 5 for k, v in good.items() if k in OUT}).close()


@pytest.mark.parametrize("kind", ["norm", "moe", "verify"])
def test_bad_calls(kind):
    L = sk.layer_lib()
    create, destroy, launch = (getattr(L, f"sk_{kind}_{n}") for n in ("plan_create", "plan_destroy", "launch"))
    out = ctypes.c_void_p(77)
    assert create(None, 1, None, ctypes.byref(out)) in (INVALID, -5) and out.value == 77  # (-5: no device here)
    host = sk.sk_layer_params_default(host_only=1)
    assert create(None, 1, ctypes.byref(host), ctypes.byref(out)) == INVALID and out.value == 77
    assert create(None, -1, ctypes.byref(host), ctypes.byref(out)) == INVALID
    assert create(None, 0, ctypes.byref(host), None) == INVALID
    for bad in (dict(host_only=2), dict(workgroups=-1), dict(workgroups=65537)):
        prm = sk.sk_layer_params_default(**bad)
        assert create(None, 0, ctypes.byref(prm), ctypes.byref(out)) == INVALID
    prm = sk.sk_layer_params_default(host_only=1)
    prm.reserved[1] = 1
    assert create(None, 0, ctypes.byref(prm), ctypes.byref(out)) == INVALID
    assert destroy(None) == 0 and launch(None, None) == INVALID
    if kind != "norm":
        assert getattr(L, f"sk_{kind}_plan_info")(None, None, None) == INVALID
    with pytest.raises(AttributeError):
        getattr(sk, f"make_{kind}_problem")(nonsense=1)


def test_structures_are_as_the_compiler_lays_them_out(tmp_path):
    source = '#include <stdio.h>\n#include <stddef.h>\n#include "sk_layer.h"\nint main(void) {\n'
    kinds = dict(sk_norm_problem=sk.sk_norm_problem, sk_moe_problem=sk.sk_moe_problem, sk_verify_problem=sk.sk_verify_problem, sk_layer_params=sk.LayerParams)
    for name, kind in kinds.items():
        source += f'printf("%zu\\n", sizeof({name}));\n' + "".join(f'printf("%zu\\n", offsetof({name}, {f[0]}));\n' for f in kind._fields_)
    (tmp_path / "s.c").write_text(source + "return 0; }\n")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(tmp_path / "s.c"), "-o", str(tmp_path / "s")], check=True)
    got = [int(x) for x in subprocess.run([str(tmp_path / "s")], capture_output=True, text=True, check=True).stdout.split()]
    want = []
    for kind in kinds.values():
        want += [ctypes.sizeof(kind)] + [getattr(kind, f[0]).offset for f in kind._fields_]
    assert got == want


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host C++ compiler")
def test_host_code_under_sanitizers(tmp_path):
    exe, csrc = str(tmp_path / "layer_driver"), os.path.join(ROOT, "paper_1901_10008_amd", "csrc")
    res = subprocess.run(["g++", "-std=c++17", *SAN, "-I", os.path.join(ROOT, "include"), "-I", csrc, os.path.join(ROOT, "tests", "sanitize", "layer_driver.cpp"),
                          os.path.join(csrc, "layer_plan.cpp"), "-o", exe], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    res = subprocess.run([exe], capture_output=True, text=True, env=ENV)
    assert res.returncode == 0 and "layer_driver: ok" in res.stdout, res.stdout + res.stderr


def _all(blob, key):
    found = []
    for m in re.finditer(re.escape(key), blob):
        at = m.end()  # a MessagePack unsigned integer
        n = {0xCC: 1, 0xCD: 2, 0xCE: 4}.get(blob[at], 0)
        found.append(int.from_bytes(blob[at + 1:at + 1 + n], "big") if n else blob[at])
    return found


def test_no_kernel_spills_or_has_a_stack():
    with open(sk.layer_lib_path(), "rb") as f:
        blob = f.read()
    n = len(_all(blob, b".vgpr_count"))
    assert n >= 8
    assert _all(blob, b".vgpr_spill_count") == [0] * n and _all(blob, b".private_segment_fixed_size") == [0] * n
