"""Host side of libsk_layer.so at the ends of its ranges, no GPU."""
import os
import shutil
import subprocess

import pytest

import paper_1901_10008_amd as sk

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SAN = ["-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-static-libasan", "-g", "-O1"]
ENV = dict(os.environ, ASAN_OPTIONS="verify_asan_link_order=0:detect_leaks=1", UBSAN_OPTIONS="print_stacktrace=1")


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host C++ compiler")
def test_plans_at_the_ends_of_their_ranges(tmp_path):
    exe, csrc = str(tmp_path / "layer_edges_driver"), os.path.join(ROOT, "paper_1901_10008_amd", "csrc")
    res = subprocess.run(["g++", "-std=c++17", *SAN, "-I", os.path.join(ROOT, "include"), "-I", csrc, os.path.join(ROOT, "tests", "sanitize", "layer_edges_driver.cpp"),
                          os.path.join(csrc, "layer_plan.cpp"), "-o", exe], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    res = subprocess.run([exe], capture_output=True, text=True, env=ENV)
    assert res.returncode == 0 and "layer_edges_driver: ok" in res.stdout, res.stdout + res.stderr


VERIFY = dict(dtype="bf16", sequences=4, rows=12, vocab=1000, temperature=1.0, first_row=1 << 40, logits=1 << 41, logits_stride=1024, drafted=1 << 42, draft_logits=1 << 43, draft_stride=1000,
              temperatures=1 << 44, accept_random=1 << 45, sample_random=1 << 46, tokens=1 << 47, accepted=1 << 48)
BYTES = dict(first_row=20, logits=11 * 2048 + 2000, drafted=48, draft_logits=12 * 2000, temperatures=16, accept_random=48, sample_random=16)


def verify_plan(*problems):
    return sk.sk_verify_plan_create([sk.make_verify_problem(**p) for p in problems], sk.sk_layer_params_default(host_only=1))


@pytest.mark.parametrize("out,size", [("tokens", 48), ("accepted", 16)])
@pytest.mark.parametrize("name", sorted(BYTES))
def test_verified_tokens_must_not_touch_inputs(name, out, size):
    """A workgroup writes a sequence's tokens while others still read its drafts: tokens over drafted are refused, as is every byte of any input of the plan."""
    at, end = VERIFY[name], VERIFY[name] + BYTES[name]
    other = VERIFY | {k: v + (1 << 35) if k in BYTES or k in ("tokens", "accepted") else v for k, v in VERIFY.items()}
    for place in (at, at - size + 4, end - 4, at + 5 * 2048 + 1000 if name == "logits" else (at + end) // 8 * 4):
        with pytest.raises(sk.SkError) as e:
            verify_plan(VERIFY | {out: place})
        assert e.value.status == -3 and "touch an input" in e.value.detail
        with pytest.raises(sk.SkError):  # an input of another problem
            verify_plan(VERIFY, other | {out: place})
    for place in (at - size, end):
        verify_plan(VERIFY | {out: place}, other).close()
        verify_plan(other, VERIFY | {out: place}).close()


def test_what_stands_between_rows_of_logits_is_no_input():
    for out, size in (("tokens", 48), ("accepted", 16)):
        for row in (0, 5, 10):
            gap = VERIFY["logits"] + row * 2048 + 2000
            verify_plan(VERIFY | {out: gap}).close()
            verify_plan(VERIFY | {out: gap + 48 - size}).close()
            for place in (gap - 4, gap + 48 - size + 4):
                with pytest.raises(sk.SkError):
                    verify_plan(VERIFY | {out: place})
    # not read: what a plan without drafts is given of them
    verify_plan(VERIFY | dict(drafted=0, tokens=VERIFY["accept_random"], accepted=VERIFY["draft_logits"])).close()
