"""The first launch of a decode step waits for everything before it in the stream (its attention does not, for pages of earlier
tokens): checked in the sources, because which kernels overlap cannot be commanded."""
import os
import re

from paper_2502_20727_b200 import build as spd_build


def source(name):
    return re.sub(r"//[^\n]*", "", open(os.path.join(spd_build.CSRC, name)).read())


def body(text, start):
    at = text.index(start)
    at, depth = text.index("{", at), 0
    for end in range(at, len(text)):
        depth += {"{": 1, "}": -1}.get(text[end], 0)
        if not depth:
            return text[at:end]


def test_the_step_prologue_overlaps_with_nothing_before_it():
    assert "launch_kernel_after(false, decode_prologue_kernel" in body(source("gemm_decode.cu"), "cudaError_t launch_decode_prologue(")
    for step in ("run_decode_fused", "run_tp"):  # ... and is what these begin with
        calls = re.findall(r"\blaunch_\w+\(", body(source("spd_api.cu"), f"int {step}(Ctx *c, const void *x, void *out"))
        assert calls[0] == "launch_decode_prologue(", step


def test_unfused_steps_begin_with_a_launch_that_waits():
    text = source("spd_api.cu")
    for step in ("int run_tokens(Ctx *c", "int run_tp_baseline(Ctx *c"):
        code = body(text, step)
        first_table = re.search(r"if \(rope_on\) LAUNCH\(K_ROPE_TABLE, launch_rope_table\(([^;]*)\)\);", code).group(1)
        first_norm = [m for m in re.findall(r"LAUNCH\(K_NORM, launch_residual_norm<\w+>\(([^;]*)\)\);", code)][0]
        assert first_table.endswith("!decode"), step
        assert first_norm.endswith("!decode || rope_on"), step
    for name in ("launch_rope_table(", "launch_residual_norm("):
        assert "launch_kernel_after(overlap," in body(source("elementwise.cu"), "cudaError_t " + name)
