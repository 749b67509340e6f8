"""Code generation checks of the kernels in 8-bit floating point (no GPU needed): the matrix instructions they use, and reads of
their results across a block boundary come late enough."""
import os
import re
import subprocess

import pytest

import test_codegen as tc

SOURCES = ("attention8.hip", "product_fp8.hip")
# Wait states before a VALU touches the result: 16 x 16 x 32 fp16 takes 4 passes (8); fp8 operands of the 128-long one 12.
NEED = {"v_mfma_f32_16x16x32_f16": 8, "v_mfma_f32_16x16x128_f8f6f4": 12}


@pytest.fixture(scope="module")
def asm():
    from paper_2606_15652_amd import build
    out = {}
    for src in build.sources():
        if os.path.basename(src) not in SOURCES:
            continue
        cmd = [os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *[f for f in build.compile_flags(src) if f != "-fPIC"],
               "--cuda-device-only", "-S", src, "-o", "-"]
        cur = None
        for line in subprocess.run(cmd, capture_output=True, text=True, check=True).stdout.splitlines():
            m = re.match(r"^(_Z\S+):\s", line + " ")
            if m:
                cur = m.group(1)
                out[cur] = []
            elif cur is not None and line.strip().startswith(".Lfunc_end"):
                cur = None
            elif cur is not None:
                out[cur].append(line)
    return out


def matrix(lines):
    return {l.split()[0] for l in lines if l.strip().startswith("v_mfma")}


def test_matrix_instructions(asm):
    kernels = [k for k in asm if re.search(r"attention8_(wide_)?kernel|product_f8_(tiled|stream)_kernel", k)]
    assert len(kernels) >= 30
    for k in kernels:
        assert matrix(asm[k]) == ({"v_mfma_f32_16x16x32_f16"} if "attention" in k else {"v_mfma_f32_16x16x128_f8f6f4"}), k


def test_results_read_across_blocks_are_far(asm, monkeypatch):
    problems = {}
    touches = tc._touches

    def touches_but_sums(op, ops, pending):
        # a matrix instruction that adds to the same registers needs no wait states (and is looked at itself)
        return touches(op, ["", *ops[1:3]] if op.startswith("v_mfma") and ops[0] == ops[3] else ops, pending)
    monkeypatch.setattr(tc, "_touches", touches_but_sums)
    for k, lines in asm.items():
        used = matrix(lines)
        if used:
            monkeypatch.setattr(tc, "required_wait_states", lambda ops, n=max(NEED[u] for u in used): n)
            bad = tc.mfma_escapes(lines)
            if bad:
                problems[k] = bad
    assert not problems, f"MFMA results read across a block boundary too soon: {problems}"


def test_products_use_no_scratch_memory(asm):
    for k, lines in asm.items():
        if "product_f8" in k or "ELi64E" in k:
            assert not any("scratch_" in l.split(";")[0] for l in lines), k
