"""Code generation checks of the fp16 and int8 matrix kernels (no GPU needed): reads of a matrix
instruction's result across a block boundary come late enough, and nothing goes through scratch memory."""
import os
import re
import subprocess

import pytest

import test_codegen as tc

SOURCES = ("attention4.hip", "product8.hip")
# Wait states before a VALU touches the result: 16 x 16 shapes take 4 passes (8), 32 x 32 shapes 8 (12) on gfx950.
NEED = {"v_mfma_f32_16x16x32_f16": 8, "v_mfma_i32_16x16x64_i8": 8, "v_mfma_f32_32x32x16_f16": 12, "v_mfma_i32_32x32x32_i8": 12}


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


def test_matrix_instructions(asm):
    matrix = [k for k in asm if re.search(r"attention4_kernel|product8_(tiled|stream)_kernel", k)]
    assert matrix
    for k in matrix:
        used = {l.split()[0] for l in asm[k] if l.strip().startswith("v_mfma")}
        assert used and used <= set(NEED), (k, used)


def test_results_read_across_blocks_are_far(asm, monkeypatch):
    problems = {}
    touches = tc._touches

    def touches_but_sums(op, ops, pending):
        # a matrix instruction that adds to the same registers needs no wait states (and is looked at itself)
        return touches(op, ["", *ops[1:3]] if op.startswith("v_mfma") and ops[0] == ops[3] else ops, pending)
    monkeypatch.setattr(tc, "_touches", touches_but_sums)
    for k, lines in asm.items():
        used = {l.split()[0] for l in lines if l.strip().startswith("v_mfma")}
        if used:
            monkeypatch.setattr(tc, "required_wait_states", lambda ops, n=max(NEED[u] for u in used): n)
            bad = tc.mfma_escapes(lines)
            if bad:
                problems[k] = bad
    assert not problems, f"MFMA results read across a block boundary too soon: {problems}"


def test_no_scratch_memory(asm):
    for k, lines in asm.items():
        assert not any("scratch_" in l.split(";")[0] for l in lines), k
