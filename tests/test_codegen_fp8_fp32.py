"""Code generation of the product's kernels for fp32 results (no GPU needed): the matrix instruction whose sums are fp32's, and no scratch."""
from test_codegen_fp8 import asm, matrix  # noqa: F401


def test_fp32_results_use_fp16_operands(asm):  # noqa: F811
    kernels = [k for k in asm if "product_fp32_" in k]
    assert len(kernels) == 5 + 7
    for k in kernels:
        assert matrix(asm[k]) == {"v_mfma_f32_16x16x32_f16"}, k
        assert not any("scratch_" in l.split(";")[0] for l in asm[k]), k
    # and no kernel of the 8-bit instruction stores them
    assert not [k for k in asm if "product_f8_tiled_kernelIf" in k or "product_f8_stream_kernelIf" in k]
