"""Labels of kernels in profiler summaries, from demangled and mangled names."""
import pytest

CASES = [
    ("moe::(anonymous namespace)::vocab_dx_kernel<256>(int, float const*)", "vocab_dx_kernel"),
    ("_ZN3moe4mfma18dense_fixup_kernelILi256ELi256EDF16bEEvPKfPKiiiiiiNS_7CutCostEiPT1_l", "dense_fixup_kernel"),
    ("_ZN3moe12_GLOBAL__N_122vocab_grad_rows_kernelILi256EEEvPKDv2_fiiPKfiliPcNS0_6RowOutE", "vocab_grad_rows_kernel"),
    ("void moe::(anonymous namespace)::adamw_kernel<float>(moe::AdamwEntry const*)", "adamw_kernel"),
    ("_ZN3moe4mfma23grouped_gemm_dma_kernelILi256ELi256ELi64ELi2ELi2ELi4ELNS0_6LayoutE1ELS2_1ELNS0_4ModeE3ELNS0_3EpiE0EDF16bDF16bEEvNS0_4ArgsE",
     "grouped_gemm<256x256x64 s2 w2x4 TN dense store out=bf16 in=bf16>"),
    ("__amd_rocclr_copyBuffer", "__amd_rocclr_copyBuffer"),
    ("_ZN2at6native29vectorized_elementwise_kernelILi4EEEvi", "vectorized_elementwise_kernel"),
]


@pytest.mark.parametrize("name,want", CASES)
def test_label(name, want):
    from paper_2505_11432_amd.profile_summary import label
    assert label(name) == want
