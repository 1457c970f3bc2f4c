"""What the compiler made of the kernels of the token statistics and the 8-bit operators."""
import re

import pytest

from test_compiled_kernels import _functions, _steady_loop, asm  # noqa: F401 (asm is a fixture)


@pytest.mark.parametrize("src", ["gemm_stats.hip", "gemm_i8.hip", "stats_rows.hip", "quantize.hip"])
def test_no_kernel_spills_vector_registers(asm, src):  # noqa: F811
    spills = dict(re.findall(r"\.name: +(_Z\w+)\n.*?\.vgpr_spill_count: (\d+)\n", asm(src), flags=re.S))
    assert spills and {k: n for k, n in spills.items() if n != "0"} == {}


@pytest.mark.parametrize("src,mfma", [("gemm_stats.hip", "v_mfma_f32_16x16x32_bf16"), ("gemm_i8.hip", "v_mfma_i32_16x16x64_i8")])
def test_few_tokens_are_multiplied_as_their_loads_arrive(asm, src, mfma):  # noqa: F811
    """The kernel for few tokens multiplies what has arrived while the rest is under way: in the loop over the units no wait asks for
    all loads of W (where a wavefront has more than one line of a row)."""
    found = {name: lines for name, lines in _functions(asm(src)).items()
             if "few_tokens_kernel" in name and "FewStats" in name and "Li8ELi1E" not in name}
    assert found
    for name, lines in found.items():
        ops = [line for line in lines if mfma in line]
        first, last = (next(i for i in order if mfma in lines[i]) for order in (range(len(lines)), range(len(lines) - 1, -1, -1)))
        waits = [int(n) for line in lines[first:last] for n in re.findall(r"vmcnt\((\d+)\)", line)]
        assert ops and waits and min(waits) > 0, name


@pytest.mark.parametrize("src,epilogue", [("gemm_stats.hip", "EpiStatsILb0ELb1E"), ("gemm_stats.hip", "EpiStatsILb0ELb0E"),
                                          ("gemm_i8.hip", "EpiStatsILb1ELb1E"), ("gemm_i8.hip", "EpiStatsILb1ELb0E")])
def test_steady_loop_of_the_vocabulary_gemm(asm, src, epilogue):  # noqa: F811
    """64 products and eight loads a slice, whose addresses are formed next to them."""
    found = [lines for name, lines in _functions(asm(src)).items() if "gemm_nt_kernel" in name and "Li256ELi256" in name and epilogue in name]
    assert len(found) == 1
    ops = [line.split()[0] for line in _steady_loop(found[0]) if re.match(r"\s+[sv]_|\s+ds_|\s+global_", line)]
    assert sum("v_mfma" in op for op in ops) == 64 and ops.count("global_load_lds_dwordx4") == 8
    first = next(i for i, op in enumerate(ops) if "v_mfma" in op)
    assert sum(op == "v_lshl_add_u64" for op in ops[:first]) == 0
