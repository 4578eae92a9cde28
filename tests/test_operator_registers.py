"""Registers that the operators' kernels rest on, as the compiler reports them (no GPU needed)."""
import os
import re
import subprocess

import pytest

from .test_build_registers import NVCC, ROOT


def used(tmp_path, header, decls):
    src = tmp_path / "op.cu"
    src.write_text(f'#include "{header}"\nnamespace ls {{\n' + "".join(f"template __global__ void {d};\n" for d in decls) + "}\n")
    r = subprocess.run([NVCC, "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "--expt-relaxed-constexpr", "-Xptxas=-v",
                        "-I", os.path.join(ROOT, "paper_2609_17184_b200", "csrc"), "-c", str(src), "-o", str(tmp_path / "op.o")],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    found = re.findall(r"Compiling entry function '(\S*)'.*?(\d+) bytes spill stores.*?Used (\d+) registers", r.stderr, re.S)
    assert len(found) == len(decls), r.stderr
    return [(name, int(spill), int(regs)) for name, spill, regs in found]


@pytest.mark.skipif(not os.path.exists(NVCC), reason="no nvcc")
def test_prefix_kernel_is_launched_with_what_its_warps_deal_out(tmp_path):
    """setmaxnreg draws on the registers of the launch: 168 for each of 384 threads are 216 for eight warps and 72 for four."""
    decls = [f"prefix_kernel<{t}, {d}>(const __grid_constant__ CUtensorMap, const __grid_constant__ CUtensorMap, const __grid_constant__ PrefixParams)"
             for t in ("__nv_bfloat16", "__half") for d in (64, 128)]
    assert all(regs == 168 for _, _, regs in used(tmp_path, "op_prefix.cuh", decls))


@pytest.mark.skipif(not os.path.exists(NVCC), reason="no nvcc")
def test_two_ctas_of_sample_kernel_share_an_sm(tmp_path):
    decls = [f"smp::sample_kernel<{t}>(const __grid_constant__ smp::Params)" for t in ("float", "__nv_bfloat16", "__half")]
    found = used(tmp_path, "op_sample.cuh", decls)
    assert all(regs <= 64 for _, _, regs in found), found


@pytest.mark.skipif(not os.path.exists(NVCC), reason="no nvcc")
def test_what_the_kernels_keep_in_local_memory_stays_small(tmp_path):
    """Registers are bounded by the launch (168 and 64 a thread), so what a kernel needs beyond them shows in its spills: bytes stored, 96 in the sampler and 128 in
    prefix_kernel at most, none in the others."""
    sample = [f"smp::sample_kernel<{t}>(const __grid_constant__ smp::Params)" for t in ("float", "__nv_bfloat16", "__half")]
    prefix = [f"prefix_kernel<{t}, {d}>(const __grid_constant__ CUtensorMap, const __grid_constant__ CUtensorMap, const __grid_constant__ PrefixParams)"
              for t in ("__nv_bfloat16", "__half") for d in (64, 128)]
    fold = [f"prefix_merge_kernel<__half, {d}, {w}>(const __grid_constant__ PrefixParams)" for d in (64, 128) for w in (1, 4)]
    append = [f"{k}<{t}, __nv_bfloat16, {lh}>(const __grid_constant__ AppendParams)" for k in ("append_kernel", "append_rows_kernel") for t in ("float", "__nv_bfloat16")
              for lh in (8, 16, 32)]
    for header, decls, most in (("op_sample.cuh", sample, 96), ("op_prefix.cuh", prefix, 128), ("op_prefix.cuh", fold, 0), ("op_append.cuh", append, 0)):
        found = used(tmp_path, header, decls)
        assert all(spill <= most for _, spill, _ in found), found
