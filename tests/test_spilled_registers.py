"""What the compiler says of the built kernels' registers: the paged kernels keep theirs out of memory, and those on a cache of bf16 do not
pay, in scalar registers, for the launches for some of the sequences that only a cache in 4 bits has."""
import os
import re
import subprocess

import pytest

from paper_2409_15104_amd import binding

LLVM = "/opt/rocm/llvm/bin"


def kernels(notes):
    """{mangled name: (spilled vector registers, spilled scalar registers)}"""
    found = {}
    for entry in re.split(r"\n\s*- \.a", notes):
        get = lambda key: re.search(r"\.%s:\s+(\S+)" % key, entry)  # noqa: E731
        if get("symbol") and get("vgpr_spill_count"):
            found[get("symbol")[1].strip("'").removesuffix(".kd")] = int(get("vgpr_spill_count")[1]), int(get("sgpr_spill_count")[1])
    return found


@pytest.fixture(scope="module")
def built(tmp_path_factory):
    if not os.path.exists(binding.LIB_PATH):
        from paper_2409_15104_amd import build

        build.build()
    if not os.path.exists(os.path.join(LLVM, "llvm-readelf")):
        pytest.skip("no reader of notes")
    d = tmp_path_factory.mktemp("notes")
    fat, dev = str(d / "fat.bin"), str(d / "dev.o")
    run = lambda *a: subprocess.run(a, check=True, capture_output=True, text=True).stdout  # noqa: E731
    run(LLVM + "/llvm-objcopy", "--dump-section", ".hip_fatbin=" + fat, binding.LIB_PATH, os.devnull)
    run(LLVM + "/clang-offload-bundler", "--unbundle", "--type=o", "--input=" + fat, "--output=" + dev,
        "--targets=hipv4-amdgcn-amd-amdhsa--gfx950")
    return kernels(run(LLVM + "/llvm-readelf", "--notes", dev))


def test_no_paged_kernel_spills_to_memory(built):
    paged = {n: s for n, s in built.items() if "paged_" in n or "norm_rope" in n}
    assert sum("paged_mx_step_kernel" in n for n in paged) == 12 and sum("17paged_step_kernel" in n for n in paged) == 4
    assert not {n: s for n, s in paged.items() if s[0]}


@pytest.mark.parametrize("name,most", [("17paged_step_kernelILi1ELi8ELi1ELb0E", 73), ("17paged_step_kernelILi2ELi4ELi2ELb0E", 38),
                                       ("17paged_step_kernelILi1ELi8ELi1ELb1E", 29), ("17paged_step_kernelILi1ELi4ELi1ELb1E", 20),
                                       ("19paged_simple_kernel", 35)])
def test_scalar_registers_of_the_kernels_on_bf16(built, name, most):
    """As many as they spilled before there was a cache in 4 bits."""
    assert [s[1] <= most for n, s in built.items() if name in n] == [True]
