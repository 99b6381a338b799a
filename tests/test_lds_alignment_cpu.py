"""Alignment of the workgroup memory that launches size (``extern __shared__``): the linker puts such an array behind a kernel's
own, at the next multiple of the alignment that its declaration has, so an array that is read 16 bytes at once has to be
declared so. Taken from the compiler's own declarations of device code; no test here touches a GPU."""
import os
import re
import subprocess

import pytest

from paper_2607_19438_amd import build

USE = {
    "group_lds": ("attn_shared.hpp", "qg::kv4_shared_kernel<128, 2, 1>", 16),
    "old_lds": ("beam_kernels.hpp", "qg::kv_reorder_kernel<false>", 4),
}


@pytest.mark.parametrize("name", USE)
def test_alignment(name, tmp_path):
    header, kernel, need = USE[name]
    src, out = tmp_path / "use.hip", tmp_path / "use.ll"
    src.write_text(f'#include "{header}"\nconst void* use() {{ return (const void*)({kernel}); }}\n')
    subprocess.run([build.HIPCC, f"--offload-arch={build.ARCH}", "-std=c++20", "-O0", "-w", "-I", build.CSRC, "--cuda-device-only", "-S", "-emit-llvm",
                    str(src), "-o", str(out)], check=True, cwd=tmp_path, capture_output=True)
    found = re.findall(rf"^@\S*{name}\S* = external .*addrspace\(3\).*, align (\d+)", out.read_text(), re.M)
    assert found and all(int(a) >= need for a in found), (name, found)
