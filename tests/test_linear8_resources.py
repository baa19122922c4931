"""What the compiler made of the kernels for projections in 8 bits, read from the built library's own metadata: none spills, and the tiles that
share a SIMD between two waves stay within half of its registers."""
import os
import shutil
import subprocess

import pytest
import yaml

from paper_2602_12957_amd.build import LIB_PATH, build_library

LLVM = "/opt/rocm/llvm/bin"


def test_kernels_of_the_projections_in_8_bits(tmp_path):
    tools = [os.path.join(LLVM, t) for t in ("llvm-objdump", "llvm-readelf")]
    if not all(os.path.exists(t) for t in tools):
        pytest.skip("no LLVM tools to read the library with")
    if not os.path.exists(LIB_PATH):
        build_library()
    shutil.copy(LIB_PATH, tmp_path / "lib.so")
    subprocess.run([tools[0], "--offloading", "lib.so"], cwd=tmp_path, check=True, capture_output=True)
    code = [f for f in os.listdir(tmp_path) if f.endswith("gfx950")]
    notes = subprocess.run([tools[1], "--notes", code[0]], cwd=tmp_path, check=True, capture_output=True, text=True).stdout
    kernels = yaml.safe_load(notes.split("---\n", 1)[1].split("\n...", 1)[0])["amdhsa.kernels"]
    for name in ("12k_quant_rowsI", "17k_quant_read_rowsI", "15k_quant_weightsI", "12k_gemm_quantI", "16k_gemm_quant_fewI"):
        forms = {k[".name"]: (k[".vgpr_spill_count"], k[".private_segment_fixed_size"], k[".vgpr_count"]) for k in kernels if name in k[".name"]}
        assert forms, name
        assert {n: f for n, f in forms.items() if f[0] or f[1]} == {}
        assert {n: f for n, f in forms.items() if f[2] > 256} == {}
