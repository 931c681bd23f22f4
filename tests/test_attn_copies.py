"""The copies to LDS of the attention kernels, in the code that was built from them (no GPU): the compiler does not look after waits inside
inline assembly, so a copy that follows a vector instruction's write of its scalar base has to bring its own."""
import os
import re
import subprocess

import pytest

import paper_2406_09041_amd.build as build

LLVM = "/opt/rocm/llvm/bin"


def _listing(source, tmp_path):
    obj = os.path.join(build.HERE, "_build", source + ".o")
    if not (os.path.exists(obj) and os.path.exists(os.path.join(LLVM, "llvm-objdump"))):
        pytest.skip("needs the objects of a build and the toolchain's llvm-objdump")
    bundle, code = str(tmp_path / "bundle"), str(tmp_path / "code")
    subprocess.check_call([os.path.join(LLVM, "llvm-objcopy"), f"--dump-section=.hip_fatbin={bundle}", obj, str(tmp_path / "rest")])
    subprocess.check_call([os.path.join(LLVM, "clang-offload-bundler"), "--unbundle", "--type=o", "--targets=hipv4-amdgcn-amd-amdhsa--gfx950",
                           f"--input={bundle}", f"--output={code}"])
    text = subprocess.run([os.path.join(LLVM, "llvm-objdump"), "-d", "--no-show-raw-insn", code], check=True, capture_output=True, text=True).stdout
    return [line.split("//")[0].strip() for line in text.splitlines() if line.startswith("\t")]


@pytest.mark.parametrize("source", ["mes_attn_prompt", "mes_attn_decode"])
def test_a_copy_reads_its_base_from_a_scalar_copy(source, tmp_path):
    lines, scalar = _listing(source, tmp_path), 0
    for before, line in zip(lines, lines[1:]):
        copy = re.match(r"global_load_lds_dwordx4 v\d+, (s\[\d+:\d+\])", line)
        if copy:
            scalar += 1
            assert before.startswith(f"s_mov_b64 {copy[1]}, "), f"{before}; {line}"
    assert scalar > 0
