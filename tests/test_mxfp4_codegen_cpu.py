"""What the compiler made of the kernels of the MXFP4 calls and of expert order, read from the objects that the build leaves
(their own gfx950 code): no vector register is spilled to memory, and scalar registers that are spilled are fetched back, lane
by lane, outside the persistent products' K-loops only."""
import os
import re
import subprocess

import pytest

import paper_2412_19437_amd as pkg

BUILD = os.path.join(os.path.dirname(pkg.__file__), "_build")
LLVM = "/opt/rocm/llvm/bin"
OBJECTS = ["ds3_gemm_mxfp4", "ds3_moe", "ds3_mxfp4"]

pytestmark = pytest.mark.skipif(not all(os.path.exists(f"{BUILD}/{o}.o") for o in OBJECTS) or not os.path.exists(f"{LLVM}/llvm-objdump"),
                                reason="no objects or no disassembler")


def run(*a):
    return subprocess.run([f"{LLVM}/{a[0]}", *map(str, a[1:])], check=True, capture_output=True, text=True).stdout


def device_code(tmp_path, name):
    fat, dev = tmp_path / "fat", tmp_path / "dev.o"
    run("llvm-objcopy", "--dump-section", f".hip_fatbin={fat}", f"{BUILD}/{name}.o", tmp_path / "copy.o")
    run("clang-offload-bundler", "--type=o", "--unbundle", f"--input={fat}", "--targets=hipv4-amdgcn-amd-amdhsa--gfx950", f"--output={dev}")
    return dev


@pytest.mark.parametrize("name", OBJECTS)
def test_no_vector_register_is_spilled(tmp_path, name):
    notes = run("llvm-readelf", "--notes", device_code(tmp_path, name))
    for field in ("private_segment_fixed_size", "vgpr_spill_count"):
        counts = re.findall(rf"\.{field}: +(\d+)", notes)
        assert counts and set(counts) == {"0"}, field


def test_the_products_k_loops_fetch_no_scalars_from_lanes(tmp_path):
    """A K-loop: from a backward branch's target to the branch, with some of the kernel's matrix instructions (the loop over the
    tiles has them all)."""
    bodies = re.split(r"\n([0-9a-f]+) <(\S+)>:\n", run("llvm-objdump", "-d", "--no-show-raw-insn", device_code(tmp_path, "ds3_gemm_mxfp4")))
    kernels = [(int(start, 16), name, body.splitlines()) for start, name, body in zip(bodies[1::3], bodies[2::3], bodies[3::3]) if "gemm_mxfp4_kernel" in name]
    assert len(kernels) == 10
    for start, name, lines in kernels:
        at = {int(m.group(1), 16): i for i, line in enumerate(lines) if (m := re.search(r"// ([0-9A-F]{12})", line))}
        count = lambda text, a, b: sum(text in line for line in lines[a:b])  # noqa: E731
        loops = 0
        for i, line in enumerate(lines):
            m = re.search(r"s_c?branch\w*\s.*<\S+\+0x([0-9a-f]+)>", line)
            first = at[start + int(m.group(1), 16)] if m else i
            if first < i and 0 < count("v_mfma", first, i) < count("v_mfma", 0, len(lines)):
                loops += 1
                assert count("v_readlane", first, i) == 0, name
        assert loops, name
