"""What the compiler says of the attention kernels that are built: those whose loops fit the registers have no scratch memory (a spilled register costs a trip to memory in the loop)."""
import os
import re
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1912_12607_amd", "csrc")
LLVM = "/opt/rocm/llvm/bin"


def scratch(name, tmp_path):
    """Bytes of scratch a lane of each kernel of an object file."""
    obj, code = os.path.join(CSRC, name + ".o"), str(tmp_path / "code.co")
    tools = [os.path.join(LLVM, t) for t in ("clang-offload-bundler", "llvm-readelf", "llvm-objcopy")]
    if not all(os.path.exists(f) for f in [obj] + tools):
        pytest.skip("no object file, or no tools to look at it")
    bundle = str(tmp_path / "bundle")
    subprocess.run([tools[2], "--dump-section", f".hip_fatbin={bundle}", obj, os.devnull], check=True)
    subprocess.run([tools[0], "--unbundle", "--type=o", "--targets=hipv4-amdgcn-amd-amdhsa--gfx950", f"--input={bundle}", f"--output={code}"], check=True)
    notes = subprocess.run([tools[1], "--notes", code], check=True, capture_output=True, text=True).stdout
    found = {}
    for kernel in notes.split(".args:")[1:]:
        symbol, size = re.search(r"\.name:\s+(\S+)", kernel.split(".group_segment_fixed_size")[-1]), re.search(r"\.private_segment_fixed_size:\s+(\d+)", kernel)
        found[symbol.group(1)] = int(size.group(1))
    return found


def arguments(symbol):
    return [int(n) for n in re.findall(r"L[ib](\d+)E", symbol)]


def test_larger_blocks_of_16_bit_tensors_spill_nothing(tmp_path):
    kernels = {s: n for s, n in scratch("token_attend_chunk", tmp_path).items() if "attend_chunk_kernel" in s}
    # (type: 0 fp32, whose dims above 128 do not fit; dims; waves; pages; 4 bits)
    assert len(kernels) >= 28
    assert not {s: n for s, n in kernels.items() if n and not (arguments(s)[0] == 0 and arguments(s)[1] == 256)}
