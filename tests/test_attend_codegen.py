"""Guard of the generated code of the attention over the 4-bit cache (CPU only: hipcc cross-compiles gfx950 to assembly).

Its kernels use all the vector registers that their number of waves leaves them, part of them for scalar values that do not fit the scalar registers.
A few scalar values more in what they share with other kernels put vector registers into memory, silently: results stay right, and decoding
takes 4 % longer (two registers: 111.1 us became 115.6).
"""
import os
import re
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2507_21433_amd", "csrc")


def test_attention_over_the_4_bit_cache_keeps_its_registers(tmp_path):
    out = str(tmp_path / "rc_attend.s")
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    subprocess.run([hipcc, "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                    "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-S", "--cuda-device-only", "-o", out, os.path.join(CSRC, "rc_attend.hip")],
                   check=True, capture_output=True, text=True, timeout=600)
    # of every kernel: bytes of scratch memory of a thread, name, vector registers in it
    found = re.findall(r"\.private_segment_fixed_size: (\d+)\n(?:.*\n)*?\s+\.symbol:\s+(\S+)\n(?:.*\n)*?\s+\.vgpr_spill_count: (\d+)\n", open(out).read())
    names = [n for _, n, _ in found]
    assert sum("attend_rows_kernel" in n for n in names) == 8 and sum("attend_many_kernel" in n for n in names) == 4 and len(names) == 16, names
    assert all(int(scratch) == 0 and int(spilled) == 0 for scratch, _, spilled in found), found
