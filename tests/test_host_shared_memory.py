"""CPU checks of the kernels' shared memory: what is read or written four
numbers at a time is declared on 16 bytes (the hardware's wide accesses need
that, and only a declaration promises it)."""
import ctypes as C
import glob
import os
import re
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2011_11188_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
WIDE = r"\((?:const )?(?:float4|float4_t|uint4)\*\)\s*&?(\w+)\["


def test_arrays_of_wide_accesses_are_declared_on_16_bytes():
    seen = 0
    for path in sorted(glob.glob(os.path.join(CSRC, "*.hip")) + glob.glob(os.path.join(CSRC, "*.h"))):
        text = open(path).read()
        for use in re.finditer(WIDE, text):
            # the array's declaration is the last one of its name before the use
            lines = re.findall(rf"^.*__shared__ .*\b{use.group(1)}\[.*$", text[:use.start()], re.M)
            if not lines:
                continue
            seen += 1
            wide = re.search(r"__shared__ (float4|float4_t|uint4) ", lines[-1])
            aligned = re.search(r"aligned\((16|\d{3,})\)", lines[-1])
            assert wide or aligned, f"{os.path.basename(path)}: {lines[-1].strip()}"
    assert seen >= 3


def test_a_logits_tiles_bias_lies_on_16_bytes(tmp_path):
    so = str(tmp_path / "host_shared.so")
    subprocess.run([HIPCC, "-x", "hip", "--offload-host-only", "-O1", "-std=c++17", "-fPIC", "-shared",
                    os.path.join(ROOT, "tests", "host_shared.hip"), "-o", so], check=True, capture_output=True)
    assert C.CDLL(so).host_xent_numbers_alignment() >= 16
