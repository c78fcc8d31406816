"""What the kernels of the operators for language models ask for, computed on the CPU from their own headers and sources."""
import os
import re
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2010_08679_amd", "csrc")


def test_a_products_scales_are_read_within_their_arrays(tmp_path):
    exe = str(tmp_path / "scale_fetch")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, os.path.join(ROOT, "tests", "c", "lm_scale_fetch.cpp"), "-o", exe])
    out = subprocess.run([exe], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout + out.stderr


def test_loads_into_lds_state_what_they_change():
    # the place in LDS is a register that the compiler may use as well, from one statement to the next
    source = open(os.path.join(CSRC, "lm_product.hip")).read()
    loads = [s for s in re.findall(r"asm volatile\((.*?)\);", source, flags=re.S) if "buffer_load" in s]
    assert loads
    for s in loads:
        text = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', s))
        assert text.startswith("s_mov_b32 m0, %0") and re.search(r':\s*"m0"', s), s
