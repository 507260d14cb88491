"""How a product is cut into tiles, on the host: cfa_tiles.h compiled on its own."""
import os
import subprocess

from paper_2607_18957_gb300 import build as cfa_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_every_number_of_tokens_has_a_cut(tmp_path):
    """Results of 2 bytes and of 4, gated and not, one group and many, 1 to 2^31 - 1 tokens."""
    exe = tmp_path / "tiles_check"
    subprocess.run([cfa_build._nvcc(), "-O2", "-std=c++17", "-I", cfa_build.INCLUDE,
                    "-I", cfa_build.CSRC, os.path.join(ROOT, "tests", "tiles_check.cpp"),
                    "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[:2000] + r.stderr
