"""Host code of the products, compiled on its own: how a product is cut into tiles (cfa_tiles.h), and the
record of waits that ran out (cfa_ops.h)."""
import os
import subprocess

from paper_2607_18957_gb300 import build as cfa_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def run(tmp_path, name):
    exe = tmp_path / name
    subprocess.run([cfa_build._nvcc(), "-O2", "-std=c++17", "-Xcompiler", "-pthread",
                    "-I", cfa_build.INCLUDE, "-I", cfa_build.CSRC,
                    os.path.join(ROOT, "tests", name + ".cpp"), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[:2000] + r.stderr


def test_every_number_of_tokens_has_a_cut(tmp_path):
    """Results of 2 bytes and of 4, gated and not, one group and many, 1 to 2^31 - 1 tokens."""
    run(tmp_path, "tiles_check")


def test_threads_are_told_of_every_wait_that_ran_out(tmp_path):
    run(tmp_path, "op_counts_check")
