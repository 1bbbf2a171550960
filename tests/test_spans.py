"""Which buffers of a call share memory (csrc/spans.h), against a map of the bytes.  No GPU."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_matrices_share_memory_where_their_bytes_do(tmp_path):
    exe = str(tmp_path / "driver")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=undefined", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_1912_09268_amd", "csrc"), os.path.join(ROOT, "tests", "spans_driver.cpp"), "-o", exe],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and r.stdout == "ok\n", r.stdout
