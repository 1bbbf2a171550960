"""Columns of a checkpoint (csrc/act_layout.h): pieces of rows stay within those that are its own, whatever the distance of rows, and
the kernels read q nowhere else.  No GPU."""
import os
import re
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1912_09268_amd", "csrc")


def test_pieces_stay_within_the_own_columns(tmp_path):
    exe = str(tmp_path / "driver")
    r = subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, os.path.join(ROOT, "tests", "act_layout_driver.cpp"), "-o", exe],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and r.stdout == "ok\n", r.stdout


def test_the_weight_gradient_reads_q_through_it():
    """Every place of q in act_linear.hip is taken by piece_at from the own columns: a place up to ld would be behind the memory of a
    checkpoint that is a part of a wider one."""
    source = open(os.path.join(CSRC, "act_linear.hip")).read()
    places = re.findall(r"= A\.q \+ (.*);", source)
    assert len(places) == source.count("A.q +") == 2
    assert all(p == "piece_at(c0 + q_col, A.q_columns, S::XW)" for p in places), places
    assert "a.q_columns = own_columns(n_channels);" in source
