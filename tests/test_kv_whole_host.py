"""The attention's workgroups that take a whole sequence, walked on the CPU (tests/c/kv_whole.cpp)."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_whole_sequences_are_met_once_inside_their_pages(tmp_path):
    exe = str(tmp_path / "kv_whole")
    cmd = ["g++", "-std=c++17", "-O2", "-Wall", "-Wextra", "-Werror", "-I",
           os.path.join(ROOT, "paper_2606_17059_amd", "csrc"), os.path.join(ROOT, "tests", "c", "kv_whole.cpp"), "-o", exe]
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout
    r = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=120)
    assert r.returncode == 0 and "kv_whole: ok" in r.stdout, r.stdout
