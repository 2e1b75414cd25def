"""How the attention of new tokens is dealt out (csrc/ha_chunk_plan.h), compiled for the host."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2412_14468_b200", "csrc")


def test_every_tile_is_taken_once(tmp_path):
    exe = str(tmp_path / "plan")
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-O2", "-I", CSRC, os.path.join(HERE, "chunk_plan_check.cpp"), "-o", exe], check=True)
    assert subprocess.run([exe], capture_output=True, text=True, timeout=300).stdout.strip() == "ok"
