"""The division of a paged attention call's work (csrc/paged_plan.hpp) where sequences have more new tokens than keys,
checked on the host under the address and undefined-behaviour sanitizers."""
import os
import subprocess

from paper_2502_21231_amd import build as BLD

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_rows_without_keys_have_room_and_are_counted(tmp_path):
    exe = str(tmp_path / "paged_plan_rows")
    subprocess.run([BLD.host_cxx(), "-O1", "-g", "-std=c++17", "-Wall", "-fsanitize=address,undefined",
                    "-fno-sanitize-recover=undefined", os.path.join(ROOT, "tests", "native", "paged_plan_rows.cpp"), "-o", exe],
                   check=True, timeout=300)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr
