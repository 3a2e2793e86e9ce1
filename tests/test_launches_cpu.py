"""What the library would launch (no GPU needed): seen by a program in the place of the HIP runtime's launch functions, and asked of the
header that chooses the kernels of an update's products."""
import os
import subprocess

import pytest

from paper_2509_13232_amd import binding as spo
from paper_2509_13232_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HERE = os.path.dirname(spo.LIB_PATH)


@pytest.mark.timeout(600)
def test_a_kernels_limit_of_lds_is_the_same_for_all_calls(tmp_path):
    if not os.path.exists(spo.LIB_PATH):
        build.build()
    exe = str(tmp_path / "launch")
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-w", "-rdynamic", "-I" + build.INCLUDE, "-I/opt/rocm/include",
                    os.path.join(ROOT, "tests", "san", "launch_driver.cpp"), "-o", exe, "-L" + HERE, "-l:" + os.path.basename(spo.LIB_PATH),
                    "-Wl,-rpath," + HERE, "-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib"], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-3000:]
    assert "limits are the kernels' own" in r.stdout


def test_sums_of_squares_have_room_whatever_tiles_leave_them(tmp_path):
    exe = str(tmp_path / "orth_choice")
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-Wall", "-Wextra",
                    "-I" + build.CSRC, os.path.join(ROOT, "tests", "san", "orth_choice_driver.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-3000:]
    assert "sums of squares have room" in r.stdout
