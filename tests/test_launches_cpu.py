"""What the library would launch (no GPU needed): seen by a program in the place of the HIP runtime's launch functions, and asked of the
header that chooses the kernels of an update's products."""
import os
import subprocess

import pytest

import update_kinds
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


@pytest.fixture(scope="module")
def orth_choice(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("orth") / "orth_choice")
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-Wall", "-Wextra",
                    "-I" + build.CSRC, os.path.join(ROOT, "tests", "san", "orth_choice_driver.cpp"), "-o", exe], check=True)

    def run(*args):
        r = subprocess.run([exe, *map(str, args)], capture_output=True, text=True, timeout=300)
        assert r.returncode == 0, r.stderr[-3000:]
        return r.stdout
    return run


def test_sums_of_squares_have_room_whatever_tiles_leave_them(orth_choice):
    assert "sums of squares have room" in orth_choice()


def test_the_stacks_of_the_gpu_tests_reach_every_kind_of_tiles(orth_choice):
    # (the product that updates X has no tiles of 192)
    reached = set()
    for batch, rows, cols, products, *kinds in update_kinds.STACKS:
        assert orth_choice(batch, rows, cols, products).split() == kinds, (batch, rows, cols, products)
        assert orth_choice(batch, cols, rows, products).split() == kinds
        reached |= {(products, which, kind) for which, kind in enumerate(kinds)}
    assert len(reached) == 2 * (4 + 4 + 3)
