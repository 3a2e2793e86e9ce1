"""Normalisations and AdamW steps on the host, at their edges (no GPU needed)."""
import os
import subprocess

import pytest
import torch

from paper_2509_13232_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


# ---------------------------------------------------------------- 8-bit codes
@pytest.fixture(scope="module")
def tops(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("state8") / "top")
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-Wall", "-Wextra", "-I" + build.CSRC,
                    os.path.join(ROOT, "tests", "san", "state8_top_driver.cpp"), "-o", exe], check=True)

    def run(blocks, mantissa):
        """[(scale, whether all is NaN)] of blocks of 64 numbers, as bits."""
        text = "\n".join(f"{mantissa} " + " ".join(f"{u:x}" for u in b) for b in blocks)
        r = subprocess.run([exe], input=text, capture_output=True, text=True, timeout=300)
        assert r.returncode == 0, r.stderr[-3000:]
        return [tuple(int(v) for v in line.split()) for line in r.stdout.splitlines()]
    return run


@pytest.mark.parametrize("mantissa", [3, 4])
def test_every_nan_and_infinity_spoils_its_block(tops, mantissa):
    # NaNs of any sign and payload: memory filled with ones is one of them
    bad = [0x7f800000, 0x7f800001, 0x7fc00000, 0x7fffffff, 0xff800000, 0xff800001, 0xffc00000, 0xffefffff, 0xfff00000, 0xfff00001, 0xfff80000, 0xfff80001, 0xffff0000,
           0xffffffff]
    if mantissa == 4:
        bad.remove(0xff800000)       # (no root is -infinity; -NaN is what a root of a NaN may be)
    ones = [0x3f800000 + i for i in range(64)]
    blocks = [ones[:i % 64] + [u] + ones[i % 64 + 1:] for i, u in enumerate(bad)]
    assert tops(blocks, mantissa) == [(255, 1)] * len(bad)
    assert tops([[u] * 64 for u in bad], mantissa) == [(255, 1)] * len(bad)
    # the largest number that a block holds, and the next one
    largest = 0x7f800000 - (1 << (23 - mantissa))
    assert tops([ones[1:] + [largest]], mantissa) == [(254, 0)] and tops([ones[1:] + [largest + 1]], mantissa) == [(255, 1)]
    assert tops([ones, [0] * 64, [1] * 64], mantissa) == [(127, 0), (15, 0), (15, 0)]
