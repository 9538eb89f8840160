"""How the keys of a tile of the many-row attention are cut, on the CPU: the rule against whole numbers of any size, and that neither it nor what is summed for it is a matter of rounding -
the kernel that makes the pieces and the one that joins them work it out each for itself."""
import os
import random
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")
CSRC = os.path.join(ROOT, "paper_2501_16385_amd", "csrc")


def body(file, name):
    """The text of a function, from its name to the brace that closes it."""
    text = open(os.path.join(CSRC, file)).read()
    at = text.index(name)
    return text[at:text.index("\n}\n", at)]


def test_pieces_of_tiles(tmp_path):
    if shutil.which("g++") is None or not os.path.exists(os.path.join(ROCM, "include", "hip", "hip_runtime.h")):
        pytest.skip("needs g++ and the HIP runtime's headers")
    exe = str(tmp_path / "share_driver")
    subprocess.run(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROCM, "include"), "-I", os.path.join(ROOT, "include"), "-I", CSRC,
                    os.path.join(ROOT, "tests", "host", "share_driver.cpp"), "-o", exe], check=True)
    rng = random.Random(3)
    calls = [(0, 0, 1, 512), (0, 0, 1024, 256), (2 << 18, 1, 1, 512), ((1 << 18) * 2 * 256, 256, 1, 512), ((1 << 19) * (1 << 25), 1 << 25, 1, 512), (34 * 16, 16, 32, 512)]
    for _ in range(30000):
        kv_heads, blocks = rng.choice([1, 2, 3, 8, 16, 32, 64, 1024]), rng.choice([256, 512])
        tiles = min(round(2 ** rng.uniform(0, 25)), (1 << 25) // kv_heads)
        calls.append((tiles * rng.randint(0, round(2 ** rng.uniform(0, 19))) + rng.randint(0, tiles), tiles, kv_heads, blocks))
    res = subprocess.run([exe], input="\n".join(" ".join(map(str, c)) for c in calls), text=True, capture_output=True, timeout=120, check=True)
    for (twice, tiles, kv_heads, blocks), line in zip(calls, res.stdout.split()):
        share, n = int(line), max(1, tiles)
        fit = blocks // (n * kv_heads)
        if fit >= 2:
            assert share == max(4, -(-3 * twice // (5 * n * fit))), (twice, tiles, kv_heads, blocks, line)
        else:                                                  # (beyond 31 bits both lose their lower ones: 11 are left at the least)
            assert abs(share - 6 - twice // n) <= (0 if twice < 1 << 31 else 2 + twice // n >> 10), (twice, tiles, kv_heads, blocks, line)


def test_what_is_summed_for_it_is_summed_in_whole_numbers():
    for file, name in (("fbq_attend.h", "int many_share("), ("fbq_attend_plan.h", "int share_of_steps(")):
        assert not re.search(r"float|double|ceil", body(file, name)), name
