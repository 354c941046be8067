"""The gated projection's choice of tiles, on the host: which sizes take which, so that the tests of the kernels reach all of them."""
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SAN = ["-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-g", "-O1"]

# (M, D, F) and the sides of Forward's, dx's and dw's tiles: all of them beyond one step, and their last rows and columns not whole
SIDES = {(4090, 4088, 2040): (256, 256, 256), (4090, 4087, 2039): (256, 256, 256), (4300, 4085, 2041): (192, 192, 256), (2500, 2050, 1300): (128, 128, 128),
         (4100, 1032, 2080): (192, 128, 128)}


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("plan") / "gated_plan")
    subprocess.check_call(["g++", "-std=c++17", *SAN, "-I", os.path.join(ROOT, "paper_1804_04806_amd", "csrc"),
                           os.path.join(ROOT, "tests", "native", "gated_plan_driver.cpp"), "-o", out])

    def ask(cases):
        r = subprocess.run([out], input="\n".join(" ".join(map(str, c)) for c in cases) + "\n", capture_output=True, text=True, timeout=300)
        assert r.returncode == 0 and r.stderr == "", r.stderr[-2000:]
        lines = [tuple(map(int, line.split())) for line in r.stdout.splitlines()]
        return [lines[i:i + 3] for i in range(0, len(lines), 3)]
    return ask


@pytest.mark.parametrize("phases", [1, 6])
def test_sides(plans, phases):
    for (shape, sides), got in zip(SIDES.items(), plans([(*s, phases) for s in SIDES])):
        assert tuple(p[0] for p in got) == sides, shape
    all_sides = [set(sides[i] for sides in SIDES.values()) for i in range(3)]
    assert all_sides == [{128, 192, 256}, {128, 192, 256}, {128, 256}]


def test_tiles_cover_the_products(plans):
    """Tiles cover rows and columns with none too many; every split has a step at least."""
    rng = random.Random(1)
    cases = [(int(2 ** rng.uniform(0, 15)), int(2 ** rng.uniform(0, 13)), int(2 ** rng.uniform(0, 14)), rng.choice([1, 6])) for _ in range(3000)]
    for (M, D, F, phases), got in zip(cases, plans(cases)):
        half = -(-F // 64) * 64
        for i, (m, n, steps) in enumerate(((M, 2 * F, -(-(-(-D // 8) * 8) // 64)), (M, D, 2 * half // 64), (2 * half, D, -(-M // 64)))):
            side, tiles_m, tiles_n, splits = got[i]
            assert side in ((64, 128, 192, 256), (128, 192, 256), (128, 256))[i]
            cols = 128 if side <= 128 else 256
            assert (tiles_m - 1) * side < m <= tiles_m * side and (tiles_n - 1) * cols < n <= tiles_n * cols
            assert 1 <= splits <= steps * phases
